"""Attention of several new tokens where a result can go wrong without a crash: infinite values."""
import math

import pytest

torch = pytest.importorskip("torch")

import cache_reference as ref  # noqa: E402
from test_gpu_cache import check, cuda, make, mk  # noqa: E402, F401

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def put_values(args, h, odd):
    """odd: (sequence, position, channel, value) of kv head h."""
    ps = args["v_cache"].shape[2]
    for b, pos, ch, x in odd:
        args["v_cache"][int(args["table"][b, pos // ps]), h, pos % ps, ch] = x


# ---- infinite values ----

@pytest.mark.parametrize("new,hq,D,dtype", [([4], 4, 128, F16), ([5], 16, 64, BF16), ([3], 2, 256, F16), ([130], 1, 64, F16), ([200], 1, 128, BF16),
                                            ([130], 1, 96, BF16)])
@pytest.mark.parametrize("cached", [700, 1100, 1500, 2100, 3000, 4100, 9000])
def test_infinite_values_of_shared_keys(mk, new, hq, D, dtype, cached):
    """Keys in any number of parts, an infinity in the first, one in the middle and one in the last."""
    n = cached + new[0]
    args = make(cached + D, [n], new, hq, 1, D, 32, dtype, 16)
    args["q"] *= 0.25  # no weight far below the others
    put_values(args, 0, [(0, 0, 3, math.inf), (0, 1, 5, -math.inf), (0, cached // 2, 7, math.inf), (0, cached - 1, 9, -math.inf), (0, 2, 11, math.nan)])
    check(mk, args)


@pytest.mark.parametrize("new,hq,hkv,D,dtype", [([4], 4, 1, 128, F16), ([3, 2], 8, 2, 64, F16), ([4], 4, 1, 128, BF16), ([6], 3, 1, 256, F16), ([4], 4, 2, 96, F16),
                                                ([130], 1, 1, 64, F16), ([140, 90], 4, 2, 128, F16), ([130], 1, 1, 128, BF16), ([130], 1, 1, 96, F16),
                                                ([130], 2, 1, 256, F16)])
@pytest.mark.parametrize("cached", [200, 3000])
@pytest.mark.parametrize("far", [26.0, 32.0, 60.0])
def test_infinite_values_of_small_weights(mk, new, hq, hkv, D, dtype, cached, far):
    """An infinite value is one however far its key is below the row's maximum, in steps that all rows see too; and only in its channel."""
    args = make(cached, [cached + n for n in new], new, hq, hkv, D, 16, dtype, 16, junk=False)
    args["q"].zero_()
    args["q"][..., 0] = 8.0
    args["k_cache"].zero_()
    for b in range(len(new)):
        pos = cached // 3
        args["k_cache"][int(args["table"][b, pos // 16]), :, pos % 16, 0] = far * D ** 0.5 / 8
        for h in range(hkv):
            put_values(args, h, [(b, 1, 3, math.inf), (b, cached // 2, 5, -math.inf), (b, cached - 1, 7, math.inf), (b, pos, 9, -math.inf),
                                 (b, 40, 11, math.nan), (b, cached - 20, 13, math.inf), (b, 50, 13, -math.inf)])
    check(mk, args)
    check(mk, args, window=cached - 5, sinks=3)

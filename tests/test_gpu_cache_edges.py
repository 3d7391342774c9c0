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

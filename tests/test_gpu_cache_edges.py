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


# ---- weights ----

# A weight's relative error in the second product.  Up to 64 rows, in two parts: the first is rounded down, which leaves less than an ulp of it
# (2^-10, 2^-7), and the rest to nearest (half an ulp of that: 2^-11, 2^-8).  More rows: rounded once.
TWO, ONE = {F16: 2.0 ** -21, BF16: 2.0 ** -15}, {F16: 2.0 ** -11, BF16: 2.0 ** -8}
# Its absolute one, of the largest weight of the row (times the scale of its block's values): float16's are times 2^11 (in two parts 2^11 to
# 2^15), where half a subnormal's step is 2^-25.
LOST = {F16: 2.0 ** -36, BF16: 2.0 ** -122}


def exact(args):
    """out, lse and the bounds of their errors of one sequence's new tokens over one kv head, in 64 bits."""
    q, (n, H, D), ps = args["q"].double(), args["q"].shape, args["k_cache"].shape[2]
    L = int(args["lengths"][0])
    j = torch.arange(L)
    page, slot = args["table"][0, j // ps].long(), j % ps
    keys, values = (args[x][page, 0, slot].float().double() for x in ("k_cache", "v_cache"))
    ks = vs = torch.ones(L, 1, dtype=torch.float64)
    if args["scales"] is not None:
        ks, vs = (args["scales"][page, 0, which, slot // 16].double()[:, None] for which in (0, 1))
    u, tiny, dt = ref.U[args["q"].dtype], ref.TINY[args["q"].dtype], args["q"].dtype
    sees = (j <= torch.arange(L - n, L)[:, None])[:, None]
    products, size = (torch.einsum("nhd,jd->nhj", a, b) for a, b in ((q, keys * ks), (q.abs(), (keys * ks).abs())))
    s = (products * D ** -0.5).masked_fill(~sees, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m)
    total = e.sum(-1, keepdim=True)
    out = torch.einsum("nhj,jd->nhd", e, values * vs) / total
    lse = (m + torch.log(total))[..., 0]
    off = D * 2.0 ** -24 * size.amax() * D ** -0.5 + 2.0 ** -21 * s.masked_fill(~sees, 0).abs().amax()
    spread = torch.einsum("nhj,jd->nhd", e, (values * vs).abs()) / total
    eight = 0 if args["scales"] is None else 2.0 ** -16
    lost = LOST[dt] * (e * vs[:, 0]).amax(-1, keepdim=True) * torch.einsum("nhj,jd->nhd", sees.double().expand_as(e), values.abs()) / total
    weight = (TWO if n * H <= 64 else ONE)[dt]
    tol = u * out.abs() + tiny + (weight + 2 * off + 2.0 ** -18 + eight) * spread + lost
    return out, lse, tol, off + 2.0 ** -21 * (1 + lse.abs()) + 2.0 ** -20 + eight


def held_to(mk, args):
    want, want_lse, tol, tol_lse = exact(args)
    got, lse = mk.cache_attention(**cuda(args), return_lse=True)
    over = ((got.cpu().double() - want).abs() / tol).max()
    assert over <= 1 and ((lse.cpu().double() - want_lse).abs() <= tol_lse).all(), float(over)


FEW = [([3], 4), ([1], 1), ([10], 3), ([32], 2)]
MANY = [([130], 1), ([40], 4)]


@pytest.mark.parametrize("new,hq", FEW + MANY)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("n", [60, 300, 3000])
def test_weights_of_values_that_cancel(mk, new, hq, dtype, D, bits, n):
    """Values of either sign: where they add up to about nothing an error of the weights stands out against the output's rounding."""
    held_to(mk, make(n + D, [n + new[0]], new, hq, 1, D, 32, dtype, bits, junk=False))


@pytest.mark.parametrize("new,hq,n", [([3], 4, 131071), ([3], 4, 20000), ([40], 1, 20000), ([130], 1, 60000), ([40], 4, 8000), ([1], 1, 131071)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("gap", [12.0, 16.0, 17.5, 19.0])
@pytest.mark.parametrize("bits,D", [(8, 64), (16, 64), (16, 128)])
def test_weights_of_many_keys_far_below_one(mk, new, hq, n, dtype, gap, bits, D):
    """One key whose value is zero, `gap` above all others: what the others' small weights add up to is the whole output."""
    args = make(n, [n], new, hq, 1, D, 64, dtype, bits, junk=False)
    args["q"].zero_()
    args["q"][..., 0] = 8.0
    g = torch.Generator().manual_seed(n)
    k, v = torch.zeros(args["k_cache"].shape), 0.5 + torch.rand(args["v_cache"].shape, generator=g)
    page, slot = int(args["table"][0, n // 2 // 64]), n // 2 % 64
    k[page, 0, slot, 0] = gap * D ** 0.5 / 8
    v[page, 0, slot] = 0
    args["k_cache"], args["v_cache"] = k.to(args["k_cache"].dtype), v.to(args["v_cache"].dtype)
    if bits == 8:
        args["scales"].fill_(1)
    held_to(mk, args)


@pytest.mark.parametrize("new,hq", FEW + MANY)
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("apart", [20, 30, 45])
def test_weights_of_scales_far_apart(mk, new, hq, dtype, apart):
    """Blocks of values 2^20 to 2^45 larger than the others, but zero in half of the channels: there the others are the output, as far as weights
    times scales go."""
    n, D = 500, 64
    args = make(n, [n], new, hq, 1, D, 32, dtype, 8, junk=False)
    args["scales"][:, :, 1] = 2.0 ** -(apart // 2)
    for b in (0, 7):
        page = int(args["table"][0, b])
        args["scales"][page, 0, 1, 0] = 2.0 ** (apart - apart // 2) if dtype == BF16 else 2.0 ** (4 if apart < 30 else 6)
        v = args["v_cache"][page, 0, :16].float()
        v[:, ::2] = 0
        args["v_cache"][page, 0, :16] = v.to(torch.float8_e4m3fn)
    if dtype == F16:
        args["scales"][:, :, 1] = torch.where(args["scales"][:, :, 1] < 1, 2.0 ** (4 - apart if apart < 30 else 6 - apart), args["scales"][:, :, 1])
    held_to(mk, args)

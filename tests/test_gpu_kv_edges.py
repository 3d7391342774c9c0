"""The paged key-value cache operators where a result can go wrong without a
crash: weights far below a row's maximum, infinite values, and the limits of
sizes and lengths.  References are 64-bit forms written here or in kv_reference.py.
"""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import kv_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
# a softmax weight's relative error in the second product: its first part is rounded down, which leaves less than an ulp of it (2^-10,
# 2^-7), and the rest is rounded to nearest (half an ulp of that: 2^-11, 2^-8)
WEIGHT = {F16: 2.0 ** -21, BF16: 2.0 ** -15}
LOST = {F16: 2.0 ** -40, BF16: 2.0 ** -126}  # and its absolute one, of the row's maximum


@pytest.fixture(scope="module")
def mk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2408_11743_amd as mk
    mk.lib()
    return mk


def gen(seed):
    return torch.Generator().manual_seed(seed)


def paged(x, ps):
    """[n, heads, D] tokens of one sequence as pages [pages, heads, ps, D], whose last slots hold NaN."""
    n, heads, D = x.shape
    pages = -(-n // ps)
    out = torch.full((pages * ps, heads, D), math.nan, dtype=x.dtype)
    out[:n] = x
    return out.view(pages, ps, heads, D).transpose(1, 2).contiguous()


def one_sequence(mk, q, keys, values, ps=64, **kw):
    """Attention of q [heads, D] over keys and values [n, kv heads, D] in pages in order: out and lse, 64 bits."""
    k, v = paged(keys, ps).cuda(), paged(values, ps).cuda()
    table = torch.arange(k.shape[0], dtype=torch.int32, device="cuda")[None]
    lengths = torch.tensor([len(keys)], dtype=torch.int32, device="cuda")
    out, lse = mk.paged_attention(q[None].cuda(), k, v, table, lengths, return_lse=True, **kw)
    return out[0].cpu().double(), lse[0].cpu().double()


def exact(q, keys, values):
    """out, lse and the bounds of their errors: weights held to WEIGHT and LOST, everything else as in kv_reference.py."""
    heads, D = q.shape
    kv_heads = keys.shape[1]
    u, tiny = ref.U[q.dtype], ref.TINY[q.dtype]
    out, tol = torch.zeros(heads, D, dtype=torch.float64), torch.zeros(heads, D, dtype=torch.float64)
    lse, tol_lse = torch.zeros(heads, dtype=torch.float64), torch.zeros(heads, dtype=torch.float64)
    for h in range(heads):
        kvh = h // (heads // kv_heads)
        products = keys[:, kvh].double() * q[h].double()
        s = products.sum(1) * D ** -0.5
        e = torch.exp(s - s.max())
        total, v = e.sum(), values[:, kvh].double()
        out[h] = (e[:, None] * v).sum(0) / total
        lse[h] = s.max() + torch.log(total)
        off = D * 2.0 ** -24 * float(products.abs().sum(1).max()) * D ** -0.5 + 2.0 ** -21 * float(s.abs().max())
        spread = (e[:, None] * v.abs()).sum(0) / total
        tol[h] = u * out[h].abs() + tiny + (WEIGHT[q.dtype] + 2 * off + 2.0 ** -18) * spread + LOST[q.dtype] * v.abs().sum(0) / total
        tol_lse[h] = off + 2.0 ** -21 * (1 + abs(float(lse[h]))) + 2.0 ** -20
    return out, lse, tol, tol_lse


# ---- softmax weights ----

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("n", [2, 40, 700])
def test_attention_of_values_that_cancel(mk, dtype, D, n):
    """Values of either sign around zero: an error of the weights stands out against the output's rounding."""
    g = gen(D + n)
    q = torch.randn(4, D, generator=g).to(dtype)
    keys = torch.randn(n, 2, D, generator=g).to(dtype)
    values = torch.randn(n, 2, D, generator=g).to(dtype)
    out, _, _, _ = exact(q, keys, values)
    # one more key of weight close to the rest's takes the sum to about zero
    values[0] -= (out.view(2, 2, D).mean(1) * n / 2).to(dtype)
    want, want_lse, tol, tol_lse = exact(q, keys, values)
    got, lse = one_sequence(mk, q, keys, values)
    assert ((got - want).abs() <= tol).all()
    assert ((lse - want_lse).abs() <= tol_lse).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n,gap", [(131071, 17.5), (131071, 14.0), (20000, 16.0), (8192, 17.0), (100, 12.0)])
@pytest.mark.parametrize("at", [0.0, 0.6])
def test_attention_of_many_keys_far_below_one(mk, dtype, n, gap, at):
    """One key whose value is zero, `gap` above all others: what the others' small weights add up to is the whole output."""
    D, g = 64, gen(n)
    q = torch.zeros(2, D).to(dtype)
    q[:, 0] = 8.0
    keys = torch.zeros(n, 1, D).to(dtype)
    keys[int(at * n), 0, 0] = gap
    values = (0.5 + torch.rand(n, 1, D, generator=g)).to(dtype)
    values[int(at * n)] = 0
    want, want_lse, tol, tol_lse = exact(q, keys, values)
    got, lse = one_sequence(mk, q, keys, values)
    assert ((got - want).abs() <= tol).all()
    assert ((lse - want_lse).abs() <= tol_lse).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("n", [1, 40, 3000])
@pytest.mark.parametrize("equal", [True, False])
def test_attention_of_infinite_values(mk, dtype, D, n, equal):
    """A weight above zero times an infinity is that infinity, whatever is left of the weight beside its first part
    (`equal`: weights of one, of which nothing is left); of both signs it is no number; other channels do not see it."""
    g = gen(D + n)
    q = torch.zeros(2, D).to(dtype) if equal else torch.randn(2, D, generator=g).to(dtype)
    keys = torch.randn(n, 1, D, generator=g).to(dtype)
    values = torch.randn(n, 1, D, generator=g).to(dtype)
    want, _, tol, _ = exact(q, keys, values)
    values[n // 2, 0, 3] = math.inf
    values[n // 3, 0, D - 1] = -math.inf
    values[n // 2, 0, 9] = math.nan
    if n > 1:
        values[0, 0, 5], values[n - 1, 0, 5] = math.inf, -math.inf
    got, _ = one_sequence(mk, q, keys, values)
    assert (got[:, 3] == math.inf).all() and (got[:, D - 1] == -math.inf).all() and torch.isnan(got[:, 9]).all()
    rest = [c for c in range(D) if c not in (3, 9, D - 1) + ((5,) if n > 1 else ())]
    assert n == 1 or torch.isnan(got[:, 5]).all()
    assert ((got - want).abs()[:, rest] <= tol[:, rest]).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 40, 300, 3000, 12000])
def test_attention_without_any_weight_is_zero(mk, dtype, D, n):
    """Every score -inf: zero and -inf, also where the values are infinite or no numbers, in one piece or many."""
    q = torch.ones(16, D).to(dtype)
    keys = torch.full((n, 1, D), -math.inf).to(dtype)
    values = torch.randn(n, 1, D, generator=gen(n)).to(dtype)
    values[n // 2] = math.inf
    values[n // 3, 0, ::2] = math.nan
    out, lse = one_sequence(mk, q, keys, values)
    assert (out == 0).all() and (lse == -math.inf).all()


# ---- page scores ----

def select_by_definition(q, bounds, table, lengths, ps, count):
    """marlin.h's formula as it stands, in 64 bits: the bound a channel's sign does not ask for is not looked at."""
    kv_heads, group = bounds.shape[1], q.shape[1] // bounds.shape[1]
    chosen = torch.full((len(lengths), kv_heads, count), -1, dtype=torch.int32)
    for b, n in enumerate(lengths.tolist()):
        used = -(-n // ps)
        for h in range(kv_heads):
            rank = []
            for i in range(used):
                page = int(table[b, i])
                if not 0 <= page < bounds.shape[0]:
                    rank.append((2, 0.0, i))
                    continue
                x = q[b, h * group:(h + 1) * group].double()
                lo, hi = bounds[page, h].double()
                s = torch.where(x > 0, x * hi, x * lo).sum(1)
                rank.append((0 if torch.isnan(s).any() else 1, -float(s.max()), i))
            rank = [(r, 0.0 if r != 1 else s, i) for r, s, i in rank]
            best = list(range(used)) if used <= count else sorted([used - 1] + [i for _, _, i in sorted(rank[:-1])[:count - 1]])
            chosen[b, h, :len(best)] = table[b, best]
    return chosen


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("sign", [1, -1])
def test_select_looks_at_the_bound_that_the_sign_asks_for(mk, dtype, sign):
    """Six pages whose nearer bound is 0 .. 5, page 0's farther one infinite: the best are the last ones."""
    q = torch.zeros(1, 1, 64).to(dtype)
    q[0, 0, 0] = sign
    bounds = torch.zeros(6, 1, 2, 64).to(dtype)
    bounds[:, 0, 1 if sign > 0 else 0, 0] = sign * torch.arange(6).to(dtype)
    bounds[0, 0, 0 if sign > 0 else 1, 0] = -sign * math.inf
    table = torch.arange(6, dtype=torch.int32)[None]
    lengths = torch.tensor([96], dtype=torch.int32)
    got, _ = mk.select_pages(q.cuda(), bounds.cuda(), table.cuda(), lengths.cuda(), 16, 3)
    assert got.flatten().tolist() == [3, 4, 5]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (17, 1), (40, 2)])
@pytest.mark.parametrize("zeros", [0.0, 0.8])
def test_select_by_its_definition(mk, dtype, D, hq, hkv, zeros):
    """Infinities and NaN in either bound or both, under queries of either sign and of zero; small integers elsewhere."""
    g = gen(D + hq)
    lengths, ps, count = torch.tensor([800, 33, 1500], dtype=torch.int32), 16, 9
    used = [-(-n // ps) for n in lengths.tolist()]
    pages = sum(used) + 1
    table = torch.full((3, max(used)), -1, dtype=torch.int32)
    perm = torch.randperm(pages, generator=g).int()
    for b, n in enumerate(used):
        table[b, :n] = perm[sum(used[:b]):sum(used[:b]) + n]
    table[2, 4] = pages + 3
    q = torch.randint(1, 3, (3, hq, D), generator=g) * (2 * torch.randint(0, 2, (3, 1, D), generator=g) - 1)
    q = (q * (torch.rand(q.shape, generator=g) >= zeros)).to(dtype)
    a, b = torch.randint(-3, 4, (2, pages, hkv, D), generator=g)
    bounds = torch.stack([torch.minimum(a, b), torch.maximum(a, b)], 2).to(dtype)
    odd = torch.tensor([math.inf, -math.inf, math.nan])
    for p in range(0, pages, 3):
        side, c = int(torch.randint(0, 3, (1,), generator=g)), int(torch.randint(0, D, (1,), generator=g))
        for one in ((0,), (1,), (0, 1))[side]:
            bounds[p, :, one, c] = odd[p // 3 % 3].to(dtype)
    got, _ = mk.select_pages(q.cuda(), bounds.cuda(), table.cuda(), lengths.cuda(), ps, count)
    assert torch.equal(got.cpu(), select_by_definition(q, bounds, table, lengths, ps, count))


# ---- limits ----

@pytest.mark.parametrize("D,hkv,short", [(256, 2, 0), (256, 2, 47), (256, 5, 1), (128, 3, 0)])
def test_attention_of_the_longest_sequence(mk, D, hkv, short):
    """2^30 tokens (a table may name a page many times): the row that a step belongs to is found where the steps of 64 rows pass
    32 bits.  Weights are all one and values small integers, so that sums are exact until pieces are joined."""
    ps, n = 1024, (1 << 30) - short
    g = gen(D + hkv)
    values = torch.randint(-3, 4, (2, hkv, ps, D), generator=g)
    table = torch.randint(0, 2, (1, n // ps + (n % ps > 0)), generator=g, dtype=torch.int32)
    k = torch.zeros(2, hkv, ps, D, dtype=BF16, device="cuda")
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = torch.zeros(1, hkv, D, dtype=BF16, device="cuda")
    out, lse = mk.paged_attention(q, k, values.to(BF16).cuda(), table.cuda(), lengths, return_lse=True)
    torch.cuda.synchronize()
    left = ps - short if short else ps
    named = torch.bincount(table[0, :-1].long(), minlength=2).double()
    total = (named[:, None, None] * values.sum(2)).sum(0) + values[table[0, -1], :, :left].sum(1)
    size = (named[:, None, None] * values.abs().sum(2)).sum(0) + values[table[0, -1], :, :left].abs().sum(1)
    want, spread = total.double() / n, size.double() / n
    assert ((out[0].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * spread).all()
    assert ((lse[0].cpu().double() - math.log(n)).abs() <= 2.0 ** -18).all()


def test_append_of_more_threads_than_a_launch_takes(mk):
    """22000 pages of 1024 + 1024 heads: 1.01 * 2^32 threads.  Most sequences' entries name no page; a few do, the last ones too."""
    n, heads, D, ps = 11000, 1024, 64, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    row = torch.randn(3, 1, heads, D, dtype=F16, device="cuda", generator=g)
    q, k, v = (x.expand(2 * n, heads, D) for x in row)
    real = [0, 1, 5000, n - 2, n - 1]
    table = torch.full((n, 2), -1, dtype=torch.int32)
    table[real] = torch.arange(2 * len(real), dtype=torch.int32).view(-1, 2)
    kc, vc, bounds = mk.kv_cache(2 * len(real), heads, ps, D, bounds=True)
    angles = mk.rotation_table(17, D)
    lengths = torch.full((n,), 17, dtype=torch.int32, device="cuda")
    starts = torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device="cuda")
    out = mk.kv_append(q, k, v, kc, vc, table.cuda(), lengths, angles, starts, bounds=bounds)
    # the same two tokens by themselves
    kc1, vc1, bounds1 = mk.kv_cache(2, heads, ps, D, bounds=True)
    one = mk.kv_append(q[:2], k[:2], v[:2], kc1, vc1, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"), lengths[:1], angles,
                       starts[:2], bounds=bounds1)
    torch.cuda.synchronize()
    for i, b in enumerate(real):
        assert torch.equal(out[2 * b:2 * b + 2], one)
        for a, c in ((kc, kc1), (vc, vc1), (bounds, bounds1)):
            assert torch.equal(a[2 * i:2 * i + 2], c)
        out[2 * b:2 * b + 2] = 0
    assert not out.any()


def test_select_of_more_threads_than_a_launch_takes(mk):
    """2^23 rows of 512 threads, the most that marlin.h admits: the same 64 sequences over and over."""
    times, n, heads, D, ps = 1024, 64, 128, 64, 16
    g = torch.Generator(device="cuda").manual_seed(6)
    q = torch.randn(1, heads, D, dtype=F16, device="cuda", generator=g)
    bounds = torch.randn(20, heads, 2, D, dtype=F16, device="cuda", generator=g)
    table = torch.randint(0, 20, (n, 4), device="cuda", generator=g).int()
    lengths = torch.randint(0, 65, (n,), device="cuda", generator=g).int()
    want, want_n = mk.select_pages(q.expand(n, heads, D), bounds, table, lengths, ps, 3)
    got, got_n = mk.select_pages(q.expand(times * n, heads, D), bounds, table.repeat(times, 1), lengths.repeat(times), ps, 3)
    assert torch.equal(got.view(times, n, heads, 3), want.expand(times, n, heads, 3))
    assert torch.equal(got_n, want_n.repeat(times))


def test_append_past_the_largest_table(mk):
    """A table of 2^30 tokens: positions from there on have no place, and do not take the last slot's."""
    ps, width, D = 1024, 1 << 20, 64
    kc, vc = mk.kv_cache(4, 1, ps, D)
    table = torch.zeros(2, width, dtype=torch.int32, device="cuda")
    table[0, -1], table[1, -1] = 2, 3
    new = torch.randn(3, 6, 1, D, device="cuda").half()
    for length in (2 ** 30 + 1, 2 ** 30 + 1024, 2 ** 31 - 1):
        lengths = torch.tensor([length, 2 ** 30], dtype=torch.int32, device="cuda")
        kc.zero_()
        q = mk.kv_append(new[0, :2], new[1, :2], new[2, :2], kc, vc, table, lengths)
        assert not q[0].any() and torch.equal(q[1], new[0, 1])
        assert torch.equal(kc[3, 0, -1], new[1, 1, 0])
        kc[3, 0, -1] = 0
        assert not kc.any()
    # prompts: four tokens of which two are past it, and two that are all
    lengths = torch.tensor([2 ** 30 + 2, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 4, 6], dtype=torch.int32, device="cuda")
    q = mk.kv_append(new[0], new[1], new[2], kc, vc, table, lengths, starts=starts)
    assert torch.equal(q[:2], new[0, :2]) and not q[2:].any()
    assert torch.equal(kc[2, 0, -2:], new[1, :2, 0])
    kc[2, 0, -2:] = 0
    assert not kc.any()


# ---- refusals ----

def test_a_workspace_elsewhere_is_refused(mk):
    q = torch.zeros(1, 2, 64, dtype=F16, device="cuda")
    k, v, bounds = mk.kv_cache(2, 1, 16, 64, bounds=True)
    table, lengths = torch.zeros(1, 2, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    host = mk.Workspace("cpu", nbytes=1 << 24)
    with pytest.raises(ValueError, match="workspace"):
        mk.paged_attention(q, k, v, table, lengths, workspace=host)
    with pytest.raises(ValueError, match="workspace"):
        mk.select_pages(q, bounds, table, lengths, 16, 1, workspace=host)


# ---- HIP errors ----

def small_call(mk):
    """Arguments of the three calls: two sequences of 40 and 50 tokens."""
    q = torch.randn(2, 4, 64, device="cuda").half()
    kv = torch.randn(2, 2, 64, device="cuda").half()
    k, v, bounds = mk.kv_cache(8, 2, 16, 64, bounds=True)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    lengths = torch.tensor([40, 50], dtype=torch.int32, device="cuda")
    return q, kv, k, v, bounds, table, lengths


def test_a_hip_error_raises_and_is_not_tried_again(mk):
    from paper_2408_11743_amd import _fast, kv, ops
    q, new, k, v, bounds, table, lengths = small_call(mk)
    mk.paged_attention(q, k, v, table, lengths)  # the stream's workspace is there
    mk.select_pages(q, bounds, table, lengths, 16, 2)
    calls = []
    stub = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p)(lambda args, stream: calls.append(0) or 6)
    at = ctypes.cast(stub, ctypes.c_void_p).value
    _fast.connect(at, at, at, kv._raw_stream, ops._default_ws, mk.MarlinError)
    try:
        for n, call in enumerate((lambda: mk.kv_append(q, new, new, k, v, table, lengths),
                                  lambda: mk.paged_attention(q, k, v, table, lengths, return_lse=True),
                                  lambda: mk.select_pages(q, bounds, table, lengths, 16, 2))):
            with pytest.raises(mk.MarlinError) as e:
                call()
            assert e.value.status == 6 and len(calls) == n + 1
    finally:
        kv._connect()
    assert mk.kv_append(q, new, new, k, v, table, lengths).shape == q.shape


def test_an_error_that_another_call_left_is_not_this_ones(mk):
    """hipSetDevice of a device that there is not leaves an error on the thread; an append in place rotates once all the same."""
    hip = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
    hip = ctypes.CDLL(hip)
    q, new, k, v, bounds, table, lengths = small_call(mk)
    angles = mk.rotation_table(64, 64)
    want = mk.kv_append(q, new, new, k, v, table, lengths, angles)
    o = mk.paged_attention(want, k, v, table, lengths)
    pages, _ = mk.select_pages(want, bounds, table, lengths, 16, 2)
    torch.cuda.synchronize()
    try:
        assert hip.hipSetDevice(9999) != 0
        got = mk.kv_append(q, new, new, k, v, table, lengths, angles, out=q)
        assert hip.hipSetDevice(9999) != 0
        o2 = mk.paged_attention(q, k, v, table, lengths)
        assert hip.hipSetDevice(9999) != 0
        pages2, _ = mk.select_pages(q, bounds, table, lengths, 16, 2)
    finally:
        hip.hipGetLastError()
    assert torch.equal(got, want) and torch.equal(o2, o) and torch.equal(pages2, pages)


# ---- gradients, tangents, modes, traces, transforms ----

def test_a_gradient_is_not_dropped(mk):
    q, new, k, v, bounds, table, lengths = small_call(mk)
    want = mk.kv_append(q, new, new, k, v, table, lengths)
    o, lse = mk.paged_attention(want, k, v, table, lengths, return_lse=True)
    x = q.clone().requires_grad_()
    for y in (mk.kv_append(x, new, new, k, v, table, lengths), mk.paged_attention(x, k, v, table, lengths),
              mk.paged_attention(x, k, v, table, lengths, return_lse=True)[1],
              mk.paged_attention(x * 1, k, v, table, lengths, out=torch.empty_like(q))):
        assert y.requires_grad
        with pytest.raises(RuntimeError, match="autograd"):
            y.float().sum().backward()
    with torch.no_grad():
        assert torch.equal(mk.kv_append(x, new, new, k, v, table, lengths), want)
        assert torch.equal(mk.paged_attention(want.clone().requires_grad_(), k, v, table, lengths), o)
    with torch.inference_mode():
        assert torch.equal(mk.paged_attention(x, k, v, table, lengths), mk.paged_attention(q, k, v, table, lengths))
    with pytest.raises(ValueError, match="out"):
        mk.paged_attention(x, k, v, table, lengths, out=torch.empty(3, 2, 4, 64, dtype=F16, device="cuda"))
    pages, n = mk.select_pages(x, bounds, table, lengths, 16, 2)
    assert not pages.requires_grad and pages.shape == (2, 2, 2)


def test_a_tangent_is_refused(mk):
    import torch.autograd.forward_ad as fwd
    q, new, k, v, bounds, table, lengths = small_call(mk)
    with fwd.dual_level():
        x = fwd.make_dual(q, torch.ones_like(q))
        for call in (lambda: mk.kv_append(x, new, new, k, v, table, lengths), lambda: mk.paged_attention(x, k, v, table, lengths),
                     lambda: torch.ops.marlin_mi355x.paged_attention(x, k, v, table, lengths)):
            with pytest.raises(RuntimeError, match="derivative"):
                call()
        assert mk.paged_attention(q, k, v, table, lengths).shape == q.shape


def test_modes_traces_and_transforms_see_the_calls(mk):
    from torch.utils._python_dispatch import TorchDispatchMode
    q, new, k, v, bounds, table, lengths = small_call(mk)
    seen = []

    class Record(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            seen.append(str(func))
            return func(*args, **(kwargs or {}))

    def step(x):
        y = mk.kv_append(x, new, new, k, v, table, lengths, bounds=bounds)
        pages, n = mk.select_pages(y, bounds, table, lengths, 16, 2)
        return mk.paged_attention(y, k, v, pages, n)

    want = step(q)
    with Record():
        got = step(q)
    assert torch.equal(got, want)
    for name in ("kv_append", "select_pages", "paged_attention"):
        assert any("marlin_mi355x.%s" % name in x for x in seen), name
    other = torch.randn_like(q)
    want = mk.paged_attention(other, k, v, table, lengths)
    traced = torch.jit.trace(lambda x: mk.paged_attention(x, k, v, table, lengths), (q,), check_trace=False)
    assert torch.equal(traced(other), want)
    both = torch.vmap(lambda x: mk.paged_attention(x, k, v, table, lengths))(torch.stack([q, other]))
    assert torch.equal(both[1], want) and torch.equal(both[0], mk.paged_attention(q, k, v, table, lengths))

"""The 8-bit cache's neighbours where a result can go wrong without a crash: infinite values, softmax weights, pages of tokens taken back,
sequences that get nothing, rows of no sequence, any number of kv heads.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import cache_back  # noqa: E402
import cache_reference as ref  # noqa: E402
from test_gpu_cache import check, cuda, expect, gen, make, mk, serve, state  # noqa: E402, F401

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def put_values(args, h, odd):
    """odd: (sequence, position, channel, value) of kv head h."""
    ps = args["v_cache"].shape[2]
    for b, pos, ch, x in odd:
        args["v_cache"][int(args["table"][b, pos // ps]), h, pos % ps, ch] = x


# ---- infinite values ----

@pytest.mark.parametrize("new,hq,D,dtype", [([4], 4, 128, F16), ([5], 16, 64, BF16), ([3], 2, 256, F16), ([130], 1, 64, F16), ([200], 1, 128, BF16),
                                            ([130], 1, 96, BF16), ([10], 3, 128, F16), ([12], 4, 128, BF16), ([10], 3, 96, F16)])
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
                                                ([130], 2, 1, 256, F16), ([10], 3, 1, 128, F16), ([12, 9], 8, 2, 128, BF16), ([10], 3, 1, 96, F16)])
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


@pytest.mark.parametrize("new,hq,starts", [(*x, True) for x in FEW + MANY] + [([1], 1, False), ([1], 16, False)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("apart", [20, 30, 45])
def test_weights_of_scales_far_apart(mk, new, hq, starts, dtype, apart):
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
    if not starts:
        args["starts"] = None
    held_to(mk, args)


# ---- tokens taken back ----

def check_back(mk, table, lengths, new, free, count, ps, tokens, back, window=None, sinks=0):
    want = cache_back.assign_pages(table, lengths, new, free, count, ps, tokens, window, sinks, back)
    on = [x.cuda() for x in (table, lengths, new, free, torch.tensor([count], dtype=torch.int32))]
    starts, slots = mk.assign_pages(*on, ps, tokens, window=window, sinks=sinks, back=back.cuda())
    for name, x, y in zip(("table", "lengths", "free", "count", "starts", "slots"), want, (on[0], on[1], on[3], on[4], starts, slots)):
        x = torch.tensor([x], dtype=torch.int32) if name == "count" else x
        assert torch.equal(x, y.cpu()), (name, x, y)


@pytest.mark.parametrize("B", [1, 2, 64, 200, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("tokens", [0, 100, 4096, 4097, 200000])
@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 5)])
def test_pages_of_tokens_taken_back(mk, B, tokens, window, sinks):
    table, lengths, new, free, count = state(B + tokens, B, 16, 200, 2 * B, windowed=window is not None)
    g = gen(B)
    back = torch.randint(-3, 40, (B,), generator=g).int()
    back[torch.rand(B, generator=g) < 0.1] = 1000
    check_back(mk, table, lengths, new, free, count, 16, tokens, back, window, sinks)
    check_back(mk, table, lengths, torch.where(new < 0, new, 1), free, count, 16, tokens, back.clamp(max=4), window, sinks)


def test_tokens_taken_back_at_the_edges(mk):
    # lengths past the table and below none, all of a sequence, a full list, the largest numbers
    table, lengths, new, free, count = state(1, 20, 16, 100, 60, width=7)
    back = torch.full((20,), 20, dtype=torch.int32)
    lengths[0], lengths[1], lengths[2] = 112, 5000, -4
    back[3], back[4], back[5], back[6] = 2 ** 31 - 1, -(2 ** 31), 100, 0
    new[0], new[1], new[3], new[4] = 1, 30, 5, -1
    check_back(mk, table, lengths, new, free, count, 16, 500, back)
    check_back(mk, table, lengths, new, free, len(free) - 2, 16, 500, back)
    table[7:12] = -1  # nothing of theirs is a page
    check_back(mk, table, lengths, new, free, count, 16, 500, back)
    with pytest.raises(ValueError):
        mk.assign_pages(*[x.cuda() for x in (table, lengths, new, free, torch.tensor([count], dtype=torch.int32))], 16, 500, back=back[:3].cuda())
    with pytest.raises(TypeError):
        mk.assign_pages(*[x.cuda() for x in (table, lengths, new, free, torch.tensor([count], dtype=torch.int32))], 16, 500, back=back.long().cuda())


@pytest.mark.parametrize("bits,dtype", [(8, F16), (16, BF16)])
@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 5)])
def test_steps_of_drafts(mk, bits, dtype, window, sinks):
    """Drafted tokens of which some are accepted, step after step over page borders: every page is in one place once, and the attention is that of
    what was kept."""
    st, _, (hq, hkv, D, B) = serve(mk, bits, dtype, window, sinks)
    g, ps, pages = gen(4), 16, 200
    back = torch.zeros(B, dtype=torch.int32)
    kept = torch.zeros(B, dtype=torch.int32)
    for i in range(40):
        new = torch.tensor([20, 3, 17, 1, 40, 16]) if i == 0 else torch.full((B,), 5)
        if i == 25:
            new[2] = -1
        tokens = int(new.clamp(min=0).sum())
        q, k, v = torch.randn(tokens, hq + 2 * hkv, D, generator=g).to(dtype).cuda().split([hq, hkv, hkv], 1)
        starts, slots = mk.assign_pages(st["table"], st["lengths"], new.int().cuda(), st["free"], st["count"], ps, tokens, window=window, sinks=sinks,
                                        back=back.cuda())
        kept = torch.where(new < 0, 0, kept - back + new.int())
        assert torch.equal(st["lengths"].cpu(), kept.int()) and int(starts[-1]) == tokens and (slots >= 0).all()
        if bits == 8:
            q = mk.kv_append8(q, k, v, st["k"], st["v"], st["s"], st["table"], st["lengths"], st["cs"], starts)
        else:
            q = mk.kv_append(q, k, v, st["k"], st["v"], st["table"], st["lengths"], st["cs"], starts)
        o = mk.cache_attention(q, st["k"], st["v"], st["table"], st["lengths"], st["s"], starts, window, sinks)
        want, _, tol, _, mine = expect(st, q, starts, window, sinks)
        assert mine.all() and ((o.cpu().double() - want).abs() <= tol).all()
        both = torch.cat([st["table"][st["table"] >= 0], st["free"][:int(st["count"])]]).long().cpu()
        assert len(both) == pages and len(both.unique()) == pages
        back = torch.randint(0, 5, (B,), generator=g).int().clamp(max=kept)  # one of five drafts is accepted at least


def test_tokens_taken_back_in_a_graph_and_by_the_operator(mk):
    table, lengths, new, free, count = state(5, 100, 16, 300, 400)
    back = torch.randint(0, 30, (100,), generator=gen(5)).int().cuda()
    first = [x.cuda() for x in (table, lengths, new, free, torch.tensor([count], dtype=torch.int32))]
    def fresh():
        return [x.clone() for x in first]
    want = fresh()
    want += mk.assign_pages(*want, 16, 3000, 200, 3, back=back)
    got = fresh()
    got += torch.ops.marlin_mi355x.assign_pages(*got, 16, 3000, 200, 3, back)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    on = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mk.assign_pages(*on, 16, 3000, 200, 3, back=back)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = mk.assign_pages(*on, 16, 3000, 200, 3, back=back)
    for _ in range(3):
        for a, b in zip(on, first):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [*on, *out]))


# ---- sequences that get nothing ----

@pytest.mark.parametrize("bits,dtype", [(8, F16), (16, F16), (8, BF16)])
@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 5)])
def test_decode_where_some_sequences_get_nothing(mk, bits, dtype, window, sinks):
    """Pages run out and some ask for nothing: the calls for one token, given 0 for their lengths, leave their tokens as they are."""
    st, step, (hq, hkv, D, B) = serve(mk, bits, dtype, window, sinks)
    g = gen(6)
    first = torch.tensor([30, 64, 1, 16, 130, 9], dtype=torch.int32)
    rows = torch.randn(int(first.sum()), hq + 2 * hkv, D, generator=g).to(dtype).cuda()
    step(rows, first.cuda(), len(rows))
    st["count"].fill_(2)  # pages for two sequences more
    ones, passed_over = torch.tensor([1, 1, 1, 1, 0, 1], dtype=torch.int32).cuda(), 0
    for _ in range(20):
        q, k, v = torch.randn(B, hq + 2 * hkv, D, generator=g).to(dtype).cuda().split([hq, hkv, hkv], 1)
        before = st["lengths"].clone()
        starts, _ = mk.assign_pages(st["table"], st["lengths"], ones, st["free"], st["count"], 16, B, window=window, sinks=sinks)
        served = starts[1:] > starts[:-1]
        assert torch.equal(st["lengths"] - before, served.int())
        now = torch.where(served, st["lengths"], 0)
        old = [x.view(torch.uint8).clone() for x in (st["k"], st["v"], st["s"]) if x is not None]
        if bits == 8:
            q = mk.kv_append8(q, k, v, st["k"], st["v"], st["s"], st["table"], now, st["cs"])
        else:
            q = mk.kv_append(q, k, v, st["k"], st["v"], st["table"], now, st["cs"])
        o = mk.cache_attention(q, st["k"], st["v"], st["table"], now, st["s"], None, window, sinks)
        mine = st["table"][~served].flatten()
        mine = mine[mine >= 0].long()
        passed_over += int((~served).sum())
        for x, y in zip([x for x in (st["k"], st["v"], st["s"]) if x is not None], old):
            assert torch.equal(x.view(torch.uint8)[mine], y[mine])
        want, _, tol, _, _ = expect({**st, "lengths": now}, q, None, window, sinks)
        assert ((o.cpu().double() - want).abs() <= tol).all() and (o[~served] == 0).all() and (q[~served] == 0).all()
    assert passed_over > 20 and int(st["count"]) == 0


# ---- rows of no sequence ----

@pytest.mark.parametrize("first,new", [(0, [6, 3]), (2, [1, 0]), (0, [40, 25]), (3, [0, 0])])
def test_rows_of_no_sequence_where_a_mode_sees_the_call(mk, first, new):
    """What a call writes into out does not go by whether it became the registered operator's."""
    from torch.utils._python_dispatch import TorchDispatchMode

    class Watch(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            seen.append(str(func))
            return func(*args, **(kwargs or {}))

    seen, n, rest = [], sum(new), 7
    a = cuda(make(1, [30 + m for m in new], new, 4, 2, 64, 16, F16, 8, junk=False))
    a["starts"] += first
    a["q"] = torch.randn(first + n + rest, 4, 64, generator=gen(7)).half().cuda()
    kv = torch.randn(2, first + n + rest, 2, 64, generator=gen(8)).half().cuda()
    k16, v16 = mk.kv_cache(len(a["k_cache"]), 2, 16, 64)
    where = a["table"], a["lengths"], None, a["starts"]
    for call in (lambda out: mk.cache_attention(**a, out=out),
                 lambda out: mk.kv_append8(a["q"], *kv, *[a[x].clone() for x in ("k_cache", "v_cache", "scales")], *where, out=out),
                 lambda out: mk.kv_append(a["q"], *kv, k16, v16, *where, out=out)):
        got = [torch.full(a["q"].shape, 123.0, dtype=F16, device="cuda") for _ in range(2)]
        call(got[0])
        with Watch():
            assert call(got[1]) is got[1]
        assert torch.equal(*got) and (got[0][:first] == 123).all() and (got[0][first + n:] == 123).all()
    assert any("marlin_mi355x.cache_attention" in x for x in seen)


# ---- kv heads that do not divide the work-groups ----

@pytest.mark.parametrize("hq,hkv", [(3, 3), (6, 3), (5, 5), (20, 5), (40, 40), (12, 12)])
@pytest.mark.parametrize("new,cached", [([4], [5000]), ([3, 5, 1], [3000, 700, 6000]), ([130], [4000]), ([140, 1, 70], [2500, 4000, 100])])
@pytest.mark.parametrize("bits,D", [(8, 128), (16, 64)])
def test_shared_keys_of_any_number_of_heads(mk, hq, hkv, new, cached, bits, D):
    """Every row of out is written, whatever the kv heads: parts, records and pieces go by their number."""
    args = make(hkv, [c + n for c, n in zip(cached, new)], new, hq, hkv, D, 32, F16, bits)
    for more in (dict(), dict(window=2000, sinks=70)):
        out = torch.full(args["q"].shape, math.nan, dtype=F16, device="cuda")
        got, lse = mk.cache_attention(**cuda(args), out=out, return_lse=True, **more)
        want, want_lse, tol, tol_lse, mine = ref.attention(**args, **more)
        assert mine.all() and ((got.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - want_lse).abs() <= tol_lse).all()

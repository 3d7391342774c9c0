"""The paged key-value cache operators on the GPU against their 64-bit forms:
types, head layouts, lengths from none to long, page borders, strides, entries that
name no page, and whatever may lie in slots that no token uses.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import kv_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def mk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2408_11743_amd as mk
    mk.lib()
    return mk


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make(seed, lengths, hq, hkv, D, ps, dtype, spare=3, junk=True, per_head=False):
    """CPU tensors: q, caches, table, lengths.  Slots past the lengths, and pages no table names, hold NaN and inf."""
    g = gen(seed)
    used = [-(-max(0, n) // ps) for n in lengths]
    width = max(1, max(used))
    heads = hkv if per_head else 1
    total = sum(used) * heads
    pages = total + spare
    perm = torch.randperm(pages, generator=g)
    table = torch.full((len(lengths), heads, width), -1, dtype=torch.int32)
    at = 0
    k = torch.randn(pages, hkv, ps, D, generator=g).to(dtype)
    v = torch.randn(pages, hkv, ps, D, generator=g).to(dtype)
    bad = torch.tensor([math.nan, math.inf, -math.inf])
    for b, n in enumerate(lengths):
        for h in range(heads):
            table[b, h, :used[b]] = perm[at:at + used[b]].int()
            at += used[b]
            if used[b] and junk and n % ps:
                last = int(table[b, h, used[b] - 1])
                for x in (k, v):
                    fill = bad[torch.randint(0, 3, (hkv, ps - n % ps, D), generator=g)].to(dtype)
                    x[last, :, n % ps:] = fill
    if junk:
        for p in perm[at:]:
            k[p] = math.nan
            v[p] = math.inf
    q = torch.randn(len(lengths), hq, D, generator=g).to(dtype)
    return q, k, v, table if per_head else table[:, 0], torch.tensor(lengths, dtype=torch.int32)


def check_attention(mk, q, k, v, table, lengths, scale=None, call=None):
    want, want_lse, tol, tol_lse = ref.attention(q, k, v, table, lengths, scale)
    args = [x.cuda() for x in (q, k, v, table, lengths)]
    got, lse = (call or mk.paged_attention)(*args, scale=scale, return_lse=True)
    torch.cuda.synchronize()
    got, lse = got.cpu().double(), lse.cpu().double()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol
    assert over.max() <= 0, (float(over.max()), int(over.argmax()))
    empty = want_lse == -math.inf
    assert (lse[empty] == -math.inf).all() and (got[empty] == 0).all()
    assert ((lse - want_lse).abs()[~empty] <= tol_lse[~empty]).all()


# ---- attention ----

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("ps", [16, 64])
def test_attention_lengths(mk, dtype, D, ps):
    lengths = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 255, 256, 257, 300]
    check_attention(mk, *make(D + ps, lengths, 4, 2, D, ps, dtype))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (5, 1), (12, 4), (16, 1), (17, 1), (40, 2), (64, 2)])
def test_attention_head_groups(mk, hq, hkv):
    check_attention(mk, *make(hq, [33, 0, 129], hq, hkv, 128, 32, F16))


@pytest.mark.parametrize("ps", [16, 32, 128, 256, 1024])
def test_attention_page_sizes(mk, ps):
    check_attention(mk, *make(ps, [ps - 1, ps, ps + 1, 2 * ps + 7], 2, 1, 64, ps, BF16))


@pytest.mark.parametrize("lengths,hq,hkv", [
    ([2500], 2, 1),                       # one row, many work-groups
    ([1], 1, 1),
    ([700, 3, 0, 1400, 0, 0, 90], 4, 4),  # rows cut and rows whole in one range
    ([513, 512, 511, 767, 769], 1, 1),    # around the shortest rows that are cut
    (list(range(0, 70)), 1, 1),           # more sequences than lanes
    ([5] * 128 + [900] + [0] * 3, 2, 2),  # more than two waves of lengths
])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_attention_splits(mk, lengths, hq, hkv, dtype):
    check_attention(mk, *make(len(lengths), lengths, hq, hkv, 64, 16, dtype))


@pytest.mark.parametrize("n", [64, 65, 128, 500, 4096, 4200])
def test_attention_many_sequences(mk, n):
    lengths = [(i * 37) % 23 if i % 50 else 200 + i % 7 for i in range(n)]
    check_attention(mk, *make(n, lengths, 1, 1, 64, 16, BF16))


def test_attention_long(mk):
    check_attention(mk, *make(5, [40001, 17, 9000], 2, 1, 64, 64, F16))


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("n,hq", [(270, 16), (700, 5), (1100, 16), (2600, 3), (9001, 16)])
def test_attention_joins_of_few_and_many_pieces(mk, D, n, hq):
    """One row in two pieces to more than a work-group has waves, alone and between short rows."""
    check_attention(mk, *make(n + D, [n], hq, 1, D, 16, F16))
    check_attention(mk, *make(n + D, [40, n, 0, 40], hq, 1, D, 32, BF16))


@pytest.mark.parametrize("D", [128, 256])
def test_attention_uneven_shares(mk, D):
    """Ranges of every number of steps modulo the waves, rows that end within a range."""
    for n in (130, 290, 450, 610, 770):
        check_attention(mk, *make(n + D, [n, n // 3, n], 4, 4, D, 16, BF16))


@pytest.mark.parametrize("D,hq", [(64, 16), (96, 16), (128, 16), (128, 136), (256, 16)])
def test_attention_larger_than_the_last_level_cache(mk, D, hq):
    """More keys and values than the caches hold are read another way; two of the sequences are looked at."""
    g = torch.Generator(device="cuda").manual_seed(D + hq)
    hkv, ps, lengths = 8, 64, [9000 * 128 // D - 100 * i for i in range(12)]
    used = [-(-n // ps) for n in lengths]
    k, v = (torch.randn(sum(used), hkv, ps, D, dtype=BF16, device="cuda", generator=g) for _ in range(2))
    assert k.numel() * 4 > 256 << 20
    q = torch.randn(12, hq, D, dtype=BF16, device="cuda", generator=g)
    table = torch.zeros(12, max(used), dtype=torch.int32, device="cuda")
    perm = torch.randperm(sum(used), device="cuda", generator=g).int()
    for b, n in enumerate(used):
        table[b, :n] = perm[sum(used[:b]):sum(used[:b]) + n]
    got, lse = mk.paged_attention(q, k, v, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), return_lse=True)
    for b, heads in ((0, slice(0, hq // hkv)), (11, slice(hq - hq // hkv, hq))):
        kvh = heads.start // (hq // hkv)
        pages = table[b, :used[b]].long()
        mine = torch.arange(used[b], dtype=torch.int32)[None]
        want, want_lse, tol, tol_lse = ref.attention(q[b:b + 1, heads].cpu(), k[pages, kvh:kvh + 1].cpu(), v[pages, kvh:kvh + 1].cpu(),
                                                     mine, torch.tensor([lengths[b]]))
        assert ((got[b:b + 1, heads].cpu().double() - want).abs() <= tol).all()
        assert ((lse[b:b + 1, heads].cpu().double() - want_lse).abs() <= tol_lse).all()


def test_attention_no_sequence_has_tokens(mk):
    check_attention(mk, *make(6, [0, 0, 0], 4, 2, 128, 16, F16))


def test_attention_no_sequences(mk):
    q, k, v, table, lengths = make(6, [5], 4, 2, 128, 16, F16)
    o = mk.paged_attention(q.cuda()[:0], k.cuda(), v.cuda(), table.cuda()[:0], lengths.cuda()[:0])
    assert o.shape == (0, 4, 128)


def test_attention_entries_that_name_no_page(mk):
    q, k, v, table, lengths = make(7, [200, 100, 64, 500], 4, 2, 64, 32, F16)
    table[0, 1] = -1
    table[0, 3] = k.shape[0]
    table[1, :4] = 2 ** 31 - 1  # nothing left: an empty row
    table[3, ::2] = -2 ** 31
    check_attention(mk, q, k, v, table, lengths)


def test_attention_lengths_outside_the_table(mk):
    q, k, v, table, lengths = make(8, [96, 96, 64], 2, 2, 64, 32, BF16, junk=False)
    lengths = torch.tensor([2 ** 31 - 1, -2 ** 31, 97], dtype=torch.int32)
    table[2, 2] = table[0, 0]
    check_attention(mk, q, k, v, table, lengths)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (40, 2)])
def test_attention_a_table_for_each_head(mk, hq, hkv):
    check_attention(mk, *make(9, [130, 31, 0, 600], hq, hkv, 64, 16, F16, per_head=True))


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_attention_scales(mk, scale):
    check_attention(mk, *make(10, [50, 400], 3, 3, 64, 16, F16), scale=scale)


def test_attention_large_scores(mk):
    # one key far above the rest, and logits spread over hundreds
    q, k, v, table, lengths = make(11, [300, 1200], 4, 2, 64, 16, BF16, junk=False)
    check_attention(mk, q * 8, k * 8, v, table, lengths)


def test_attention_strided_queries_and_tables(mk):
    q, k, v, table, lengths = make(12, [60, 200, 33], 4, 2, 64, 16, F16)
    wide = torch.randn(3, 9, 64).half()
    wide[:, 2:6] = q
    rows = torch.full((3, table.shape[1] + 5), -7, dtype=torch.int32)
    rows[:, 2:2 + table.shape[1]] = table

    def call(q_, k_, v_, table_, lengths_, **kw):
        return mk.paged_attention(wide.cuda()[:, 2:6], k_, v_, rows.cuda()[:, 2:2 + table.shape[1]], lengths_, **kw)
    check_attention(mk, q, k, v, table, lengths, call=call)

    def turned(q_, k_, v_, table_, lengths_, **kw):  # heads before sequences
        return mk.paged_attention(q_.transpose(0, 1).contiguous().transpose(0, 1), k_, v_, table_, lengths_, **kw)
    check_attention(mk, q, k, v, table, lengths, call=turned)

    def odd(q_, k_, v_, table_, lengths_, **kw):  # channels apart, and rows at an odd address: copied
        x = torch.empty(3, 4, 129, dtype=F16, device="cuda")
        x[:, :, 1::2] = q_
        a, l1 = mk.paged_attention(x[:, :, 1::2], k_, v_, table_, lengths_, **kw)
        y = torch.empty(3 * 4 * 64 + 1, dtype=F16, device="cuda")[1:].view(3, 4, 64).copy_(q_)
        b, l2 = mk.paged_attention(y, k_, v_, table_, lengths_, **kw)
        assert torch.equal(a, b) and torch.equal(l1, l2)
        return a, l1
    check_attention(mk, q, k, v, table, lengths, call=odd)


def test_attention_broadcast_queries(mk):
    q, k, v, table, lengths = make(13, [60, 200, 33], 4, 2, 64, 16, F16)
    q = q[:1, :1].expand(3, 4, 64)
    check_attention(mk, q, k, v, table, lengths, call=lambda a, *r, **kw: mk.paged_attention(
        a[:1, :1].expand(3, 4, 64), *r, **kw))


def test_attention_infinities_and_nan_among_the_keys(mk):
    q, k, v, table, lengths = make(14, [100, 100, 700], 2, 1, 64, 16, F16)
    q.abs_()
    for i in range(100):  # every score -inf: no weight anywhere
        k[table[0, i // 16], 0, i % 16] = -math.inf
    k[table[1, 2], 0, 3] = math.nan
    k[table[2, 30], 0, 5] = -math.inf  # one key that has no weight
    out, lse = mk.paged_attention(q.cuda(), k.cuda(), v.cuda(), table.cuda(), lengths.cuda(), return_lse=True)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    k[table[1, 2], 0, 3] = 0
    want, want_lse, tol, tol_lse = ref.attention(q[2:], k, v, table[2:], lengths[2:])
    finite = k[table[2, 30], 0, 5].clone().fill_(0)
    assert torch.isfinite(finite).all()
    w = torch.cat([out[2:].cpu().double()])
    s = ref.attention(q[2:], torch.where(torch.isinf(k), torch.tensor(-100.0).half(), k), v, table[2:], lengths[2:])
    assert ((w - s[0]).abs() <= s[2]).all()


def test_attention_repeats_bit_for_bit_and_leaves_its_counters(mk):
    q, k, v, table, lengths = (x.cuda() for x in make(15, [3000, 40, 900], 8, 2, 128, 16, F16))
    ws = mk.Workspace("cuda")
    first = mk.paged_attention(q, k, v, table, lengths, workspace=ws)
    for _ in range(5):
        assert torch.equal(mk.paged_attention(q, k, v, table, lengths, workspace=ws), first)
    assert int(ws.buf[:1 << 20].count_nonzero()) == 0
    # a workspace shared with the GEMM and a call of another head size
    wp = torch.randint(0, 256, (256 * 192 // 2,), dtype=torch.uint8, device="cuda")
    sp = torch.rand(2 * 192, device="cuda").half() * 0.01
    A = torch.randn(5, 256, device="cuda").half()
    c = mk.gemm(A, wp, sp, 256, 192, workspace=ws)
    other = [x.cuda() for x in make(16, [2000], 4, 1, 256, 16, BF16)]
    o = mk.paged_attention(*other, workspace=ws)
    for _ in range(3):
        assert torch.equal(mk.gemm(A, wp, sp, 256, 192, workspace=ws), c)
        assert torch.equal(mk.paged_attention(*other, workspace=ws), o)
        assert torch.equal(mk.paged_attention(q, k, v, table, lengths, workspace=ws), first)


@pytest.mark.parametrize("D,hq,lengths", [
    (128, 16, [6001, 7000, 8100, 33]), (256, 16, [5000, 9000]), (256, 5, [21000]), (64, 16, [9001]), (128, 7, [16001, 16]),
    (96, 32, [12000])])
def test_attention_joins_in_teams(mk, D, hq, lengths):
    """Rows of so many pieces that teams of work-groups join them: right, the same bits each time, counters left at zero."""
    args = make(D + hq, lengths, hq, 1, D, 64, BF16)
    check_attention(mk, *args)
    args = [x.cuda() for x in args]
    ws = mk.Workspace("cuda")
    first = mk.paged_attention(*args, workspace=ws)
    for _ in range(4):
        assert torch.equal(mk.paged_attention(*args, workspace=ws), first)
    assert int(ws.buf[:1 << 20].count_nonzero()) == 0


def test_attention_on_another_stream(mk):
    q, k, v, table, lengths = make(17, [3000, 40, 900], 8, 2, 128, 16, F16)
    side = torch.cuda.Stream()
    args = [x.cuda() for x in (q, k, v, table, lengths)]
    base = mk.paged_attention(*args)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [mk.paged_attention(*args) for _ in range(4)]
    here = [mk.paged_attention(*args) for _ in range(4)]
    torch.cuda.synchronize()
    for o in outs + here:
        assert torch.equal(o, base)


def test_offsets_beyond_32_bits(mk):
    # 2^31 elements lie 4 GiB into each cache: the last page starts behind them
    ps, hkv, D = 256, 8, 128
    pages = (1 << 31) // (ps * hkv * D) + 3
    k = torch.zeros(pages, hkv, ps, D, dtype=F16, device="cuda")
    v = torch.zeros_like(k)
    g = gen(18)
    small = torch.randn(2, 2, hkv, ps, D, generator=g).half()
    where = [pages - 1, 0]
    for i, p in enumerate(where):
        k[p], v[p] = small[0, i].cuda(), small[1, i].cuda()
    q = torch.randn(1, 16, D, generator=g).half()
    table = torch.tensor([where], dtype=torch.int32)
    near = torch.tensor([[0, 1]], dtype=torch.int32)
    lengths = torch.tensor([400], dtype=torch.int32)
    want, _, tol, _ = ref.attention(q, small[0], small[1], near, lengths)
    got = mk.paged_attention(q.cuda(), k, v, table.cuda(), lengths.cuda())
    assert ((got.cpu().double() - want).abs() <= tol).all()
    # and an append there
    new = torch.randn(3, 1, hkv, D, generator=g).half().cuda()
    mk.kv_append(new[0], new[1], new[2], k, v, table.cuda().flip(1), torch.tensor([300], dtype=torch.int32, device="cuda"))
    assert torch.equal(k[pages - 1, :, 300 - 256 - 1], new[1, 0]) and torch.equal(v[pages - 1, :, 43], new[2, 0])


# ---- append ----

def check_append(mk, q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts=None, interleaved=False, bounds=None):
    put, want_q, q_tol = ref.append(q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, interleaved)
    dev = [None if x is None else x.cuda() for x in (q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, bounds)]
    dev[:3] = torch.cat(dev[:3], 1).split([q.shape[1], k.shape[1], v.shape[1]], 1)  # slices of one projection's rows
    out = mk.kv_append(*dev[:7], cos_sin=dev[7], starts=dev[8], interleaved=interleaved, bounds=dev[9])
    torch.cuda.synchronize()
    assert ((out.cpu().double() - want_q).abs() <= q_tol).all()
    got_k, got_v = dev[3].cpu(), dev[4].cpu()
    want_k, want_v = k_cache.clone(), v_cache.clone()
    for (page, slot), ((key, tol), value) in put.items():
        assert ((got_k[page, :, slot].double() - key).abs() <= tol).all(), (page, slot)
        want_k[page, :, slot] = got_k[page, :, slot]
        want_v[page, :, slot] = value
    # everything else is untouched, and values are the same bits
    assert torch.equal(got_k.view(torch.int16), want_k.view(torch.int16))
    assert torch.equal(got_v.view(torch.int16), want_v.view(torch.int16))
    if bounds is not None:
        got_b, want_b = dev[9].cpu(), bounds.clone()
        for page in {p for p, _ in put}:
            slots = sorted(s for p, s in put if p == page)
            keys = got_k[page][:, slots]
            stack = [keys] if slots[0] == 0 else [keys, bounds[page]]
            for i, pick in ((0, torch.argmin), (1, torch.argmax)):
                every = torch.cat([stack[0]] + [x[:, i:i + 1] for x in stack[1:]], 1)
                want_b[page, :, i] = torch.gather(every, 1, pick(ref.order(every), 1, keepdim=True))[:, 0]
        assert torch.equal(got_b.view(torch.int16), want_b.view(torch.int16))
    return out


def append_inputs(seed, lengths, new, hq, hkv, D, ps, dtype, rot, width=None):
    g = gen(seed)
    used = [-(-max(0, n) // ps) for n in lengths]
    width = max(1, max(used)) if width is None else width
    pages = sum(used) + 3
    perm = torch.randperm(pages, generator=g).int()
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        n = min(n, width)
        table[b, :n] = perm[at:at + n]
        at += n
    tokens = sum(new)
    qkv = torch.randn(tokens, hq + 2 * hkv, D, generator=g).to(dtype)
    caches = torch.randn(2, pages, hkv, ps, D, generator=g).to(dtype)
    angle = torch.arange(max(1, max(lengths)), dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float() if rot else None
    starts = torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32)
    bounds = torch.randn(pages, hkv, 2, D, generator=g).to(dtype)
    return (qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], caches[0], caches[1], table,
            torch.tensor(lengths, dtype=torch.int32), cos_sin), starts, bounds


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,rot", [(64, 64), (96, 96), (128, 128), (256, 256), (96, 48), (128, 32), (256, 0), (64, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_one_token(mk, dtype, D, rot, interleaved):
    lengths = [1, 16, 17, 32, 0, 100, 64]
    args, _, bounds = append_inputs(D + rot, lengths, [1] * 7, 6, 2, D, 16, dtype, rot)
    check_append(mk, *args, interleaved=interleaved, bounds=bounds)
    check_append(mk, *args, interleaved=interleaved)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,rot", [(64, 64), (96, 96), (128, 128), (256, 256), (96, 48), (128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_prompts(mk, dtype, D, rot, interleaved):
    new = [1, 16, 0, 33, 5, 70, 2, 31]
    before = [0, 0, 9, 0, 14, 27, 31, 1]
    lengths = [a + b for a, b in zip(new, before)]
    args, starts, bounds = append_inputs(D + rot + 1, lengths, new, 6, 3, D, 16, dtype, rot)
    check_append(mk, *args, starts=starts, interleaved=interleaved, bounds=bounds)
    check_append(mk, *args, starts=starts, interleaved=interleaved)


@pytest.mark.parametrize("ps", [16, 32, 64, 256, 1024])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (9, 9), (40, 5)])
def test_append_prompts_page_sizes(mk, ps, hq, hkv):
    new = [ps, ps + 1, 2 * ps - 1, 3]
    lengths = [ps, ps + 8, 2 * ps, 2 * ps + 1]
    args, starts, bounds = append_inputs(ps + hq, lengths, new, hq, hkv, 64, ps, F16, 64)
    check_append(mk, *args, starts=starts, bounds=bounds)


@pytest.mark.parametrize("n", [64, 65, 150, 4200])
def test_append_prompts_many_sequences(mk, n):
    new = [(i * 7) % 5 for i in range(n)]
    lengths = [n + (i * 11) % 40 for i, n in enumerate(new)]
    args, starts, bounds = append_inputs(3, lengths, new, 2, 1, 64, 16, BF16, 64)
    check_append(mk, *args, starts=starts, bounds=bounds)


@pytest.mark.parametrize("prompts", [False, True])
def test_append_tokens_that_have_no_place(mk, prompts):
    # positions below 0 and past the table, entries that name no page, angles that end early
    new = [20, 40, 5, 30, 12] if prompts else [1] * 5
    lengths = [8, 100, 0, 30, 2000] if prompts else [0, 100, -5, 30, 2 ** 31 - 1]
    args, starts, bounds = append_inputs(21, [max(0, min(n, 100)) for n in lengths], new, 4, 2, 64, 16, F16, 32, width=5)
    args = list(args)
    args[6] = torch.tensor(lengths, dtype=torch.int32)
    args[5][3, 1] = -1
    args[5][3, 0] = args[3].shape[0]
    args[7] = args[7][:70]
    check_append(mk, *args, starts=starts if prompts else None, bounds=bounds)


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_prompts_large(mk, interleaved):
    """Prompts larger than the last-level cache are read another way: the same bits as one sequence at a time."""
    g = torch.Generator(device="cuda").manual_seed(25)
    hq, hkv, D, ps, new = 24, 4, 128, 32, [9001, 7013, 8191]
    lengths = torch.tensor([9001, 7013 + 45, 8191 + 7], dtype=torch.int32, device="cuda")
    used = [-(-n // ps) for n in lengths.tolist()]
    qkv = torch.randn(sum(new), hq + 2 * hkv, D, dtype=F16, device="cuda", generator=g)
    assert qkv.numel() * 2 > 128 << 20
    q, k, v = qkv.split([hq, hkv, hkv], 1)
    table = torch.full((3, max(used)), -1, dtype=torch.int32, device="cuda")
    perm = torch.randperm(sum(used) + 1, device="cuda", generator=g).int()
    for b, n in enumerate(used):
        table[b, :n] = perm[sum(used[:b]):sum(used[:b]) + n]
    angles = mk.rotation_table(9001, D)
    sides = []
    for whole in (True, False):
        kc, vc, bounds = mk.kv_cache(sum(used) + 1, hkv, ps, D, F16, bounds=True)
        starts = torch.tensor([0] + list(torch.tensor(new).cumsum(0)), dtype=torch.int32, device="cuda")
        if whole:
            out = mk.kv_append(q, k, v, kc, vc, table, lengths, angles, starts, interleaved, bounds)
        else:
            outs = []
            for b, n in enumerate(new):
                at = slice(sum(new[:b]), sum(new[:b]) + n)
                outs.append(mk.kv_append(q[at], k[at], v[at], kc, vc, table[b:b + 1], lengths[b:b + 1], angles,
                                         starts[b:b + 2] - starts[b], interleaved, bounds))
            out = torch.cat(outs)
        sides.append((out, kc, vc, bounds))
    for a, b in zip(*sides):
        assert torch.equal(a, b)


def test_append_past_the_angles(mk):
    args, starts, bounds = append_inputs(22, [90, 100], [30, 40], 4, 2, 64, 16, F16, 32)
    args = list(args)
    args[7] = args[7][:75].contiguous()
    check_append(mk, *args, starts=starts, bounds=bounds)


@pytest.mark.parametrize("prompts", [False, True])
def test_append_bounds_order_infinities_zeros_and_nan(mk, prompts):
    for dtype in (F16, BF16):
        new = [16, 9, 7] if prompts else [1, 1, 1]
        lengths = [16, 25, 7] if prompts else [16, 25, 1]
        (q, k, v, kc, vc, table, ln, _), starts, bounds = append_inputs(23, lengths, new, 2, 2, 64, 16, dtype, 0)
        odd = torch.tensor([math.inf, -math.inf, 0.0, -0.0, math.nan, 1.5, -2.5, 6e-8])
        g = gen(24)
        k = odd[torch.randint(0, 8, k.shape, generator=g)].to(dtype)
        bounds = odd[torch.randint(0, 4, bounds.shape, generator=g)].to(dtype)
        dev = [x.cuda() for x in (q, k, v, kc, vc, table, ln)]
        b = bounds.cuda()
        mk.kv_append(*dev, starts=starts.cuda() if prompts else None, bounds=b)
        got_k, b = dev[3].cpu(), b.cpu()
        at = 0
        for s, n in enumerate(new):
            for i in range(n):
                pos = lengths[s] - n + i
                assert torch.equal(got_k[table[s, pos // 16], :, pos % 16].view(torch.int16), k[at + i].view(torch.int16))
            page, first = int(table[s, (lengths[s] - 1) // 16]), (lengths[s] - 1) // 16 * 16
            keys = k[at + max(0, first - (lengths[s] - n)):at + n]
            every = ref.order(torch.cat([keys] + ([] if lengths[s] - n <= first else [bounds[page][:, :1].transpose(0, 1)])))
            assert torch.equal(ref.order(b[page, :, 0]), every.amin(0))
            every = ref.order(torch.cat([keys] + ([] if lengths[s] - n <= first else [bounds[page][:, 1:].transpose(0, 1)])))
            assert torch.equal(ref.order(b[page, :, 1]), every.amax(0))
            at += n


def test_append_in_place_and_strided(mk):
    args, starts, _ = append_inputs(25, [40, 17], [40, 3], 4, 2, 64, 16, F16, 64)
    dev = [x.cuda() for x in args]
    want = mk.kv_append(*dev, starts=starts.cuda())
    q = dev[0].clone()
    got = mk.kv_append(q, *dev[1:], starts=starts.cuda(), out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want)
    turned = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in dev[:3]]
    assert torch.equal(mk.kv_append(*turned, *dev[3:], starts=starts.cuda()), want)


def test_append_one_token_many_sequences(mk):
    lengths = [(i * 11) % 40 for i in range(1000)]
    args, _, bounds = append_inputs(4, lengths, [1] * 1000, 2, 1, 64, 16, F16, 64)
    check_append(mk, *args, bounds=bounds)


def test_append_no_tokens(mk):
    args, starts, _ = append_inputs(26, [5, 9], [0, 0], 4, 2, 64, 16, F16, 64)
    before = args[3].clone()
    dev = [x.cuda() for x in args]
    assert mk.kv_append(*dev, starts=starts.cuda()).shape == (0, 4, 64)
    assert torch.equal(dev[3].cpu(), before)


# ---- selection ----

def select_inputs(seed, lengths, hq, hkv, D, ps, dtype):
    """Small integers: every score is exact in fp32, and many are equal."""
    g = gen(seed)
    used = [-(-max(0, n) // ps) for n in lengths]
    pages = sum(used) + 2
    perm = torch.randperm(pages, generator=g).int()
    table = torch.full((len(lengths), max(1, max(used))), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = perm[at:at + n]
        at += n
    q = torch.randint(-2, 3, (len(lengths), hq, D), generator=g)
    q = (q * (torch.rand(q.shape, generator=g) < 8 / D)).to(dtype)
    a, b = torch.randint(-3, 4, (2, pages, hkv, D), generator=g)
    bounds = torch.stack([torch.minimum(a, b), torch.maximum(a, b)], 2).to(dtype)
    return q, bounds, table, torch.tensor(lengths, dtype=torch.int32)


def check_select(mk, q, bounds, table, lengths, ps, count):
    want, tokens = ref.select(q, bounds, table, lengths, ps, count)
    got, n = mk.select_pages(q.cuda(), bounds.cuda(), table.cuda(), lengths.cuda(), ps, count)
    assert torch.equal(n.cpu(), tokens)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("count", [1, 2, 7])
def test_select(mk, dtype, D, count):
    lengths = [0, 1, 16, 17, 100, 112, 113, 500, 1030]
    check_select(mk, *select_inputs(D + count, lengths, 6, 2, D, 16, dtype), 16, count)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (16, 1), (17, 1), (40, 2), (8, 8)])
def test_select_head_groups(mk, hq, hkv):
    check_select(mk, *select_inputs(hq, [700, 90], hq, hkv, 64, 32, F16), 32, 5)


@pytest.mark.parametrize("pages,count", [(2100, 64), (2100, 2099), (2100, 2100), (2100, 2500), (513, 512), (9000, 1000)])
def test_select_many_pages(mk, pages, count):
    check_select(mk, *select_inputs(pages, [16 * pages - 3], 2, 1, 64, 16, BF16), 16, count)


@pytest.mark.parametrize("pages,count", [(4095, 30), (4096, 4000), (4097, 4000), (4097, 1), (16385, 64), (16386, 3000)])
def test_select_registers_lds_and_memory(mk, pages, count):
    check_select(mk, *select_inputs(pages, [16 * pages - 5, 16 * (pages // 2), 16], 2, 1, 64, 16, F16), 16, count)


def test_select_many_rows(mk):
    lengths = [(i * 997) % 9000 + 1 if i % 9 else 0 for i in range(40)]
    check_select(mk, *select_inputs(77, lengths, 8, 8, 64, 16, BF16), 16, 12)


def test_select_equal_scores(mk):
    q, bounds, table, lengths = select_inputs(31, [1600], 2, 1, 64, 16, F16)
    check_select(mk, torch.zeros_like(q), bounds, table, lengths, 16, 10)
    check_select(mk, q, torch.ones_like(bounds), table, lengths, 16, 10)


def test_select_nan_infinities_and_no_pages(mk):
    q, bounds, table, lengths = select_inputs(32, [800, 800], 2, 1, 64, 16, F16)
    q[:] = q + 1
    bounds[table[0, 7], 0, :, 3] = math.nan
    bounds[table[0, 20], 0, :, 5] = -math.inf
    bounds[table[1, 11], 0] = -60000.0
    table[1, 4:40:3] = -1
    table[1, 5] = bounds.shape[0]
    check_select(mk, q, bounds, table, lengths, 16, 6)
    check_select(mk, q, bounds, table, lengths, 16, 47)


def test_select_then_attend_is_attention_over_those_pages(mk):
    q, k, v, table, lengths = make(33, [1000, 90, 0, 333], 8, 2, 64, 16, F16, junk=False)
    bounds = torch.zeros(k.shape[0], 2, 2, 64, dtype=F16)
    for b, n in enumerate(lengths.tolist()):
        for i in range(-(-n // 16)):
            keys = k[table[b, i], :, :min(16, n - 16 * i)]
            bounds[table[b, i]] = torch.stack([keys.amin(1), keys.amax(1)], 1)
    pages, tokens = mk.select_pages(q.cuda(), bounds.cuda(), table.cuda(), lengths.cuda(), 16, 9)
    check_attention(mk, q, k, v, pages.cpu(), tokens.cpu())
    # with room for every page it is the whole attention, bit for bit
    pages, tokens = mk.select_pages(q.cuda(), bounds.cuda(), table.cuda(), lengths.cuda(), 16, table.shape[1])
    assert torch.equal(tokens.cpu(), lengths)
    args = q.cuda(), k.cuda(), v.cuda()
    assert torch.equal(mk.paged_attention(*args, pages, tokens), mk.paged_attention(*args, table.cuda(), lengths.cuda()))


# ---- a step ----

def test_captured_step_follows_the_lengths(mk):
    lengths = [30, 1, 0, 200]
    room = 260
    (q, k, v, kc, vc, table, _, cos_sin), _, _ = append_inputs(41, [room] * 4, [1] * 4, 8, 2, 64, 16, F16, 64)
    dev = [x.cuda() for x in (q, k, v, table, cos_sin)]
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    caches = [[kc.cuda(), vc.cuda(), torch.zeros(kc.shape[0], 2, 2, 64, dtype=F16, device="cuda")] for _ in range(2)]

    def step(c):
        x = mk.kv_append(dev[0], dev[1], dev[2], c[0], c[1], dev[3], n, cos_sin=dev[4], bounds=c[2])
        pages, tokens = mk.select_pages(x, c[2], dev[3], n, 16, 4)
        return mk.paged_attention(x, c[0], c[1], dev[3], n), mk.paged_attention(x, c[0], c[1], pages, tokens)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step(caches[0])
    caches[0][0].copy_(kc.cuda()), caches[0][1].copy_(vc.cuda()), caches[0][2].zero_()
    for i in range(6):
        n += 7 if i == 3 else 1
        dev[0].normal_(), dev[1].normal_(), dev[2].normal_()
        graph.replay()
        want = step(caches[1])
        torch.cuda.synchronize()
        for a, b in zip(list(got) + caches[0], list(want) + caches[1]):
            assert torch.equal(a, b), i


def test_registered_operators_are_the_functions(mk):
    ns = torch.ops.marlin_mi355x
    args, starts, bounds = append_inputs(42, [40, 17], [40, 3], 4, 2, 64, 16, F16, 64)
    dev = [x.cuda() for x in args]
    b1, b2 = bounds.cuda(), bounds.cuda()
    other = [dev[3].clone(), dev[4].clone()]
    a = mk.kv_append(*dev, starts=starts.cuda(), bounds=b1)
    b = ns.kv_append(*dev[:3], *other, b2, *dev[5:], starts.cuda())
    assert torch.equal(a, b) and torch.equal(dev[3], other[0]) and torch.equal(dev[4], other[1]) and torch.equal(b1, b2)
    one = [dev[5], dev[6]]
    x, lse = mk.paged_attention(a[[39, 42]], *other, *one, scale=0.2, return_lse=True)
    y, lse2 = ns.paged_attention(a[[39, 42]], *other, *one, 0.2)
    assert torch.equal(x, y) and torch.equal(lse, lse2)
    for u, w in zip(mk.select_pages(a[[39, 42]], b1, *one, 16, 2), ns.select_pages(a[[39, 42]], b1, *one, 16, 2)):
        assert torch.equal(u, w)


@pytest.mark.parametrize("select", [0, 3])
def test_example_layer(mk, select):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_layer.py")
    spec = importlib.util.spec_from_file_location("decode_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(["--hidden", "512", "--heads", "8", "--kv-heads", "2", "--head-dim", "64", "--sequences", "5",
                         "--prompt", "90", "--steps", "9", "--select", str(select)])


# ---- refusals ----

def test_refusals(mk):
    q, k, v, table, lengths = (x.cuda() for x in make(51, [40, 50], 4, 2, 64, 16, F16, junk=False))
    ok = dict(q=q, k_cache=k, v_cache=v, table=table, lengths=lengths)

    def refuse(kind, fn=mk.paged_attention, base=ok, **change):
        with pytest.raises(kind):
            fn(**{**base, **change})

    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(table=table.long()), dict(lengths=lengths.long()),
                dict(k_cache=k.float()), dict(v_cache=v.to(BF16)), dict(table=table.cpu())):
        refuse(TypeError, **bad)
    for bad in (dict(q=q[0]), dict(q=q[:1]), dict(q=q[..., :32]), dict(k_cache=k[:, :1], v_cache=v[:, :1]),
                dict(v_cache=v[:-1]), dict(k_cache=k.transpose(0, 1), v_cache=v.transpose(0, 1)),
                dict(table=table[:1]), dict(lengths=lengths[:1]), dict(table=table.t().contiguous().t()),
                dict(table=table[:, None].expand(2, 3, -1)), dict(out=torch.empty(2, 4, 64, device="cuda")),
                dict(out=torch.empty(2, 4, 32, device="cuda", dtype=F16)), dict(k_cache=k._neg_view())):
        refuse(ValueError, **bad)
    for bad, status in ((dict(q=q[:, :3]), 2), (dict(scale=math.nan), 8), (dict(scale=math.inf), 8)):
        with pytest.raises(mk.MarlinError) as e:
            mk.paged_attention(**{**ok, **bad})
        assert e.value.status == status
    small = torch.zeros(4, 2, 8, 64, dtype=F16, device="cuda")
    with pytest.raises(mk.MarlinError):
        mk.paged_attention(q, small, small, table, lengths)

    kn = torch.randn(2, 2, 64, device="cuda").half()
    cos_sin = mk.rotation_table(64, 64)
    ap = dict(q=q, k=kn, v=kn, k_cache=k, v_cache=v, table=table, lengths=lengths, cos_sin=cos_sin)
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    for bad in (dict(k=kn.float()), dict(cos_sin=cos_sin.double()), dict(starts=starts.long())):
        refuse(TypeError, mk.kv_append, ap, **bad)
    for bad in (dict(k=kn[:1]), dict(v=kn[:, :1]), dict(cos_sin=cos_sin[:, ::2]), dict(starts=starts[:2]),
                dict(bounds=k), dict(q=q[:1], k=kn[:1], v=kn[:1]), dict(lengths=lengths[:1])):
        refuse(ValueError, mk.kv_append, ap, **bad)
    for bad, status in ((dict(cos_sin=mk.rotation_table(64, 24)), 8), (dict(cos_sin=mk.rotation_table(64, 80)), 8)):
        with pytest.raises(mk.MarlinError) as e:
            mk.kv_append(**{**ap, **bad})
        assert e.value.status == status

    bounds = torch.zeros(k.shape[0], 2, 2, 64, dtype=F16, device="cuda")
    se = dict(q=q, bounds=bounds, table=table, lengths=lengths, page_size=16, select=3)
    for bad in (dict(bounds=bounds.float()), dict(q=q.to(BF16)), dict(table=table.long())):
        refuse(TypeError, mk.select_pages, se, **bad)
    for bad in (dict(bounds=k), dict(q=q[:1]), dict(lengths=lengths[:1])):
        refuse(ValueError, mk.select_pages, se, **bad)
    for bad, status in ((dict(select=0), 8), (dict(page_size=24), 2), (dict(page_size=0), 2), (dict(q=q[:, :3]), 2)):
        with pytest.raises(mk.MarlinError) as e:
            mk.select_pages(**{**se, **bad})
        assert e.value.status == status

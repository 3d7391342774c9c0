"""The 8-bit cache, attention with windows and of several new tokens, and the page tables on the GPU against their plain forms: types,
head layouts, lengths from none to long, borders of pages, blocks, steps and windows, strides, entries and scales that name nothing, and
whatever may lie where no token looks.
"""
import math

import pytest

torch = pytest.importorskip("torch")

import cache_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def mk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2408_11743_amd as mk
    mk.lib()
    return mk


def gen(seed):
    return torch.Generator().manual_seed(seed)


def make(seed, lengths, new, hq, hkv, D, ps, dtype, bits, junk=True, spare=3, room=0, per_head=False):
    """CPU tensors q, caches, table, lengths, scales, starts.  Slots past the lengths and pages that no table names hold NaN and
    infinities, their scales none; new: tokens of each sequence, or None for one each without starts."""
    g = gen(seed)
    used = [-(-max(0, n) // ps) for n in lengths]
    width, heads = max(1, max(used)) + room, hkv if per_head else 1
    total = sum(used) * heads
    perm = torch.randperm(total + spare, generator=g)
    table = torch.full((len(lengths), heads, width), -1, dtype=torch.int32)
    k, v = (torch.randn(total + spare, hkv, ps, D, generator=g) for _ in range(2))
    k[..., :3] *= 3
    scales = None
    if bits == 8:
        scales = 2.0 ** torch.randint(-9, 5, (total + spare, hkv, 2, ps // 16), generator=g).float()
        scales[::3] *= 1.25  # not only powers of two
        k, v = ((x * 60).clamp(-448, 448).to(E4M3) for x in (k, v))
        scales[:, :, 0] /= 64
        scales[:, :, 0] = scales[:, :, 0].clamp(max=2.0 ** -7)
        junk_k = junk_v = torch.tensor([math.nan]).to(E4M3)
    else:
        k, v = k.to(dtype), v.to(dtype)
        junk_k = junk_v = torch.tensor([math.nan, math.inf, -math.inf]).to(dtype)

    def bits_of(x):
        return x.view(torch.uint8) if bits == 8 else x.view(torch.int16)

    at = 0
    for b, n in enumerate(lengths):
        for h in range(heads):
            table[b, h, :used[b]] = perm[at:at + used[b]].int()
            at += used[b]
            if used[b] and junk and n % ps:
                last = int(table[b, h, used[b] - 1])
                for x, odd in ((k, junk_k), (v, junk_v)):
                    pick = torch.randint(0, len(odd), (hkv, ps - n % ps, D), generator=g)
                    bits_of(x)[last, :, n % ps:] = bits_of(odd)[pick]
                if bits == 8 and -(-(n % ps) // 16) < ps // 16:
                    scales[last, :, :, -(-(n % ps) // 16):] = math.nan
    if junk:
        for p in perm[at:]:
            bits_of(k)[p] = bits_of(junk_k)[0]
            bits_of(v)[p] = bits_of(junk_v)[-1]
            if bits == 8:
                scales[p] = math.nan
    tokens = len(lengths) if new is None else sum(new)
    q = torch.randn(tokens, hq, D, generator=g).to(dtype)
    starts = None if new is None else torch.tensor([0] + new).cumsum(0).int()
    return dict(q=q, k_cache=k, v_cache=v, table=table if per_head else table[:, 0], lengths=torch.tensor(lengths, dtype=torch.int32),
                scales=scales, starts=starts)


def cuda(args):
    return {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in args.items()}


def check(mk, args, call=None, **more):
    want, want_lse, tol, tol_lse, mine = ref.attention(**args, **more)
    got, lse = (call or mk.cache_attention)(**cuda(args), **more, return_lse=True)
    torch.cuda.synchronize()
    got, lse = got.cpu().double()[mine], lse.cpu().double()[mine]
    want, want_lse, tol, tol_lse = want[mine], want_lse[mine], tol[mine], tol_lse[mine]
    if args["q"].dtype == F16:  # what rounds to an infinity
        want = torch.where(want.abs() >= 65520, want.sign() * math.inf, want)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)])
    over = ((got - want).abs() - tol)[~odd]
    assert over.numel() == 0 or over.max() <= 0, (float(over.max()), int(over.argmax()))
    empty = want_lse == -math.inf
    assert (lse[empty] == -math.inf).all() and (got[empty] == 0).all()
    assert ((lse - want_lse).abs()[~empty] <= tol_lse[~empty]).all()
    return got


# ---- attention of one token: 8 bits, windows ----

@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("ps", [16, 64])
def test_token_8bit_lengths(mk, dtype, D, ps):
    lengths = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 255, 256, 257, 300]
    check(mk, make(D + ps, lengths, None, 4, 2, D, ps, dtype, 8))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (5, 1), (12, 4), (16, 1), (17, 1), (40, 2), (64, 2)])
def test_token_8bit_head_groups(mk, hq, hkv):
    check(mk, make(hq, [33, 0, 129], None, hq, hkv, 128, 32, F16, 8))


@pytest.mark.parametrize("D,n,hq", [(64, 2600, 3), (96, 9001, 16), (128, 5000, 2), (256, 2600, 16), (128, 40001, 1)])
def test_token_8bit_long_rows_in_pieces(mk, D, n, hq):
    check(mk, make(n + D, [40, n, 0, 40], None, hq, 1, D, 32, F16, 8))


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 0), (31, 33), (32, 32), (33, 4), (64, 16), (100, 1000), (1000, 4),
                                          (1 << 30, 1 << 30)])
def test_token_windows(mk, bits, window, sinks):
    lengths = [0, 1, 7, 16, 31, 32, 33, 34, 35, 36, 48, 63, 64, 65, 66, 67, 96, 97, 99, 100, 101, 128, 130, 257, 700, 1003, 1004, 1005]
    check(mk, make(window + sinks, lengths, None, 4, 2, 64, 16, F16, bits), window=window, sinks=sinks)


@pytest.mark.parametrize("D,dtype,bits", [(96, BF16, 8), (128, F16, 16), (128, BF16, 8), (256, F16, 8), (256, BF16, 16)])
def test_token_windows_wide_heads(mk, D, dtype, bits):
    lengths = [0, 15, 200, 513, 1300, 5000, 3]
    for window, sinks in ((70, 5), (1000, 40), (4999, 0)):
        check(mk, make(D, lengths, None, 6, 2, D, 64, dtype, bits), window=window, sinks=sinks)


@pytest.mark.parametrize("bits", [8, 16])
def test_token_windows_of_rows_in_pieces(mk, bits):
    check(mk, make(9, [9000, 0, 12000, 5], None, 2, 1, 128, 32, F16, bits), window=8000, sinks=100)
    check(mk, make(10, [300 + i for i in range(200)], None, 4, 4, 64, 16, BF16, bits), window=100, sinks=20)


@pytest.mark.parametrize("bits", [8, 16])
def test_token_pages_given_up_and_lengths_past_the_table(mk, bits):
    """Entries that name no page are masked, in a window or outside it; a length past the table counts for positions."""
    args = make(3, [200, 200, 128, 128], None, 4, 2, 64, 16, F16, bits)
    args["table"][0, 1:5] = -1
    args["table"][1, 11] = 10 ** 6
    args["lengths"][2] = 300
    args["lengths"][3] = 2 ** 31 - 1
    for window, sinks in ((None, 0), (100, 4), (60, 16), (250, 0)):
        check(mk, args, window=window, sinks=sinks)


def test_token_table_of_each_head(mk):
    check(mk, make(4, [70, 0, 33], None, 6, 3, 64, 16, F16, 8, per_head=True))
    check(mk, make(5, [170, 0, 90], None, 6, 3, 128, 16, BF16, 16, per_head=True), window=50, sinks=3)


def test_token_without_a_window_is_paged_attention(mk):
    args = cuda(make(6, [300, 0, 5000], None, 8, 2, 128, 32, F16, 16))
    del args["scales"], args["starts"]
    for a, b in zip(mk.paged_attention(**args, return_lse=True), mk.cache_attention(**args, return_lse=True)):
        assert torch.equal(a, b)
    a = mk.cache_attention(**args, window=1 << 30)
    torch.testing.assert_close(a, mk.paged_attention(**args), rtol=0, atol=0)


# ---- several tokens ----

NEW = {"one each": [1] * 9, "drafts": [4, 1, 3, 0, 5, 4, 4, 2, 8], "mixed": [1, 70, 1, 0, 3, 33, 1, 1, 2],
       "prompts": [65, 130, 1, 0, 129, 128, 64, 257, 300]}
CACHED = [0, 5, 300, 7, 130, 64, 1000, 0, 63]


@pytest.mark.parametrize("kind", list(NEW))
@pytest.mark.parametrize("D,dtype,bits", [(64, F16, 16), (64, BF16, 8), (96, F16, 8), (96, BF16, 16), (128, F16, 16), (128, F16, 8),
                                          (128, BF16, 16), (128, BF16, 8), (256, F16, 8), (256, BF16, 16)])
def test_several_tokens(mk, kind, D, dtype, bits):
    new = NEW[kind]
    args = make(D + len(kind), [c + n for c, n in zip(CACHED, new)], new, 4, 2, D, 16, dtype, bits)
    check(mk, args)
    check(mk, args, window=50, sinks=5)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (5, 1), (12, 4), (17, 1), (40, 2), (64, 1), (200, 1)])
@pytest.mark.parametrize("new", [[2, 5], [40, 1, 90]])
def test_several_tokens_head_groups(mk, hq, hkv, new):
    check(mk, make(hq + len(new), [30 + n for n in new], new, hq, hkv, 64, 32, F16, 16))
    check(mk, make(hq + len(new), [30 + n for n in new], new, hq, hkv, 128, 32, BF16, 8), window=20, sinks=2)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 0), (31, 33), (64, 64), (63, 65), (65, 1), (100, 1000), (1 << 30, 3)])
@pytest.mark.parametrize("new", [[3, 1, 4, 2], [200, 130, 64, 65]])
def test_several_tokens_windows(mk, bits, window, sinks, new):
    cached = [0, 63, 200, 129]
    check(mk, make(window, [c + n for c, n in zip(cached, new)], new, 2, 1, 64, 16, F16, bits), window=window, sinks=sinks)


@pytest.mark.parametrize("ps", [16, 32, 128, 1024])
def test_several_tokens_page_sizes(mk, ps):
    for new in ([3, 2, 4], [150, 1, 80]):
        check(mk, make(ps, [ps - 1 + new[0], ps + new[1], 2 * ps + new[2]], new, 2, 1, 64, ps, BF16, 8))


@pytest.mark.parametrize("new,cached,hq,hkv,D", [
    ([4], [9000], 4, 1, 128),        # few rows, keys shared by many work-groups
    ([5, 0, 2], [3000, 10, 7000], 16, 2, 64),
    ([2], [5000], 16, 1, 256),
    ([128], [4000], 1, 1, 128),      # a tile of many rows, its keys shared
    ([200, 3], [2500, 2500], 2, 1, 96),
    ([140], [3000], 1, 1, 256),
])
@pytest.mark.parametrize("bits", [8, 16])
def test_keys_shared_by_work_groups(mk, new, cached, hq, hkv, D, bits):
    args = make(D + len(new), [c + n for c, n in zip(cached, new)], new, hq, hkv, D, 32, F16, bits)
    first = check(mk, args)
    assert torch.equal(first, check(mk, args))  # to the bit, whoever arrives last
    check(mk, args, window=2000, sinks=70)


@pytest.mark.parametrize("new,hq", [(130, 1), (18, 2)])
def test_shared_keys_behind_windows(mk, new, hq):
    """The last tile of a sequence has two rows, whose window is of fewer steps than that of those before; at every remainder."""
    for window in range(1500, 2140, 33):
        check(mk, make(window, [2600], [new], hq, 1, 64, 16, F16, 16), window=window, sinks=window % 40)


@pytest.mark.parametrize("n", [64, 70, 200])
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("least", [1, 65])
def test_keys_of_many_sequences_shared(mk, n, bits, least):
    """Parts are as small as their number allows, found from the lengths of 64 sequences at a time."""
    new = [least + i % 3 for i in range(n)]
    args = make(n + least, [(i * 997) % 3000 + m for i, m in enumerate(new)], new, 1, 1, 64, 32, F16, bits)
    assert torch.equal(check(mk, args), check(mk, args))


@pytest.mark.parametrize("tokens", [4, 5, 8, 9, 16, 17, 24])
@pytest.mark.parametrize("D,bits", [(64, 8), (64, 16), (96, 8), (96, 16), (128, 8), (128, 16), (256, 8), (256, 16)])
def test_rows_that_kernels_are_chosen_by(mk, tokens, D, bits):
    args = make(tokens + D, [700 + tokens, tokens, 90 + tokens], [tokens] * 3, 8, 2, D, 16, BF16, bits)
    check(mk, args)
    check(mk, args, window=300, sinks=20)


@pytest.mark.parametrize("new", [None, [5, 3], [90, 70]])
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-42, 3.0])
def test_scales_of_the_softmax(mk, new, bits, scale):
    check(mk, make(3, [100, 90], new, 4, 2, 64, 16, F16, bits), scale=scale)


@pytest.mark.parametrize("n", [63, 64, 65, 500, 4200])
def test_many_sequences(mk, n):
    new = [(i * 7) % 4 if i % 50 else 20 for i in range(n)]
    cached = [(i * 37) % 23 for i in range(n)]
    check(mk, make(n, [c + m for c, m in zip(cached, new)], new, 1, 1, 64, 16, BF16, 16))
    if n <= 500:
        new = [70 if i % 9 == 0 else 65 for i in range(n)]
        check(mk, make(n, [c + m for c, m in zip(cached, new)], new, 1, 1, 64, 16, F16, 8))


@pytest.mark.parametrize("new", [[6, 6, 6, 6, 6], [90, 90, 90, 90, 90]])
@pytest.mark.parametrize("bits", [8, 16])
def test_tokens_without_a_position_and_past_the_table(mk, new, bits):
    """More new tokens than the length says, lengths of none, tables that end before the tokens, pages and scales that are none."""
    args = make(8, [n + 70 for n in new], new, 4, 2, 64, 16, F16, bits)
    args["lengths"][0] = 3
    args["lengths"][1] = -5
    args["table"][2, 1:3] = -1
    args["table"][2, 4] = 10 ** 7
    args["table"] = args["table"][:, :6]
    if bits == 8:
        s, t = args["scales"], args["table"]
        s[int(t[3, 0]), 0, 0] = 0
        s[int(t[3, 1]), 1, 1] = math.inf
        s[int(t[3, 2]), :, 0] = -1
        s[int(t[3, 3]), :, 1] = 2.0 ** 41
        s[int(t[4, 0])] = 2.0 ** -41
        s[int(t[4, 1]), :, 1] = 2.0 ** -40
        s[int(t[4, 2]), :, 1] = 2.0 ** 40
    check(mk, args)
    check(mk, args, window=30, sinks=2)


def test_token_8bit_scales_that_are_none_and_far_apart(mk):
    args = make(8, [200, 100, 100], None, 4, 2, 64, 16, F16, 8)
    s, t = args["scales"], args["table"]
    for i, x in enumerate((0, math.inf, -1, 2.0 ** 41, 2.0 ** -41, math.nan)):
        s[int(t[0, i]), i % 2, i // 2 % 2] = x
    s[int(t[1, 1]), :, 1], s[int(t[1, 3]), :, 1] = 2.0 ** -40, 2.0 ** 10
    s[t[2, :7].long()] = 0
    check(mk, args)


@pytest.mark.parametrize("new,D,bits", [([5, 3], 128, 16), ([100, 70], 128, 16), ([5, 3], 64, 8), ([100, 70], 256, 8), ([100, 70], 96, 16),
                                        ([4, 6], 96, 8), ([4, 6], 256, 16), ([80, 90], 64, 16)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_values_that_are_not_finite_are_those_that_see_them(mk, new, D, bits, dtype):
    """A later token's infinities and NaN, within a step of its own and in older pages behind a window, reach no token that does not see it."""
    args = make(2, [60 + n for n in new], new, 4, 2, D, 16, dtype, bits)
    v = args["v_cache"]
    for b, n in enumerate(new):
        for pos, ch, x in ((60 + n - 1, 0, math.nan), (60 + n - 2, 3, math.inf), (60 + n // 2, 7, -math.inf), (60 + n // 2, 9, math.nan),
                           (2, 5, math.inf), (20, 11, -math.inf), (20, 3, math.inf)):
            page = int(args["table"][b, pos // 16])
            if bits == 8:
                v.view(torch.uint8)[page, 1, pos % 16, ch] = 0x7F
            else:
                v[page, 1, pos % 16, ch] = x
    check(mk, args)
    check(mk, args, window=30, sinks=4)
    check(mk, args, window=2, sinks=0)


@pytest.mark.parametrize("new", [[6, 3, 8], [90, 30, 128]])
def test_strides_and_out(mk, new):
    """q a slice of a projection's rows, tables with a stride, rows of out that belong to no sequence."""
    args = make(1, [40 + n for n in new], new, 4, 2, 64, 16, F16, 8)
    want, _, tol, _, _ = ref.attention(**args)
    g = cuda(args)
    rows = torch.randn(sum(new) + 5, 4 + 2 + 2, 64, device="cuda").half()
    rows[:sum(new), 1:5] = g["q"]
    g["q"] = rows[:, 1:5]
    wide = torch.full((3, 40), 7, dtype=torch.int32, device="cuda")
    wide[:, :g["table"].shape[1]] = g["table"]
    g["table"] = wide[:, :g["table"].shape[1]]
    out = torch.full((sum(new) + 5, 4, 64), 123.0, dtype=F16, device="cuda")
    got = mk.cache_attention(**g, out=out)
    assert got is out and (out[sum(new):] == 123).all()
    assert ((out[:sum(new)].cpu().double() - want).abs() <= tol).all()
    # views that the kernels cannot read are copied
    odd = torch.empty(sum(new), 4, 65, dtype=F16, device="cuda")
    odd[..., 1:] = g["q"][:sum(new)]
    g["q"] = odd[..., 1:]
    assert torch.equal(mk.cache_attention(**g), out[:sum(new)])


@pytest.mark.parametrize("new", [None, [3, 5, 2], [100, 40, 90]])
def test_offsets_past_32_bits(mk, new):
    """A cache of 2^32 bytes and more, its last pages."""
    hkv, ps, D = 8, 64, 128
    pages = (1 << 32) // (hkv * ps * D) + 40
    lengths = [700, 33, 1000]
    args = make(11, lengths, new, 8, hkv, D, ps, F16, 8, spare=0)
    g = cuda(args)
    k, v, s = mk.kv_cache8(pages, hkv, ps, D)
    n = args["k_cache"].shape[0]
    k.view(torch.uint8)[-n:], v.view(torch.uint8)[-n:], s[-n:] = (x.view(torch.uint8) if x.dtype == E4M3 else x
                                                                 for x in (g["k_cache"], g["v_cache"], g["scales"]))
    table = torch.where(g["table"] >= 0, g["table"] + (pages - n), -1)
    a = mk.cache_attention(**g)
    b = mk.cache_attention(g["q"], k, v, table, g["lengths"], s, g["starts"])
    assert torch.equal(a, b)


# ---- append ----

def fresh(mk, pages, hkv, ps, D, seed=0):
    """Caches that hold older codes, NaN among them, and scales, some of them none."""
    g = gen(seed)
    k, v = (torch.randint(0, 256, (pages, hkv, ps, D), generator=g, dtype=torch.uint8).view(E4M3) for _ in range(2))
    s = 2.0 ** torch.randint(-12, 8, (pages, hkv, 2, ps // 16), generator=g).float()
    s[0::7] = 0
    s[1::7] = math.nan
    return k, v, s


def check_append(mk, k, v, caches, table, lengths, **more):
    kc, vc, sc = caches
    want = ref.append8(k, v, kc, vc, sc, table, lengths, **more)
    on = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in more.items()}
    got = [x.cuda() for x in caches]
    q = torch.randn(k.shape[0], 2 * k.shape[1], k.shape[2]).to(k.dtype)
    q_out = mk.kv_append8(q.cuda(), k.cuda(), v.cuda(), *got, table.cuda(), lengths.cuda(), **on)
    # the queries are kv_append's
    other = mk.kv_cache(*kc.shape, dtype=k.dtype)
    assert torch.equal(q_out, mk.kv_append(q.cuda(), k.cuda(), v.cuda(), *other, table.cuda(), lengths.cuda(), **on))
    for name, x, y in zip(("keys", "values"), want, got):
        y = y.view(torch.uint8).cpu()
        nan = (x & 0x7F) == 0x7F
        assert torch.equal((y & 0x7F) == 0x7F, nan), name
        assert torch.equal(x[~nan], y[~nan]), (name, int((x != y)[~nan].sum()))
    assert torch.equal(torch.nan_to_num(want[2], nan=-3.0), torch.nan_to_num(got[2].cpu(), nan=-3.0))
    return got


def tables(lengths, ps, pages, seed=0, room=0):
    g = gen(seed)
    used = [-(-max(0, n) // ps) for n in lengths]
    table = torch.full((len(lengths), max(1, max(used)) + room), -1, dtype=torch.int32)
    perm = torch.randperm(pages, generator=g).int()
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = perm[at:at + n]
        at += n
    return table


def numbers(seed, shape, dtype):
    """Of many magnitudes, zeros, infinities and NaN among them."""
    g = gen(seed)
    x = torch.randn(shape, generator=g) * 2.0 ** torch.randint(-9, 9, shape[:2] + (1,), generator=g)
    x[torch.rand(shape, generator=g) < 0.05] = 0
    x = x.to(dtype)
    odd = torch.rand(shape, generator=g) < 0.002
    x[odd] = torch.tensor([math.inf, -math.inf, math.nan]).to(dtype)[torch.randint(0, 3, (int(odd.sum()),), generator=g)]
    return x


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("interleaved,part", [(False, 1), (True, 1), (False, 2), (True, 2), (False, 0)])
def test_append8_tokens(mk, D, dtype, interleaved, part):
    lengths = [1, 2, 15, 16, 17, 18, 32, 33, 0, 100, 48, 49, 64, -3]
    n, rot = len(lengths), 0 if part == 0 else D // part // 16 * 16
    k, v = numbers(D, (n, 3, D), dtype), numbers(D + 1, (n, 3, D), dtype)
    check_append(mk, k, v, fresh(mk, 40, 3, 32, D), tables(lengths, 32, 40), torch.tensor(lengths, dtype=torch.int32),
                 cos_sin=mk.rotation_table(200, rot, device="cpu") if rot else None, interleaved=interleaved)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("ps", [16, 64])
def test_append8_prompts(mk, D, dtype, ps):
    new = [1, 16, 5, 0, 33, 100, 17, 2, 31]
    cached = [0, 0, 11, 4, 15, 30, 16, 47, 1]
    lengths = [c + n for c, n in zip(cached, new)]
    lengths[6] = 3  # more new tokens than the length says
    k, v = numbers(D, (sum(new), 5, D), dtype), numbers(D + 1, (sum(new), 5, D), dtype)
    starts = torch.tensor([0] + new).cumsum(0).int()
    for interleaved in (False, True):
        check_append(mk, k, v, fresh(mk, 40, 5, ps, D), tables(lengths, ps, 40), torch.tensor(lengths, dtype=torch.int32),
                     cos_sin=mk.rotation_table(200, D, device="cpu"), interleaved=interleaved, starts=starts)


def test_append8_skips(mk):
    """Positions past the table or the angles, and pages that are none."""
    for new in (None, [40, 40, 40, 40]):
        lengths = [100, 60, 70, 90]
        table = tables(lengths, 16, 40)
        table[1, 2:] = -1
        table[2, 3] = 10 ** 6
        table = table[:, :5]
        n = 4 if new is None else sum(new)
        k, v = numbers(1, (n, 2, 64), F16), numbers(2, (n, 2, 64), F16)
        check_append(mk, k, v, fresh(mk, 40, 2, 16, 64), table, torch.tensor(lengths, dtype=torch.int32), cos_sin=mk.rotation_table(75, 32, device="cpu"),
                     starts=None if new is None else torch.tensor([0] + new).cumsum(0).int())


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_append8_every_number(mk, dtype):
    """Every number of the type as a value, sorted, so that a block's are of a kind: the rounding of each."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(dtype)
    order = torch.argsort(x.float().abs().nan_to_num(0), stable=True)
    v = x[order].view(-1, 1, 256)
    n = v.shape[0]
    k = v.flip(0).contiguous()
    check_append(mk, k, v, fresh(mk, 20, 1, 16, 256), tables([n], 16, 20), torch.tensor([n], dtype=torch.int32),
                 starts=torch.tensor([0, n], dtype=torch.int32))
    many = torch.full((n,), 1, dtype=torch.int32)
    check_append(mk, k, v, fresh(mk, n, 1, 16, 256), tables([1] * n, 16, n), many)  # each in a block of its own


def test_append8_scales_at_the_border(mk):
    """448 times a power of two, and the next number above and below it."""
    near = [448.0, 448.25, 447.75, 224.0, 224.125, 1.75, 1.751, 1.749, 2.0 ** -14 * 1.75, 65504.0, 6e-8, 0.0]
    v = torch.tensor(near).half().view(-1, 1, 1).repeat(1, 1, 64)
    n = len(near)
    got = check_append(mk, v, v, fresh(mk, n, 1, 16, 64), tables([1] * n, 16, n), torch.ones(n, dtype=torch.int32))
    s = got[2].cpu()[tables([1] * n, 16, n)[:, 0].long(), 0, 1, 0]
    assert s[:8].tolist() == [1, 2, 1, 0.5, 1, 2.0 ** -8, 2.0 ** -7, 2.0 ** -8] and s[-1] == 2.0 ** -40
    big = torch.tensor([3e38, -3e38, 1e-38, 2.0 ** 49, 448 * 2.0 ** 40]).bfloat16().view(-1, 1, 1).repeat(1, 1, 64)
    check_append(mk, big, big, fresh(mk, 5, 1, 16, 64), tables([1] * 5, 16, 5), torch.ones(5, dtype=torch.int32))


@pytest.mark.parametrize("D,dtype", [(64, F16), (128, BF16), (96, F16)])
def test_append8_step_by_step(mk, D, dtype):
    """A block that grows token by token, each of another magnitude: codes rounded anew as the scale grows; and in pieces of some."""
    hkv, ps, caches = 2, 16, fresh(mk, 12, 2, 16, D)
    table = tables([40, 40, 40], ps, 12)
    g = gen(5)
    caches = [x.clone() for x in caches]
    for n in range(1, 41):
        k, v = (torch.randn(3, hkv, D, generator=g) * 2.0 ** torch.randint(-6, 7, (3, hkv, 1), generator=g) for _ in range(2))
        caches = [x.cpu() for x in check_append(mk, k.to(dtype), v.to(dtype), caches, table, torch.full((3,), n, dtype=torch.int32))]
    at = 0
    while at < 38:
        new = [int(x) for x in torch.randint(0, 7, (3,), generator=g)]
        new[0] = max(1, new[0])
        k, v = (numbers(at + i, (sum(new), hkv, D), dtype) for i in range(2))
        lengths = torch.tensor([at + n for n in new], dtype=torch.int32)
        caches = [x.cpu() for x in check_append(mk, k, v, caches, table, lengths, starts=torch.tensor([0] + new).cumsum(0).int())]
        at += min(new)
        at += 1 if min(new) == 0 else 0


def test_append8_strides(mk):
    """q, k and v slices of one projection's rows; out in the place of q."""
    new, hkv, D = [20, 3, 40], 2, 128
    T = sum(new)
    rows = numbers(3, (T, 8, D), F16)
    q, k, v = rows[:, :4], rows[:, 4:6], rows[:, 6:]
    lengths, table = torch.tensor([25, 3, 40], dtype=torch.int32), tables([25, 3, 40], 32, 10)
    starts, cs = torch.tensor([0] + new).cumsum(0).int(), mk.rotation_table(60, D, device="cpu")
    caches = fresh(mk, 10, hkv, 32, D)
    want = ref.append8(k, v, *caches, table, lengths, cos_sin=cs, starts=starts)
    on = [x.cuda() for x in caches]
    g = rows.cuda()
    mk.kv_append8(g[:, :4], g[:, 4:6], g[:, 6:], *on, table.cuda(), lengths.cuda(), cs.cuda(), starts.cuda())
    finite = (want[0] & 0x7F) != 0x7F
    assert torch.equal(on[0].view(torch.uint8).cpu()[finite], want[0][finite])
    finite = (want[1] & 0x7F) != 0x7F
    assert torch.equal(on[1].view(torch.uint8).cpu()[finite], want[1][finite])
    dense = q.contiguous().cuda()
    a = mk.kv_append8(dense.clone(), g[:, 4:6], g[:, 6:], *on, table.cuda(), lengths.cuda(), cs.cuda(), starts.cuda())
    b = mk.kv_append8(dense, g[:, 4:6], g[:, 6:], *on, table.cuda(), lengths.cuda(), cs.cuda(), starts.cuda(), out=dense)
    assert b is dense and torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_append8_past_32_bits(mk):
    hkv, ps, D = 8, 64, 128
    pages = (1 << 32) // (hkv * ps * D) + 8
    k, v, s = mk.kv_cache8(pages, hkv, ps, D)
    for new in (None, [70]):
        n = 1 if new is None else 70
        x = numbers(n, (n, hkv, D), F16)
        table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32)
        lengths = torch.tensor([n], dtype=torch.int32)
        starts = None if new is None else torch.tensor([0, n], dtype=torch.int32)
        small = [torch.zeros(2, hkv, ps, D, dtype=torch.uint8).view(E4M3), torch.zeros(2, hkv, ps, D, dtype=torch.uint8).view(E4M3),
                 torch.zeros(2, hkv, 2, ps // 16)]
        want = ref.append8(x, x, *small, torch.tensor([[1, 0]], dtype=torch.int32), lengths, starts=starts)
        mk.kv_append8(x.cuda(), x.cuda(), x.cuda(), k, v, s, table.cuda(), lengths.cuda(), starts=None if starts is None else starts.cuda())
        for a, b in zip(want[:2], (k, v)):
            b = b[-2:].view(torch.uint8).cpu()
            fine = (a & 0x7F) != 0x7F
            assert torch.equal(a[fine], b[fine])
        assert torch.equal(want[2], s[-2:].cpu())


# ---- page tables ----

def check_pages(mk, table, lengths, new, free, count, ps, tokens, window=None, sinks=0):
    want = ref.assign_pages(table, lengths, new, free, count, ps, tokens, window, sinks)
    on = [x.cuda() for x in (table, lengths, new, free, torch.tensor([count], dtype=torch.int32))]
    starts, slots = mk.assign_pages(*on, ps, tokens, window=window, sinks=sinks)
    for name, x, y in zip(("table", "lengths", "free", "count", "starts", "slots"), want, (on[0], on[1], on[3], on[4], starts, slots)):
        x = torch.tensor([x], dtype=torch.int32) if name == "count" else x
        assert torch.equal(x, y.cpu()), (name, x, y)
    return want


def state(seed, B, ps, most, spare, ends=0.2, least=0, width=None, windowed=False):
    """A random state of B sequences: table, lengths, free list and its count."""
    g = gen(seed)
    lengths = torch.randint(0, most + 1, (B,), generator=g).int()
    used = (lengths + ps - 1) // ps
    pages = int(used.sum()) + spare
    perm = torch.randperm(pages, generator=g).int()
    width = width or int(used.max()) + 4
    table = torch.full((B, width), -1, dtype=torch.int32)
    have = torch.arange(width) < used[:, None]
    table[have] = perm[:int(used.sum())]
    if windowed:
        table[have & (torch.rand(have.shape, generator=g) < 0.15)] = -1
    free = torch.full((pages,), -7, dtype=torch.int32)
    free[:spare] = perm[int(used.sum()):]
    new = torch.randint(least, 3 * ps, (B,), generator=g).int()
    new[torch.rand(B, generator=g) < ends] = -1
    return table, lengths, new, free, spare


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 200, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("tokens", [0, 1, 100, 2048, 2049, 4096, 4097, 200000])
def test_pages_of_many_sequences(mk, B, tokens):
    table, lengths, new, free, count = state(B + tokens, B, 16, 200, 3 * B)
    check_pages(mk, table, lengths, new, free, count, 16, tokens)
    new[:] = torch.where(new < 0, new, 1)
    check_pages(mk, table, lengths, new, free, count, 16, tokens)


@pytest.mark.parametrize("spare", [0, 1, 5, 40, 1000])
@pytest.mark.parametrize("ps", [16, 32, 1024])
def test_pages_run_out(mk, spare, ps):
    for ends in (0, 0.3):
        table, lengths, new, free, count = state(spare + ps, 50, ps, 5 * ps, spare, ends=ends)
        check_pages(mk, table, lengths, new, free, count, ps, 100000)
        new[3], new[10] = 2 ** 31 - 1, -(2 ** 31)  # never fits; ends
        check_pages(mk, table, lengths, new, free, count, ps, 100000)


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 16), (17, 1), (100, 33), (1000, 0), (1 << 30, 5), (64, 1 << 30)])
def test_pages_behind_a_window(mk, window, sinks):
    for windowed in (False, True):
        table, lengths, new, free, count = state(window, 120, 16, 3000, 200, windowed=windowed)
        check_pages(mk, table, lengths, new, free, count, 16, 5000, window, sinks)


def test_pages_at_the_edges(mk):
    # full rows, lengths past the table and below none, free counts that are none, free entries that name no page
    table, lengths, new, free, count = state(1, 20, 16, 100, 60, width=7)
    lengths[0], lengths[1], lengths[2] = 112, 5000, -4
    new[0], new[1], new[2], new[3] = 1, -1, 5, 0
    check_pages(mk, table, lengths, new, free, count, 16, 500)
    check_pages(mk, table, lengths, new, free, -3, 16, 500)
    lengths[1] = 0
    new[1] = 3
    free[50:60] = torch.tensor([-1, 10 ** 6, 3, -9, 2, 1, 0, 4, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)
    check_pages(mk, table, lengths, new, free, count, 16, 500)
    free[:] = torch.arange(len(free))
    check_pages(mk, table, lengths, new, free, 10 ** 9, 16, 500)
    # pages given back beyond the list's room are not kept
    new[:] = -1
    check_pages(mk, table, lengths, new, free, len(free) - 2, 16, 500)
    # no sequences
    check_pages(mk, torch.zeros(0, 3, dtype=torch.int32), torch.zeros(0, dtype=torch.int32), torch.zeros(0, dtype=torch.int32), free, 5, 16, 9)


def test_pages_of_strided_rows(mk):
    table, lengths, new, free, count = state(4, 30, 32, 500, 90)
    want = ref.assign_pages(table, lengths, new, free, count, 32, 3000)
    wide = torch.full((30, table.shape[1] + 9), -5, dtype=torch.int32, device="cuda")
    wide[:, 3:3 + table.shape[1]] = table.cuda()
    on = wide[:, 3:3 + table.shape[1]]
    mk.assign_pages(on, lengths.cuda(), new.cuda(), free.cuda(), torch.tensor([count], dtype=torch.int32, device="cuda"), 32, 3000)
    assert torch.equal(on.cpu(), want[0]) and (wide[:, :3] == -5).all() and (wide[:, 3 + table.shape[1]:] == -5).all()


# ---- together, on streams, in graphs ----

def serve(mk, bits, dtype, window, sinks, seed=0):
    """A server's state: a pool, tables, and what a step of one layer does with new tokens' rows."""
    hq, hkv, D, ps, B, pages, width = 4, 2, 64, 16, 6, 200, 40
    st = dict(table=torch.full((B, width), -1, dtype=torch.int32, device="cuda"), lengths=torch.zeros(B, dtype=torch.int32, device="cuda"),
              free=torch.randperm(pages, generator=gen(seed)).int().cuda(), count=torch.tensor([pages], dtype=torch.int32, device="cuda"),
              cs=mk.rotation_table(1000, D))
    if bits == 8:
        st["k"], st["v"], st["s"] = mk.kv_cache8(pages, hkv, ps, D)
    else:
        st["k"], st["v"] = mk.kv_cache(pages, hkv, ps, D, dtype=dtype)
        st["s"] = None

    def step(rows, new, tokens, several=True):
        q, k, v = rows.split([hq, hkv, hkv], 1)
        starts, slots = mk.assign_pages(st["table"], st["lengths"], new, st["free"], st["count"], ps, tokens, window=window, sinks=sinks)
        starts = starts if several else None
        if bits == 8:
            q = mk.kv_append8(q, k, v, st["k"], st["v"], st["s"], st["table"], st["lengths"], st["cs"], starts)
        else:
            q = mk.kv_append(q, k, v, st["k"], st["v"], st["table"], st["lengths"], st["cs"], starts)
        return q, mk.cache_attention(q, st["k"], st["v"], st["table"], st["lengths"], st["s"], starts, window, sinks), starts, slots
    return st, step, (hq, hkv, D, B)


def expect(st, q, starts, window, sinks):
    args = dict(q=q.cpu(), k_cache=st["k"].cpu(), v_cache=st["v"].cpu(), table=st["table"].cpu(), lengths=st["lengths"].cpu(),
                scales=None if st["s"] is None else st["s"].cpu(), starts=None if starts is None else starts.cpu())
    return ref.attention(**args, window=window, sinks=sinks)


@pytest.mark.parametrize("bits,dtype", [(8, F16), (16, F16), (8, BF16)])
@pytest.mark.parametrize("window,sinks", [(None, 0), (40, 5)])
def test_steps_of_a_server(mk, bits, dtype, window, sinks):
    """Prompts, decode steps, drafted tokens, sequences that end and others that take their place."""
    st, step, (hq, hkv, D, B) = serve(mk, bits, dtype, window, sinks)
    g = gen(1)
    plans = [[30, 70, 1, 0, 130, 9]] + [[1] * 6] * 3 + [[3, 1, 4, 2, 4, 1], [-1, 1, 1, 50, 1, -1], [20, 1, 1, 1, 0, 77]] + [[1] * 6] * 20
    seen = torch.zeros(200, dtype=torch.int64)
    for new in plans:
        tokens = sum(max(0, n) for n in new)
        rows = torch.randn(tokens, hq + 2 * hkv, D, generator=g).to(dtype).cuda()
        ones = new == [1] * 6
        q, o, starts, slots = step(rows, torch.tensor(new, dtype=torch.int32).cuda(), tokens, several=not ones)
        want, _, tol, _, mine = expect(st, q, starts, window, sinks)
        assert mine.all() and ((o.cpu().double() - want).abs() <= tol).all()
        n_free = int(st["count"])
        named = st["table"][st["table"] >= 0].long().cpu()
        both = torch.cat([named, st["free"][:n_free].long().cpu()])
        assert len(both) == 200 and len(both.unique()) == 200  # every page is somewhere, once
        # the slots are where the keys went
        assert (slots >= 0).all() and len(slots.unique()) == tokens


@pytest.mark.parametrize("bits", [8, 16])
def test_steps_as_graphs(mk, bits):
    """A decode step and a prompts' step as two graphs of one stream's workspace, replayed in turn with eager work between; every replay
    against the eager form."""
    st, step, (hq, hkv, D, B) = serve(mk, bits, F16, 300, 4)
    other, eager, _ = serve(mk, bits, F16, 300, 4)
    g = gen(2)
    rows = {n: torch.randn(n, hq + 2 * hkv, D, generator=g).half().cuda() for n in (6, 90)}
    new = {6: torch.ones(6, dtype=torch.int32).cuda(), 90: torch.tensor([20, 3, 40, 0, 26, 1], dtype=torch.int32).cuda()}
    graphs, outs = {}, {}
    keep = {k: x.clone() for k, x in st.items() if isinstance(x, torch.Tensor)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())  # the copies are made before the first steps change what they are of
    with torch.cuda.stream(side):
        for n in (6, 90):
            step(rows[n], new[n], n)
    torch.cuda.synchronize()
    for n in (6, 90):
        graphs[n] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[n], stream=side):
            outs[n] = step(rows[n], new[n], n)
    for k, x in keep.items():
        (st[k].view(torch.uint8) if st[k].dtype == E4M3 else st[k]).copy_(x.view(torch.uint8) if x.dtype == E4M3 else x)
    for n in (90, 6, 6, 90, 6, 90, 6, 6):
        rows[n].copy_(torch.randn(rows[n].shape, generator=g))
        graphs[n].replay()
        want = eager(rows[n], new[n], n)
        torch.cuda.synchronize()
        for a, b in zip(outs[n], want):
            assert torch.equal(a, b)
    for k, x in other.items():
        if isinstance(x, torch.Tensor):
            assert torch.equal(st[k].view(torch.uint8), x.view(torch.uint8)) if x.dtype == E4M3 else torch.equal(st[k], x)


def test_two_streams_at_once(mk):
    """Calls on two streams at a time have a workspace each."""
    args = [cuda(make(i, [3000, 4], [5, 2], 8, 2, 128, 32, F16, 8)) for i in range(2)]
    want = [mk.cache_attention(**a) for a in args]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(mk.cache_attention(**args[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i]) for i in range(2) for x in got[i])


def test_workspace_of_the_caller(mk):
    args = cuda(make(1, [3000], [4], 8, 2, 64, 32, F16, 16))
    want = mk.cache_attention(**args)
    ws = mk.Workspace("cuda")
    assert torch.equal(mk.cache_attention(**args, workspace=ws), want) and ws.buf.numel() > 1 << 20
    assert (ws.buf[:1 << 20] == 0).all()  # counters are back at zero
    table, lengths, new, free, count = (x.cuda() if isinstance(x, torch.Tensor) else torch.tensor([x], dtype=torch.int32).cuda()
                                        for x in state(1, 30, 16, 100, 60))
    mk.assign_pages(table, lengths, new, free, count, 16, 100, workspace=ws)
    assert (ws.buf[:1 << 20] == 0).all()


# ---- operators and refusals ----

def test_registered_operators(mk):
    ops = torch.ops.marlin_mi355x
    a = cuda(make(1, [30, 70], [4, 40], 4, 2, 64, 16, F16, 8))
    o, lse = ops.cache_attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], a["scales"], a["starts"], 20, 3)
    want = mk.cache_attention(**a, window=20, sinks=3, return_lse=True)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    torch.library.opcheck(ops.cache_attention, (a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"], a["scales"], a["starts"], 20, 3),
                          test_utils="test_faketensor")  # the others multiply their arguments, which codes do not take
    b = cuda(make(1, [30, 70], [4, 40], 4, 2, 64, 16, F16, 16))
    torch.library.opcheck(ops.cache_attention, (b["q"], b["k_cache"], b["v_cache"], b["table"], b["lengths"], None, b["starts"], 20, 3))
    s = [x.cuda() if isinstance(x, torch.Tensor) else torch.tensor([x], dtype=torch.int32).cuda() for x in state(1, 8, 16, 60, 30)]
    torch.library.opcheck(ops.assign_pages, (*s, 16, 100, 40, 2))
    k = torch.randn(2, 2, 64).half().cuda()
    caches = mk.kv_cache8(9, 2, 16, 64)
    torch.library.opcheck(ops.kv_append8, (k, k, k, *caches, a["table"][:, :2].contiguous(), torch.tensor([3, 4], dtype=torch.int32).cuda()),
                          test_utils="test_faketensor")


def test_gradients_and_tangents_are_refused(mk):
    a = cuda(make(1, [30, 70], [4, 40], 4, 2, 64, 16, F16, 8))
    a["q"].requires_grad_()
    o = mk.cache_attention(**a)
    with pytest.raises(Exception):
        o.sum().backward()
    k = torch.randn(2, 2, 64).half().cuda()
    q = k.clone().requires_grad_()
    with pytest.raises(Exception):
        mk.kv_append8(q, k, k, *mk.kv_cache8(9, 2, 16, 64), a["table"][:, :2].contiguous(), torch.tensor([3, 4], dtype=torch.int32).cuda()).sum().backward()
    with torch.no_grad(), torch.autograd.forward_ad.dual_level():
        a["q"] = torch.autograd.forward_ad.make_dual(a["q"].detach(), torch.ones_like(a["q"]))
        with pytest.raises(RuntimeError):
            mk.cache_attention(**a)


def test_refusals(mk):
    a = cuda(make(1, [30, 70], [4, 40], 4, 2, 64, 16, F16, 8))
    one = cuda(make(1, [30, 70], None, 4, 2, 64, 16, F16, 8))

    def refused(kind, f, *args, **change):
        with pytest.raises(kind):
            f(*args, **change)
    call = mk.cache_attention
    for kind, change in ((TypeError, dict(scales=None)), (TypeError, dict(q=a["q"].float())), (TypeError, dict(scales=a["scales"].half())),
                         (ValueError, dict(scales=a["scales"][:, :, :1])), (ValueError, dict(scales=a["scales"][1:])),
                         (ValueError, dict(window=0)), (ValueError, dict(window=-3)), (mk.MarlinError, dict(sinks=-1)),
                         (mk.MarlinError, dict(window=(1 << 30) + 1)), (TypeError, dict(window=2.5)), (mk.MarlinError, dict(scale=math.nan)),
                         (TypeError, dict(table=a["table"].long())), (ValueError, dict(table=a["table"][:, None])),
                         (ValueError, dict(starts=a["starts"][:2])), (ValueError, dict(starts=None)), (TypeError, dict(starts=a["starts"].long())),
                         (ValueError, dict(lengths=a["lengths"][:1])), (ValueError, dict(q=a["q"][..., :32])),
                         (mk.MarlinError, dict(q=a["q"][:, :3])), (ValueError, dict(out=a["q"][:3])), (ValueError, dict(k_cache=a["k_cache"][1:])),
                         (TypeError, dict(v_cache=a["v_cache"].half())), (TypeError, dict(lengths=a["lengths"].cpu()))):
        refused(kind, call, **{**a, **change})
    refused(ValueError, call, **{**one, "q": one["q"][:1]})
    k = torch.randn(2, 2, 64).half().cuda()
    ints = torch.tensor([3, 4], dtype=torch.int32).cuda()
    kc, vc, s = mk.kv_cache8(9, 2, 16, 64)
    good = dict(q=k, k=k, v=k, k_cache=kc, v_cache=vc, scales=s, table=one["table"][:, :2].contiguous(), lengths=ints)
    mk.kv_append8(**good)
    for kind, change in ((TypeError, dict(k=k.bfloat16())), (TypeError, dict(q=k.float())), (TypeError, dict(k_cache=kc.half())),
                         (ValueError, dict(scales=s[:3])), (TypeError, dict(scales=s.double())), (ValueError, dict(v=k[:, :1])),
                         (ValueError, dict(lengths=ints[:1])), (ValueError, dict(starts=ints)), (TypeError, dict(cos_sin=s.double()[0, 0])),
                         (mk.MarlinError, dict(cos_sin=torch.zeros(9, 24).cuda())), (ValueError, dict(out=k[:1])),
                         (ValueError, dict(k=k[:1], v=k[:1]))):
        refused(kind, mk.kv_append8, **{**good, **change})
    t, n, new, free, count = (x.cuda() if isinstance(x, torch.Tensor) else torch.tensor([x], dtype=torch.int32).cuda()
                              for x in state(1, 8, 16, 60, 30))
    good = dict(table=t, lengths=n, new=new, free=free, free_count=count, page_size=16, tokens=50)
    for kind, change in ((TypeError, dict(table=t.long())), (ValueError, dict(lengths=n[:3])), (ValueError, dict(new=new[:3])),
                         (ValueError, dict(free_count=free[:2])), (mk.MarlinError, dict(page_size=24)), (mk.MarlinError, dict(page_size=8)),
                         (mk.MarlinError, dict(tokens=-1)), (mk.MarlinError, dict(tokens=(1 << 24) + 1)), (ValueError, dict(window=0)),
                         (mk.MarlinError, dict(sinks=-1)), (ValueError, dict(table=t[:1].expand(8, -1))), (TypeError, dict(free=free.cpu())),
                         (mk.MarlinError, dict(free=free[:0])), (TypeError, dict(tokens=2.5))):
        refused(kind, mk.assign_pages, **{**good, **change})


@pytest.mark.parametrize("more", [["--bits", "8"], ["--window", "40", "--sinks", "3"], ["--bits", "8", "--window", "64", "--page-size", "32"]])
def test_example_layer(mk, more):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_layer.py")
    spec = importlib.util.spec_from_file_location("decode_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(["--hidden", "512", "--heads", "8", "--kv-heads", "2", "--head-dim", "64", "--sequences", "5",
                         "--prompt", "90", "--steps", "9", *more])

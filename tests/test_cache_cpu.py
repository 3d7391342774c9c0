"""The 8-bit cache, windows, several new tokens and page tables without a GPU: the argument structs of marlin.h against the binding's, every
refusal that the host makes before any HIP call, the native call module, the PyTorch operators' fake implementations, and the plain
forms that the GPU tests compare with, against second ways and with mistakes planted in copies of them."""
import ctypes
import inspect
import math
import os
import random
import re

import pytest

torch = pytest.importorskip("torch")

import cache_reference as ref  # noqa: E402
import kv_reference  # noqa: E402
import paper_2408_11743_amd as mk  # noqa: E402
from paper_2408_11743_amd import _binding as B  # noqa: E402
from paper_2408_11743_amd import cache  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULLP, SHAPE, ALIGN, WS, ARG = 0, 1, 2, 4, 5, 8
FAKE = 0x10000  # aligned, never dereferenced: every call below fails validation first
E4M3 = torch.float8_e4m3fn


def struct_fields(name):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "marlin.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, text).group(1)
    fields = []
    for line in body.split(";"):
        line = line.strip()
        if line:
            assert re.match(r"(const )?(void|float|int32_t|int64_t) \*|(u?int64_t|double) ", line), line  # 8 bytes each
            fields += [n.strip(" *") for n in re.sub(r"^(const )?\w+ ", "", line).split(",")]
    return fields


@pytest.mark.parametrize("name,fields,pack", [
    ("marlin_kv_append8_args", B.KV_APPEND8_FIELDS, B.pack_kv_append8),
    ("marlin_cache_attention_args", B.CACHE_ATTENTION_FIELDS, B.pack_cache_attention),
    ("marlin_assign_pages_args", B.ASSIGN_PAGES_FIELDS, B.pack_assign_pages)])
def test_structs_are_the_bindings(name, fields, pack):
    assert struct_fields(name) == fields
    packed = pack(*range(len(fields)))
    assert len(packed) == 8 * len(fields)
    if "scale" in fields:
        i = fields.index("scale")
        assert ctypes.c_double.from_buffer_copy(packed, 8 * i).value == i


APPEND = dict(q=FAKE, k=FAKE, v=FAKE, q_row=1024, q_head=128, k_row=1024, k_head=128, v_row=1024, v_head=128, q_out=FAKE,
              k_cache=FAKE, v_cache=FAKE, scales=FAKE, cos_sin=FAKE, positions=4096, rot=128, interleaved=0, table=FAKE,
              table_row=8, lengths=FAKE, starts=None, tokens=3, B=3, heads=8, kv_heads=2, head_dim=128, pages=100,
              page_size=16, width=8, dtype=0)
ATTEND = dict(q=FAKE, q_row=1024, q_head=128, k_cache=FAKE, v_cache=FAKE, scales=FAKE, table=FAKE, table_row=8, table_head=0,
              lengths=FAKE, starts=None, tokens=3, window=0, sinks=0, out=FAKE, lse=None, workspace=FAKE,
              workspace_bytes=1 << 40, B=3, heads=8, kv_heads=2, head_dim=128, pages=100, page_size=16, width=8, scale=0.1, dtype=0)
PAGES = dict(table=FAKE, table_row=8, lengths=FAKE, new_tokens=FAKE, free_pages=FAKE, free_count=FAKE, starts=FAKE, slots=FAKE,
             workspace=FAKE, workspace_bytes=1 << 40, B=3, width=8, pages=100, page_size=16, tokens=9, window=0, sinks=0)
CALLS = {"append": (mk.marlin_kv_append8, APPEND), "attend": (mk.marlin_cache_attention, ATTEND), "pages": (mk.marlin_assign_pages, PAGES)}


def status(which, **change):
    call, args = CALLS[which]
    try:
        call(**{**args, **change})
    except B.MarlinError as e:
        return e.status
    return OK


@pytest.mark.parametrize("which", ["append", "attend"])
def test_shared_refusals(which):
    for change in (dict(B=-1), dict(B=(1 << 16) + 1), dict(heads=7), dict(kv_heads=0), dict(heads=1), dict(kv_heads=3),
                   dict(heads=2048, kv_heads=2), dict(head_dim=80), dict(head_dim=0), dict(head_dim=512), dict(pages=0),
                   dict(pages=1 << 31), dict(page_size=8), dict(page_size=24), dict(page_size=2048), dict(page_size=-16),
                   dict(width=0), dict(width=(1 << 26) + 1), dict(q_row=4), dict(q_head=129), dict(q_row=-8), dict(table_row=-1),
                   dict(tokens=2), dict(tokens=-1, starts=FAKE), dict(tokens=(1 << 24) + 1, starts=FAKE)):
        assert status(which, **change) == SHAPE, change
    for name in ("q", "k_cache", "v_cache", "table", "lengths"):
        assert status(which, **{name: None}) == NULLP, name
    for name in ("q", "k_cache", "v_cache"):
        assert status(which, **{name: FAKE + 8}) == ALIGN, name
    for name in ("table", "lengths", "scales", "starts"):
        assert status(which, **{name: FAKE + 2}) == ALIGN, name
    assert status(which, dtype=2) == ARG and status(which, dtype=-1) == ARG
    # nothing to do: nothing is looked at
    assert status(which, B=0, tokens=0, q=None, table=None) == OK
    assert status(which, tokens=0, starts=FAKE, q=None, k_cache=None) == OK


def test_append_refusals():
    for name in ("k", "v", "q_out", "scales", "cos_sin"):
        assert status("append", **{name: None}) == NULLP, name
    for name in ("k", "v", "q_out", "cos_sin"):
        assert status("append", **{name: FAKE + 4}) == ALIGN, name
    for change in (dict(rot=8), dict(rot=-16), dict(rot=144), dict(interleaved=2), dict(interleaved=-1)):
        assert status("append", **change) == ARG, change
    for change in (dict(positions=0), dict(positions=(1 << 30) + 1), dict(k_row=12), dict(v_head=-8)):
        assert status("append", **change) == SHAPE, change


def test_attention_refusals():
    for name in ("out", "workspace"):
        assert status("attend", **{name: None}) == NULLP, name
        assert status("attend", **{name: FAKE + 8}) == ALIGN, name
    assert status("attend", lse=FAKE + 2) == ALIGN
    for scale in (math.nan, math.inf, -math.inf, 1e300, 3e38):
        assert status("attend", scale=scale) == ARG, scale
    for change in (dict(window=-1), dict(window=(1 << 30) + 1), dict(sinks=-1), dict(sinks=(1 << 30) + 1)):
        assert status("attend", **change) == ARG, change
    assert status("attend", table_head=-1) == SHAPE
    assert status("attend", table_head=4, starts=FAKE) == SHAPE  # a table for each head is of one token a sequence
    assert status("attend", B=1 << 16, tokens=1 << 16, heads=64, kv_heads=64, width=1 << 16) == SHAPE  # too many steps to number
    assert status("attend", starts=FAKE, tokens=1 << 24, heads=128, kv_heads=1) == SHAPE  # too many rows of a head
    need = mk.marlin_paged_attention_workspace_bytes(128)
    assert mk.marlin_cache_attention_workspace_bytes(0, 3, 3, 8, 2, 128) == need
    assert status("attend", workspace_bytes=need - 1) == WS
    need = mk.marlin_cache_attention_workspace_bytes(1, 3, 3, 8, 2, 128)
    assert need > 1 << 20 and status("attend", starts=FAKE, workspace_bytes=need - 1) == WS
    assert [mk.marlin_cache_attention_workspace_bytes(1, *x) for x in ((-1, 3, 8, 2, 128), (3, -1, 8, 2, 128), (3, 3, 8, 3, 128),
                                                                      (3, 3, 8, 2, 80), (1 << 24, 3, 1024, 2, 64))] == [0] * 5
    # the workspace stays within bounds whatever the sizes
    rng = random.Random(0)
    for _ in range(300):
        kv_heads = rng.choice([1, 2, 8, 40])
        need = mk.marlin_cache_attention_workspace_bytes(1, rng.choice([1, 7, 100, 4000, 1 << 20]), rng.choice([1, 5, 300, 1 << 16]),
                                                         kv_heads * rng.choice([1, 4, 16]), kv_heads, rng.choice([64, 96, 128, 256]))
        assert 1 << 20 <= need <= 160 << 20


def test_pages_refusals():
    for change in (dict(B=-1), dict(B=(1 << 16) + 1), dict(pages=0), dict(pages=1 << 31), dict(page_size=8), dict(page_size=24),
                   dict(page_size=2048), dict(width=0), dict(width=(1 << 26) + 1), dict(table_row=-1), dict(tokens=-1), dict(tokens=(1 << 24) + 1)):
        assert status("pages", **change) == SHAPE, change
    for name in ("table", "lengths", "new_tokens", "free_pages", "free_count", "starts", "slots", "workspace"):
        assert status("pages", **{name: None}) == NULLP, name
        assert status("pages", **{name: FAKE + 2}) == ALIGN, name
    assert status("pages", slots=FAKE + 4) == ALIGN
    for change in (dict(window=-1), dict(window=(1 << 30) + 1), dict(sinks=-1), dict(sinks=(1 << 30) + 1)):
        assert status("pages", **change) == ARG, change
    need = mk.marlin_assign_pages_workspace_bytes(3)
    assert status("pages", workspace_bytes=need - 1) == WS
    assert mk.marlin_assign_pages_workspace_bytes(-1) == 0 == mk.marlin_assign_pages_workspace_bytes((1 << 16) + 1)


def test_binding_names_every_field():
    args = dict(ATTEND)
    del args["window"]
    with pytest.raises(TypeError, match="window"):
        mk.marlin_cache_attention(**args)


def test_native_module_leaves_host_tensors_to_python():
    fast = cache._connect()
    x, ints = torch.zeros(2, 4, 64).half(), torch.zeros(2, 2, dtype=torch.int32)
    k, v, s = mk.kv_cache8(3, 2, 16, 64, device="cpu")
    assert k.dtype == v.dtype == E4M3 and k.shape == (3, 2, 16, 64) and s.shape == (3, 2, 2, 1) and not s.any()
    assert fast.kv_append8(x, x[:, :2], x[:, :2], k, v, s, ints, ints[0], None, None, False, None) is None
    assert fast.cache_attention(x, k, v, ints, ints[0], s, None, None, 0, None, False, None, None) is None
    assert fast.assign_pages(ints, ints[0], ints[0], ints[0], ints[0, :1], 16, 4, None, 0, None) is None
    assert fast.assign_pages(ints) is None and fast.cache_attention(None, 1, "x", ints, 0, 0, 0, 0, 0, 0, 0, 0, 0) is None
    with pytest.raises(TypeError):
        mk.cache_attention(x, k, v, ints, ints[0], s)
    with pytest.raises(TypeError):
        mk.kv_append8(x, x[:, :2], x[:, :2], k, v, s, ints, ints[0])
    with pytest.raises(TypeError):
        mk.assign_pages(ints, ints[0], ints[0], ints[0], ints[0, :1], 16, 4)
    with pytest.raises(ValueError):
        mk.kv_cache8(3, 2, 24, 64, device="cpu")


def test_fake_implementations():
    def meta(*shape, dtype=torch.float16):
        return torch.empty(*shape, dtype=dtype, device="meta")

    ops, i32 = torch.ops.marlin_mi355x, torch.int32
    k = meta(9, 2, 16, 64, dtype=E4M3)
    table, lengths, scales = meta(3, 4, dtype=i32), meta(3, dtype=i32), meta(9, 2, 2, 1, dtype=torch.float32)
    o, lse = ops.cache_attention(meta(5, 4, 64), k, k, table, lengths, scales, meta(4, dtype=i32), 7, 1)
    assert o.shape == (5, 4, 64) and lse.shape == (5, 4) and lse.dtype == torch.float32
    assert ops.kv_append8(meta(3, 4, 64), meta(3, 2, 64), meta(3, 2, 64), k, meta(9, 2, 16, 64, dtype=E4M3), scales, table, lengths).shape == (3, 4, 64)
    starts, slots = ops.assign_pages(table, lengths, meta(3, dtype=i32), meta(9, dtype=i32), meta(1, dtype=i32), 16, 11)
    assert starts.shape == (4,) and starts.dtype == i32 and slots.shape == (11,) and slots.dtype == torch.int64
    with pytest.raises(TypeError):
        ops.cache_attention(meta(5, 4, 64, dtype=torch.float32), k, k, table, lengths)


# ---- the plain forms ----

def small(seed, bits=16, several=True):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(9, 4, 8, generator=g).half()
    k, v = (torch.randn(6, 2, 16, 8, generator=g).half() for _ in range(2))
    scales = None
    if bits == 8:
        k, v = ((x * 50).to(E4M3) for x in (k, v))
        scales = 2.0 ** torch.randint(-8, 2, (6, 2, 2, 1), generator=g).float()
    table = torch.tensor([[3, 0], [5, 1], [2, 4]], dtype=torch.int32)
    return dict(q=q, k_cache=k, v_cache=v, table=table, lengths=torch.tensor([20, 3, 31], dtype=torch.int32), scales=scales,
                starts=torch.tensor([0, 4, 5, 9], dtype=torch.int32))


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("window,sinks", [(None, 0), (5, 0), (7, 2), (1, 30)])
def test_attention_reference_token_by_token(bits, window, sinks):
    """Each token alone, its keys copied out as a dense softmax of the torch library in 64 bits."""
    a = small(1, bits)
    out, lse, tol, _, _ = ref.attention(**a, window=window, sinks=sinks)
    for b in range(3):
        for i in range(int(a["starts"][b]), int(a["starts"][b + 1])):
            pos = int(a["lengths"][b]) - int(a["starts"][b + 1]) + i
            j = [x for x in range(pos + 1) if not window or x > pos - window or x < sinks]
            for h in range(4):
                K, V = (torch.stack([x[a["table"][b, y // 16], h // 2, y % 16].float().double() *
                                     (1 if bits == 16 else a["scales"][a["table"][b, y // 16], h // 2, which, 0].double()) for y in j])
                        for which, x in enumerate((a["k_cache"], a["v_cache"])))
                s = K @ a["q"][i, h].double() * 8 ** -0.5
                torch.testing.assert_close(out[i, h], torch.softmax(s, 0) @ V, rtol=1e-12, atol=1e-12)
                torch.testing.assert_close(lse[i, h], torch.logsumexp(s, 0), rtol=1e-12, atol=1e-12)
    assert (tol > 0).all()


def test_attention_reference_is_kv_references_for_one_token():
    a = small(2)
    a["q"], a["starts"] = a["q"][:3], None
    got = ref.attention(**a)
    want = kv_reference.attention(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lengths"])
    torch.testing.assert_close(got[0], want[0], rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(got[1], want[1], rtol=1e-12, atol=1e-12)


def test_nearest_is_the_types_conversion():
    """Every float16, and points around every border between codes, against the library's conversion."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.float16).float()
    x = x[torch.isfinite(x)].clamp(-448, 448)
    assert torch.equal(ref.nearest(x.double()), x.to(E4M3).view(torch.uint8))
    grid = torch.arange(127, dtype=torch.uint8).view(E4M3).float().double()
    border = (grid[1:] + grid[:-1]) / 2
    x = torch.cat([border, border * (1 + 2.0 ** -20), border * (1 - 2.0 ** -20)]).float()
    assert torch.equal(ref.nearest(x.double()), x.to(E4M3).view(torch.uint8))


def test_scale_is_the_least():
    for a in (0.0, 2.0 ** -60, 1e-9, 0.3, 1.75, 1.7500001, 447.9, 448.0, 448.1, 65504.0, 3e38):
        s = ref.scale_of(a)
        assert math.log2(s) == round(math.log2(s)) and -40 <= math.log2(s) <= 40
        assert a <= 448 * s or s == 2.0 ** 40
        assert s == 2.0 ** -40 or a > 448 * s / 2


def test_append_reference_keeps_what_it_should():
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(30, 2, 32, generator=g).half() for _ in range(2))
    kc, vc = (torch.randint(0, 126, (5, 2, 32, 32), generator=g, dtype=torch.uint8).view(E4M3) for _ in range(2))
    scales = torch.ones(5, 2, 2, 2)
    table, lengths = torch.tensor([[4, 1]], dtype=torch.int32), torch.tensor([41], dtype=torch.int32)
    a, b, s = ref.append8(k, v, kc, vc, scales, table, lengths, starts=[0, 30])
    touched = [(4, i) for i in range(11, 32)] + [(1, i) for i in range(9)]
    for x, codes, which in ((k, a, 0), (v, b, 1)):
        for n, (page, slot) in enumerate(touched):  # each within half a step, of four bits or of the least one
            got = codes[page, :, slot].view(E4M3).float() * s[page, :, which, slot // 16][:, None]
            off = (got - x[n].float()).abs()
            assert (off <= torch.maximum(2.0 ** -4 * x[n].float().abs(), 2.0 ** -10 * s[page, :, which, slot // 16][:, None])).all()
        rest = torch.ones(5, 32, dtype=torch.bool)
        for page, slot in touched:
            rest[page, slot] = False
        rest[4, :11] = False  # older tokens of the first block
        old = (kc if which == 0 else vc).view(torch.uint8)
        assert torch.equal(codes.permute(0, 2, 1, 3)[rest], old.permute(0, 2, 1, 3)[rest])
    assert (s[[0, 2, 3]] == 1).all() and (s[4, :, :, 0] == 1).all() and (s[4, :, :, 1] < 1).all()


def invariants(before, after, page_size, tokens):
    """What a step's tables have to be, whoever made them."""
    table0, lengths0, free0, count0, new = before
    table, lengths, free, count, starts, slots = after
    pages = len(free0)
    given = starts[1:] - starts[:-1]
    assert starts[0] == 0 and (given >= 0).all() and starts[-1] <= tokens
    for b in range(len(lengths0)):
        assert given[b] in (0, max(0, int(new[b])))
        assert lengths[b] == (0 if new[b] < 0 else lengths0[b] + given[b])
    now = torch.cat([table[table >= 0], free[:count]])
    then = torch.cat([table0[table0 >= 0], free0[:count0]])
    assert torch.equal(now.sort().values, then.sort().values) and len(now.unique()) == len(now) <= pages
    used = slots[slots >= 0]
    assert len(used.unique()) == len(used) and (slots[int(starts[-1]):] == -1).all()


def state(rng, B, ps=16):
    lengths = [rng.randrange(0, 100) for _ in range(B)]
    used = [-(-n // ps) for n in lengths]
    spare = rng.randrange(0, 4 * B)
    perm = list(range(sum(used) + spare))
    rng.shuffle(perm)
    table = torch.full((B, max(used) + rng.randrange(1, 4)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = torch.tensor(perm[at:at + n], dtype=torch.int32)
        at += n
    free = torch.full((len(perm) or 1,), -1, dtype=torch.int32)
    free[:spare] = torch.tensor(perm[at:], dtype=torch.int32)
    new = [rng.choice([-1, 0, 1, 1, 1, 5, 40]) for _ in range(B)]
    return table, torch.tensor(lengths, dtype=torch.int32), torch.tensor(new, dtype=torch.int32), free, spare


def test_pages_reference_holds_the_invariants():
    rng = random.Random(1)
    for _ in range(300):
        table, lengths, new, free, count = state(rng, rng.randrange(1, 9))
        tokens, window = rng.choice([0, 5, 60, 1000]), rng.choice([None, None, 1, 16, 40])
        after = ref.assign_pages(table, lengths, new, free, count, 16, tokens, window, rng.choice([0, 1, 20]))
        invariants((table, lengths, free, count, new), after, 16, tokens)


MISTAKES = [
    ("free[room]", "free[room - 1]", ref.assign_pages),                       # a page is taken twice
    ("table[b, i] = -1", "pass", ref.assign_pages),                           # a page that was given back is kept
    ("starts[-1] + n <= tokens", "True", ref.assign_pages),                   # more tokens than rows
    ("lengths[b] = 0", "pass", ref.assign_pages),                             # an ended sequence lives on
    ("had[b] + n <= cap", "True", ref.assign_pages),                          # past the row
    ("j <= pos", "j < pos", ref.attention),                                   # a token does not see itself
    ("j > pos - window", "j >= pos - window", ref.attention),                 # a window of one more
    ("j < sinks", "j <= sinks", ref.attention),                               # a sink of one more
    ("max(0, int(lengths[b])) - n", "0", ref.attention),                      # positions from zero
    ("2.0 ** 40)).all(2)", "2.0 ** 40)).any(2)", ref.held),                   # one good scale is enough
]


@pytest.mark.parametrize("good,bad,function", MISTAKES, ids=[m[1] for m in MISTAKES])
def test_planted_mistakes_are_found(good, bad, function):
    source = inspect.getsource(function)
    assert good in source
    space = dict(vars(ref))
    exec(source.replace(good, bad), space)
    wrong = space[function.__name__]
    if function is ref.assign_pages:
        rng = random.Random(2)
        with pytest.raises((AssertionError, IndexError)):
            for _ in range(300):
                table, lengths, new, free, count = state(rng, rng.randrange(2, 9))
                tokens = rng.choice([30, 500])
                after = wrong(table, lengths, new, free, count, 16, tokens, None, 0)
                invariants((table, lengths, free, count, new), after, 16, tokens)
        return
    a = small(3, bits=8)
    a["scales"][0, :, 1] = 0  # a block whose values have no scale
    if function is ref.held:
        space["held"] = wrong
        exec(inspect.getsource(ref.attention), space)
        wrong = space["attention"]
    want, _, tol, _, _ = ref.attention(**a, window=9, sinks=3)
    got = wrong(**a, window=9, sinks=3)[0]
    assert ((got - want).abs() > tol).any()

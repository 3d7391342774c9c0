"""The paged key-value cache's entry points without a GPU: the argument structs
of marlin.h against the binding's, every refusal that the host makes before
any HIP call, the native call module, the PyTorch operators' fake
implementations, and the 64-bit forms the GPU tests compare with against
differences and a second way."""
import ctypes
import math
import os
import re

import pytest

torch = pytest.importorskip("torch")

import kv_reference as ref  # noqa: E402
import paper_2408_11743_amd as mk  # noqa: E402
from paper_2408_11743_amd import _binding as B  # noqa: E402
from paper_2408_11743_amd import kv  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULLP, SHAPE, ALIGN, WS, ARG = 0, 1, 2, 4, 5, 8
FAKE = 0x10000  # aligned, never dereferenced: every call below fails validation first


def struct_fields(name):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "marlin.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, text).group(1)
    fields = []
    for line in body.split(";"):
        line = line.strip()
        if line:
            assert re.match(r"(const )?(void|float|int32_t) \*|(u?int64_t|double) ", line), line  # 8 bytes each
            names = re.sub(r"^(const )?\w+ ", "", line)
            fields += [n.strip(" *") for n in names.split(",")]
    return fields


@pytest.mark.parametrize("name,fields,pack", [
    ("marlin_kv_append_args", B.KV_APPEND_FIELDS, B.pack_kv_append),
    ("marlin_paged_attention_args", B.PAGED_ATTENTION_FIELDS, B.pack_paged_attention),
    ("marlin_select_pages_args", B.SELECT_PAGES_FIELDS, B.pack_select_pages)])
def test_structs_are_the_bindings(name, fields, pack):
    assert struct_fields(name) == fields
    packed = pack(*range(len(fields)))
    assert len(packed) == 8 * len(fields)
    if "scale" in fields:
        i = fields.index("scale")
        assert ctypes.c_double.from_buffer_copy(packed, 8 * i).value == i


APPEND = dict(q=FAKE, k=FAKE, v=FAKE, q_row=1024, q_head=128, k_row=1024, k_head=128, v_row=1024, v_head=128, q_out=FAKE,
              k_cache=FAKE, v_cache=FAKE, bounds=None, cos_sin=FAKE, positions=4096, rot=128, interleaved=0, table=FAKE,
              table_row=8, lengths=FAKE, starts=None, tokens=3, B=3, heads=8, kv_heads=2, head_dim=128, pages=100,
              page_size=16, width=8, dtype=0)
ATTEND = dict(q=FAKE, q_row=1024, q_head=128, k_cache=FAKE, v_cache=FAKE, table=FAKE, table_row=8, table_head=0,
              lengths=FAKE, out=FAKE, lse=None, workspace=FAKE, workspace_bytes=1 << 40, B=3, heads=8, kv_heads=2,
              head_dim=128, pages=100, page_size=16, width=8, scale=0.1, dtype=0)
SELECT = dict(q=FAKE, q_row=1024, q_head=128, bounds=FAKE, table=FAKE, table_row=8, lengths=FAKE, chosen=FAKE,
              chosen_lengths=FAKE, workspace=FAKE, workspace_bytes=1 << 40, B=3, heads=8, kv_heads=2, head_dim=128,
              pages=100, page_size=16, width=8, select=4, dtype=0)
CALLS = {"append": (mk.marlin_kv_append, APPEND), "attend": (mk.marlin_paged_attention, ATTEND),
         "select": (mk.marlin_select_pages, SELECT)}


def status(which, **change):
    call, args = CALLS[which]
    try:
        call(**{**args, **change})
    except B.MarlinError as e:
        return e.status
    return OK


@pytest.mark.parametrize("which", list(CALLS))
def test_shared_refusals(which):
    for change in (dict(B=-1), dict(B=(1 << 16) + 1), dict(heads=7), dict(kv_heads=0), dict(heads=1), dict(kv_heads=3),
                   dict(heads=2048, kv_heads=2), dict(head_dim=80), dict(head_dim=0), dict(head_dim=512),
                   dict(pages=0), dict(pages=1 << 31), dict(page_size=8), dict(page_size=24), dict(page_size=2048),
                   dict(page_size=0), dict(page_size=-16), dict(width=0), dict(width=(1 << 26) + 1), dict(q_row=4),
                   dict(q_head=129), dict(q_row=-8), dict(table_row=-1)):
        assert status(which, **change) == SHAPE, change
    for name in ("q", "table", "lengths"):
        assert status(which, **{name: None}) == NULLP, name
    assert status(which, q=FAKE + 8) == ALIGN
    for name in ("table", "lengths"):
        assert status(which, **{name: FAKE + 2}) == ALIGN, name
    assert status(which, dtype=2) == ARG and status(which, dtype=-1) == ARG
    # no sequences: nothing is looked at
    assert status(which, B=0, q=None, table=None, **(dict(tokens=0) if which == "append" else {})) == OK


def test_append_refusals():
    for name in ("k", "v", "q_out", "k_cache", "v_cache", "cos_sin"):
        assert status("append", **{name: None}) == NULLP, name
        assert status("append", **{name: FAKE + 4}) == ALIGN, name
    assert status("append", bounds=FAKE + 8) == ALIGN and status("append", starts=FAKE + 1) == ALIGN
    for change in (dict(rot=8), dict(rot=-16), dict(rot=144), dict(interleaved=2), dict(interleaved=-1)):
        assert status("append", **change) == ARG, change
    for change in (dict(tokens=2), dict(tokens=-1, starts=FAKE), dict(tokens=(1 << 24) + 1, starts=FAKE),
                   dict(positions=0), dict(k_row=12), dict(v_head=-8)):
        assert status("append", **change) == SHAPE, change
    assert status("append", tokens=0, starts=FAKE, q=None, k_cache=None) == OK


def test_attention_refusals():
    for name in ("k_cache", "v_cache", "out", "workspace"):
        assert status("attend", **{name: None}) == NULLP, name
        assert status("attend", **{name: FAKE + 8}) == ALIGN, name
    assert status("attend", lse=FAKE + 2) == ALIGN
    for scale in (math.nan, math.inf, -math.inf, 1e300, 3e38):
        assert status("attend", scale=scale) == ARG, scale
    assert status("attend", table_head=-1) == SHAPE
    assert status("attend", B=1 << 16, heads=64, kv_heads=64, width=1 << 16) == SHAPE  # too many steps to number
    need = mk.marlin_paged_attention_workspace_bytes(128)
    assert status("attend", workspace_bytes=need - 1) == WS and status("attend", workspace_bytes=0) == WS
    assert [mk.marlin_paged_attention_workspace_bytes(d) > 1 << 20 for d in (64, 96, 128, 256)] == [True] * 4
    assert [mk.marlin_paged_attention_workspace_bytes(d) for d in (0, 32, 80, 512, -64)] == [0] * 5


def test_select_refusals():
    for name in ("bounds", "chosen", "chosen_lengths", "workspace"):
        assert status("select", **{name: None}) == NULLP, name
        assert status("select", **{name: FAKE + 2}) == ALIGN, name
    for n in (0, -1, (1 << 20) + 1):
        assert status("select", select=n) == ARG, n
    need = mk.marlin_select_pages_workspace_bytes(3, 2, 8)
    assert need == (1 << 20) + 3 * 2 * 8 * 4
    assert status("select", workspace_bytes=need - 1) == WS
    assert status("select", B=1 << 16, width=1 << 20) == SHAPE
    for bad in ((-1, 2, 8), (3, 0, 8), (3, 2, 0), (1 << 16, 8, 1 << 20)):
        assert mk.marlin_select_pages_workspace_bytes(*bad) == 0, bad


def test_binding_names_every_field():
    args = dict(ATTEND)
    del args["lse"]
    with pytest.raises(TypeError, match="lse"):
        mk.marlin_paged_attention(**args)


def test_native_module_leaves_other_tensors_to_python():
    from paper_2408_11743_amd import _fast
    x = torch.zeros(2, 4, 64).half()
    cache = torch.zeros(3, 2, 16, 64).half()
    ints = torch.zeros(2, 2, dtype=torch.int32)
    assert _fast.kv_append(x, x[:, :2], x[:, :2], cache, cache, ints, ints[0], None, None, False, None, None) is None
    assert _fast.paged_attention(x, cache, cache, ints, ints[0], None, False, None, None) is None
    assert _fast.select_pages(x, torch.zeros(3, 2, 2, 64).half(), ints, ints[0], 16, 1, None) is None
    assert _fast.paged_attention(None, 1, "x", ints, ints[0], None, False, None, None) is None
    assert _fast.kv_append(x) is None


def test_cpu_tensors_are_refused():
    x = torch.zeros(2, 4, 64).half()
    k, v, bounds = kv.kv_cache(3, 2, 16, 64, device="cpu", bounds=True)
    assert k.shape == v.shape == (3, 2, 16, 64) and bounds.shape == (3, 2, 2, 64)
    table, lengths = torch.zeros(2, 2, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        mk.kv_append(x, x[:, :2], x[:, :2], k, v, table, lengths)
    with pytest.raises(TypeError):
        mk.paged_attention(x, k, v, table, lengths)
    with pytest.raises(TypeError):
        mk.select_pages(x, bounds, table, lengths, 16, 1)
    for bad in ((0, 2, 16, 64), (3, 2, 24, 64), (3, 2, 8, 64), (3, 2, 16, 80)):
        with pytest.raises(ValueError):
            kv.kv_cache(*bad, device="cpu")
    with pytest.raises(TypeError):
        kv.kv_cache(3, 2, 16, 64, dtype=torch.float32, device="cpu")


def test_rotation_table():
    t = mk.rotation_table(5, 8, base=100.0, device="cpu")
    assert t.dtype == torch.float32 and t.shape == (5, 8)
    for j in range(5):
        for i in range(4):
            a = j * 100.0 ** (-2 * i / 8)
            assert abs(float(t[j, i]) - math.cos(a)) < 1e-7 and abs(float(t[j, 4 + i]) - math.sin(a)) < 1e-7


def test_rotation_table_refusals():
    for positions, rot in ((5, 7), (5, -2), (-1, 8)):
        with pytest.raises(ValueError):
            mk.rotation_table(positions, rot, device="cpu")
    assert mk.rotation_table(0, 8, device="cpu").shape == (0, 8) and mk.rotation_table(3, 0, device="cpu").shape == (3, 0)


def test_operators_are_registered_with_shapes():
    def meta(*shape, dtype=torch.float16):
        return torch.empty(*shape, dtype=dtype, device="meta")
    q, kc = meta(3, 8, 64), meta(9, 2, 16, 64)
    table, lengths = meta(3, 4, dtype=torch.int32), meta(3, dtype=torch.int32)
    ns = torch.ops.marlin_mi355x
    for bounds in (None, meta(9, 2, 2, 64)):
        assert ns.kv_append(q, meta(3, 2, 64), meta(3, 2, 64), kc, kc.clone(), bounds, table, lengths).shape == q.shape
    o, lse = ns.paged_attention(q, kc, kc, table, lengths)
    assert o.shape == q.shape and o.dtype == torch.float16 and lse.shape == (3, 8) and lse.dtype == torch.float32
    pages, tokens = ns.select_pages(q, meta(9, 2, 2, 64), table, lengths, 16, 5)
    assert pages.shape == (3, 2, 5) and pages.dtype == torch.int32 and tokens.shape == (3,)
    with pytest.raises(TypeError):
        ns.paged_attention(q.float(), kc, kc, table, lengths)
    schema = str(ns.kv_append.default._schema)
    assert "!) k_cache" in schema and "!) v_cache" in schema and "bounds" in schema


# ---- the 64-bit forms ----

def test_reference_attention_is_softmax():
    g = torch.Generator().manual_seed(1)
    k, v = torch.randn(2, 4, 1, 16, 64, generator=g).half()
    q = torch.randn(1, 2, 64, generator=g).half()
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32)
    out, lse, tol, tol_lse = ref.attention(q, k, v, table, torch.tensor([37]))
    keys = torch.cat([k[2, 0], k[0, 0], k[3, 0]])[:37].double()
    values = torch.cat([v[2, 0], v[0, 0], v[3, 0]])[:37].double()
    for h in range(2):
        s = keys @ q[0, h].double() / 8
        assert torch.allclose(out[0, h], torch.softmax(s, 0) @ values, atol=1e-12)
        assert abs(float(lse[0, h] - torch.logsumexp(s, 0))) < 1e-12
    # a mistake of one position, of one page or of the scale is far outside the bounds
    for wrong in (ref.attention(q, k, v, table, torch.tensor([36])), ref.attention(q, k, v, table, torch.tensor([37]), 0.126),
                  ref.attention(q, k, v, torch.tensor([[2, 3, 0]], dtype=torch.int32), torch.tensor([37]))):
        assert ((wrong[0] - out).abs() > tol).any()


def test_reference_rotation_is_a_rotation():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(3, 64, generator=g).double()
    angles = mk.rotation_table(9, 32, device="cpu")[7].double()
    for interleaved in (False, True):
        y, _ = ref.rotate(x, angles, 32, interleaved)
        assert torch.allclose(y.norm(dim=1), x.norm(dim=1), atol=1e-5)
        assert torch.equal(y[:, 32:], x[:, 32:]) and not torch.allclose(y[:, :32], x[:, :32])
        back = angles.clone()
        back[16:] *= -1
        z, _ = ref.rotate(y, back, 32, interleaved)
        assert torch.allclose(z, x, atol=1e-5)


def test_reference_order_of_16_bit_floats():
    for dtype in (torch.float16, torch.bfloat16):
        x = torch.tensor([-math.nan, -math.inf, -1.0, -0.0, 0.0, 1e-7, 1.0, math.inf, math.nan]).to(dtype)
        x.view(torch.int16)[0] |= -0x8000  # the sign a cast gives to a NaN is its own affair
        x.view(torch.int16)[8] &= 0x7FFF
        assert (ref.order(x).diff() > 0).all()


def test_reference_selection():
    q = torch.tensor([[[1.0, -1.0]]])
    lo, hi = torch.tensor([[-1.0, 0], [0, -2], [0, 0], [-1, 0], [9, 9]]), torch.tensor([[1.0, 1], [0, 0], [3, 5], [1, 1], [9, 9]])
    bounds = torch.stack([lo, hi], 1)[:, None]
    table = torch.tensor([[0, 1, 2, 3, 4]], dtype=torch.int32)
    # scores 1, 2, 3, 1 and the last page
    assert ref.select(q, bounds, table, torch.tensor([16 * 4 + 3]), 16, 3)[0].flatten().tolist() == [1, 2, 4]
    assert ref.select(q, bounds, table, torch.tensor([16 * 4 + 3]), 16, 4)[0].flatten().tolist() == [0, 1, 2, 4]
    assert ref.select(q, bounds, table, torch.tensor([16 * 4 + 3]), 16, 3)[1].tolist() == [35]

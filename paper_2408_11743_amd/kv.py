"""Tensor helpers of the paged key-value cache: what a served layer runs between
its 4-bit projections.

A cache is a pair of tensors [pages, kv heads, page size, head dim] in float16 or
bfloat16 (``kv_cache`` makes them), and for each sequence a row of pages in an
int32 table; which pages are free is the caller's to know.  A decode step of one
layer is

    q = kv_append(q, k, v, k_cache, v_cache, table, lengths, cos_sin)
    o = paged_attention(q, k_cache, v_cache, table, lengths)

with ``lengths`` the sequences' tokens, the new ones included.  With the pages'
bounds kept (``kv_append(..., bounds=bounds)``) a long context can be read through its
most promising pages alone:

    pages, tokens = select_pages(q, bounds, table, lengths, page_size, 64)
    o = paged_attention(q, k_cache, v_cache, pages, tokens)

As in ``ops``, these functions check their arguments, allocate outputs and call the
C entry points on the current stream.  They read no tensor on the host, so a
step can be captured into a HIP graph (one eager call on the capturing stream first, which
makes the workspace).  There is no autograd formula (inference only): where a gradient is
asked for, or a dispatch mode, trace or transform is to see the call, it becomes that of the
operator registered in ``torch_op``, whose backward raises (it uses the stream's own
workspace, not one that is passed), and a tangent raises here.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import _binding as B
from . import ops

_DTYPE = {torch.float16: 0, torch.bfloat16: 1}
_raw_stream = torch._C._cuda_getCurrentRawStream


def kv_cache(pages: int, kv_heads: int, page_size: int, head_dim: int, dtype=torch.float16, device="cuda",
             bounds: bool = False):
    """(k_cache, v_cache), and with ``bounds=True`` the pages' bounds [pages, kv
    heads, 2, head dim] for ``select_pages``; zero-filled."""
    shape = (int(pages), int(kv_heads), int(page_size), int(head_dim))
    if dtype not in _DTYPE:
        raise TypeError("kv_cache: dtype must be float16 or bfloat16")
    if (min(shape) < 1 or shape[3] not in (64, 96, 128, 256) or shape[2] & (shape[2] - 1)
            or not 16 <= shape[2] <= 1024):
        raise ValueError("kv_cache: page_size must be a power of two from 16 to 1024, head_dim 64, 96, 128 or 256")
    k, v = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
    if not bounds:
        return k, v
    return k, v, torch.zeros((shape[0], shape[1], 2, shape[3]), dtype=dtype, device=device)


def rotation_table(positions: int, rot: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """float32 [positions, rot]: row j holds cos(j f_i), then sin(j f_i), f_i =
    base^(-2i / rot), the table ``kv_append`` rotates by (computed in 64 bits)."""
    if rot < 0 or rot % 2 or positions < 0:
        raise ValueError("rotation_table: rot must be even, and neither it nor positions negative")
    f = float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _need(ok: bool, func: str, what: str) -> None:
    if not ok:
        raise ValueError("%s: %s" % (func, what))


# A decode step waits for the host between these small launches, so a call is
# first handed to a native module (csrc/fast.cpp), which does it where the tensors are as
# they nearly always are.  Anything else comes back as None, with nothing done,
# to the checks below, which name what is wrong or copy a view that the kernels
# cannot read; a HIP error raises there and then.  A token of 32 + 16 heads appended: 11.4 us a call in Python.
_native = None


def _connect():
    """The native module, connected to the library's entry points; raises if either has not been built."""
    global _native
    handle = B.lib()
    try:
        from . import _fast
    except ImportError as e:
        raise RuntimeError("the native call module is missing: build it with `python -m paper_2408_11743_amd.build`") from e
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
    _fast.connect(address(handle.marlin_kv_append), address(handle.marlin_paged_attention),
                  address(handle.marlin_select_pages), _raw_stream, ops._default_ws, B.MarlinError)
    _native = _fast
    return _fast


_dispatch_modes = torch._C._len_torch_dispatch_stack
_transforms, _tracing = torch._C._functorch.peek_interpreter_stack, torch._C._get_tracing_state
_forward_ad = torch.autograd.forward_ad


def _watched(*args) -> bool:
    """Something beside the kernels is to see a call with these arguments (see the module's docstring)."""
    tensors = [x for x in args if isinstance(x, torch.Tensor)]
    return (_dispatch_modes() > 0 or _transforms() is not None or _tracing() is not None
            or any(type(x) not in (torch.Tensor, torch.nn.Parameter) for x in tensors)
            or (torch.is_grad_enabled() and any(x.requires_grad for x in tensors)))


def _no_tangents(func: str, *tensors) -> None:
    if _forward_ad._current_level >= 0:
        for x in tensors:
            if isinstance(x, torch.Tensor) and _forward_ad.unpack_dual(x).tangent is not None:
                raise RuntimeError("%s: there is no forward derivative" % func)


def _rows(func: str, name: str, x: torch.Tensor, dtype, device, kind: str = "of the cache's dtype") -> torch.Tensor:
    """x [rows, heads, head dim] as the kernels read it: channels contiguous, rows
    and heads at multiples of 16 bytes (any other view is copied)."""
    if x.dtype != dtype or not x.is_cuda:
        raise TypeError("%s: %s must be a device tensor %s" % (func, name, kind))
    _need(x.dim() == 3, func, "%s must be [tokens, heads, head_dim]" % name)
    _need(x.device == device, func, "all tensors must be on one device")
    if x.is_neg():
        x = x.resolve_neg()
    s = x.stride()
    if s[2] != 1 or (s[0] | s[1]) & 7 or x.data_ptr() & 15:
        x = x.contiguous()
        if x.data_ptr() & 15 or x.stride(0) & 7 or x.stride(1) & 7:  # a dense view at an odd address or of one row
            x = x.clone(memory_format=torch.contiguous_format)
    return x


def _check_caches(func: str, k_cache: torch.Tensor, v_cache: torch.Tensor) -> None:
    if k_cache.dtype not in _DTYPE or v_cache.dtype != k_cache.dtype or not k_cache.is_cuda:
        raise TypeError("%s: the caches must be float16 or bfloat16 device tensors of one dtype" % func)
    _need(k_cache.dim() == 4 and v_cache.shape == k_cache.shape and k_cache.is_contiguous() and v_cache.is_contiguous(),
          func, "the caches must be contiguous [pages, kv_heads, page_size, head_dim]")
    _need(v_cache.device == k_cache.device, func, "all tensors must be on one device")
    _need(not (k_cache.is_neg() or v_cache.is_neg()), func, "the caches must not be lazily negated views")


def _check_ints(func: str, name: str, x: torch.Tensor, dims: int, device) -> None:
    if x.dtype != torch.int32 or not x.is_cuda:
        raise TypeError("%s: %s must be an int32 device tensor" % (func, name))
    _need(x.dim() == dims and (x.stride(-1) == 1 or x.shape[-1] <= 1), func,
          "%s must have %d dimensions, the last one contiguous" % (name, dims))
    _need(x.device == device, func, "all tensors must be on one device")


def _check_out(func: str, out: torch.Tensor, shape, dtype, device) -> None:
    _need(out.shape == shape and out.dtype == dtype and out.device == device and out.is_contiguous()
          and not out.is_neg(), func, "out must be a contiguous tensor of q's shape, dtype and device")


def _into(func: str, out, result: torch.Tensor, starts: torch.Tensor | None = None) -> torch.Tensor:
    """A registered operator's result, in the caller's tensor if there is one: with starts, the rows that belong to sequences."""
    if out is None:
        return result
    _check_out(func, out, result.shape, result.dtype, result.device)
    if starts is not None:
        row = torch.arange(result.shape[0], dtype=starts.dtype, device=starts.device)
        mine = (row >= starts[0]) & (row < starts[-1])
        result = torch.where(mine[:, None, None], result, out)
    return out.copy_(result)


_empty_like, _contiguous = torch.empty_like, torch.contiguous_format


def _workspace(func: str, index: int, stream: int, workspace, nbytes: int) -> torch.Tensor:
    """The caller's workspace, or the one ``ops.gemm`` uses on this device and stream, of nbytes at least."""
    if workspace is None:
        workspace = ops._default_ws.get((index, stream))
        if workspace is None:
            workspace = ops._default_ws.setdefault((index, stream), ops.Workspace("cuda:%d" % index))
    buf = workspace.buf
    _need(buf.is_cuda and buf.device.index == index and buf.is_contiguous(), func, "the workspace must be on the device of the tensors")
    return buf if buf.numel() >= nbytes else workspace.ensure(nbytes)


def kv_append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
              table: torch.Tensor, lengths: torch.Tensor, cos_sin: torch.Tensor | None = None,
              starts: torch.Tensor | None = None, interleaved: bool = False, bounds: torch.Tensor | None = None,
              out: torch.Tensor | None = None) -> torch.Tensor:
    """Rotates the new tokens' queries and keys and puts keys and values into their
    pages (``marlin_kv_append``); returns the rotated queries.

    q [tokens, heads, head dim], k and v [tokens, kv heads, head dim] may be
    slices of one projection's rows.  One token per sequence, or with ``starts``
    int32 [sequences + 1] sequence b's rows are starts[b] .. starts[b + 1] - 1
    and its last one has position lengths[b] - 1.  ``cos_sin`` float32
    [positions, rot] (``rotation_table``) rotates the first rot channels, in
    halves or ``interleaved`` pairs; None rotates nothing.  ``bounds``: the pages' bounds,
    kept up to date."""
    done = (_native or _connect()).kv_append(q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, interleaved,
                                             bounds, out)
    if done is not None:
        return done
    if _watched(q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, bounds, out):
        y = torch.ops.marlin_mi355x.kv_append(q, k, v, k_cache, v_cache, bounds, table, lengths, cos_sin, starts,
                                              bool(interleaved))
        return _into("kv_append", out, y, starts)
    return _kv_append(q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, interleaved, bounds, out)


def _kv_append(q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, interleaved, bounds, out):
    """The call with its checks, which name what is wrong or copy a view that the kernels cannot read."""
    _no_tangents("kv_append", q, k, v, k_cache, v_cache, cos_sin, bounds)
    f, dtype, device = "kv_append", k_cache.dtype, k_cache.device
    _check_caches(f, k_cache, v_cache)
    q, k, v = (_rows(f, name, x, dtype, device) for name, x in (("q", q), ("k", k), ("v", v)))
    _check_ints(f, "table", table, 2, device)
    _check_ints(f, "lengths", lengths, 1, device)
    dev, qs, cs, ts = device.index, q.shape, k_cache.shape, table.shape
    _need(qs[2] == cs[3] and k.shape == (qs[0], cs[1], cs[3]) and v.shape == k.shape, f,
          "q, k and v must be [tokens, heads or kv_heads, %d]" % cs[3])
    _need(lengths.shape[0] == ts[0], f, "lengths must have one entry per row of table")
    pages, kv_heads, page_size, D = cs
    tokens, heads, _ = qs
    n, width = ts
    if starts is not None:
        _check_ints(f, "starts", starts, 1, device)
        _need(starts.shape[0] == n + 1, "kv_append", "starts must have one entry more than table has rows")
    elif tokens != n:
        raise ValueError("kv_append: without starts there is one token per row of table")
    positions = rot = 0
    if cos_sin is not None:
        if cos_sin.dtype is not torch.float32:
            raise TypeError("kv_append: cos_sin must be float32")
        shape = cos_sin.shape
        _need(len(shape) == 2 and cos_sin.is_contiguous() and cos_sin.device == device and not cos_sin.is_neg(),
              "kv_append", "cos_sin must be a contiguous [positions, rot] tensor on the cache's device")
        positions, rot = shape
    if bounds is not None:
        _need(bounds.dtype is dtype and bounds.shape == (pages, kv_heads, 2, D) and bounds.is_contiguous()
              and bounds.device == device and not bounds.is_neg(), "kv_append",
              "bounds must be a contiguous [pages, kv_heads, 2, head_dim] tensor of the cache's dtype and device")
    if out is None:
        out = _empty_like(q, memory_format=_contiguous)
    else:
        _check_out("kv_append", out, (tokens, heads, D), dtype, k_cache.device)
    qt, kt, vt, tt = q.stride(), k.stride(), v.stride(), table.stride()
    with torch.cuda.device(dev):
        status = B.lib().marlin_kv_append(B.pack_kv_append(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), qt[0], qt[1], kt[0], kt[1], vt[0], vt[1], out.data_ptr(),
            k_cache.data_ptr(), v_cache.data_ptr(), 0 if bounds is None else bounds.data_ptr(),
            cos_sin.data_ptr() if rot else 0, positions, rot, 1 if interleaved else 0, table.data_ptr(), tt[0],
            lengths.data_ptr(), 0 if starts is None else starts.data_ptr(), tokens, n, heads, kv_heads, D, pages,
            page_size, width, _DTYPE[dtype]), _raw_stream(dev))
    if status:
        raise B.MarlinError("marlin_kv_append", status)
    return out


def paged_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor,
                    lengths: torch.Tensor, scale: float | None = None, return_lse: bool = False,
                    out: torch.Tensor | None = None, workspace: "ops.Workspace | None" = None):
    """Attention of one token per sequence, q [sequences, heads, head dim], over
    the cache (``marlin_paged_attention``): out like q, dense, and with ``return_lse``
    (out, float32 [sequences, heads] logarithms of the softmax's sums).

    ``table`` [sequences, width], or [sequences, kv heads, width] where each kv
    head has pages of its own (``select_pages``); ``scale`` defaults to
    1 / sqrt(head dim).  A sequence without tokens gives 0 and -inf."""
    done = (_native or _connect()).paged_attention(q, k_cache, v_cache, table, lengths, scale, return_lse, out, workspace)
    if done is not None:
        return done
    if _watched(q, k_cache, v_cache, table, lengths, out):
        o, lse = torch.ops.marlin_mi355x.paged_attention(q, k_cache, v_cache, table, lengths, scale)
        o = _into("paged_attention", out, o)
        return (o, lse) if return_lse else o
    return _paged_attention(q, k_cache, v_cache, table, lengths, scale, return_lse, out, workspace)


def _paged_attention(q, k_cache, v_cache, table, lengths, scale, return_lse, out, workspace):
    _no_tangents("paged_attention", q, k_cache, v_cache)
    f, dtype, device = "paged_attention", k_cache.dtype, k_cache.device
    _check_caches(f, k_cache, v_cache)
    q = _rows(f, "q", q, dtype, device)
    per_head = table.dim() == 3
    _check_ints(f, "table", table, 3 if per_head else 2, device)
    _check_ints(f, "lengths", lengths, 1, device)
    dev, qs, cs, ts = device.index, q.shape, k_cache.shape, table.shape
    _need(qs[2] == cs[3], f, "q must be [sequences, heads, %d]" % cs[3])
    _need(ts[0] == qs[0] and lengths.shape[0] == qs[0] and (not per_head or ts[1] == cs[1]), f,
          "table must be [sequences, width] or [sequences, kv_heads, width] and lengths [sequences]")
    pages, kv_heads, page_size, D = cs
    n, heads, _ = qs
    if out is None:
        out = _empty_like(q, memory_format=_contiguous)
    else:
        _check_out("paged_attention", out, (n, heads, D), dtype, k_cache.device)
    lse = torch.empty((n, heads), dtype=torch.float32, device=k_cache.device) if return_lse else None
    stream = _raw_stream(dev)
    qt, tt = q.stride(), table.stride()
    ptrs = (q.data_ptr(), qt[0], qt[1], k_cache.data_ptr(), v_cache.data_ptr(), table.data_ptr(), tt[0],
            tt[1] if per_head else 0, lengths.data_ptr(), out.data_ptr(), 0 if lse is None else lse.data_ptr())
    sizes = (n, heads, kv_heads, D, pages, page_size, ts[-1], 1.0 / math.sqrt(D) if scale is None else scale,
             _DTYPE[dtype])
    for nbytes in (0, B.marlin_paged_attention_workspace_bytes(D)):  # grown if the call says WORKSPACE_TOO_SMALL
        buf = _workspace(f, dev, stream, workspace, nbytes)
        with torch.cuda.device(dev):
            status = B.lib().marlin_paged_attention(
                B.pack_paged_attention(*ptrs, buf.data_ptr(), buf.numel(), *sizes), stream)
        if status != 5:
            break
    if status:
        raise B.MarlinError("marlin_paged_attention", status)
    return (out, lse) if return_lse else out


def select_pages(q: torch.Tensor, bounds: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, page_size: int,
                 select: int, workspace: "ops.Workspace | None" = None):
    """The ``select`` pages of each sequence and kv head that by their bounds can hold
    the keys nearest the queries, the last page always among them
    (``marlin_select_pages``): (pages int32 [sequences, kv heads, select] in the
    order of their positions, tokens int32 [sequences]) for ``paged_attention``."""
    done = (_native or _connect()).select_pages(q, bounds, table, lengths, page_size, select, workspace)
    if done is not None:
        return done
    if _watched(q, bounds, table, lengths):
        return torch.ops.marlin_mi355x.select_pages(q, bounds, table, lengths, page_size, select)
    return _select_pages(q, bounds, table, lengths, page_size, select, workspace)


def _select_pages(q, bounds, table, lengths, page_size, select, workspace):
    f, dtype, device = "select_pages", bounds.dtype, bounds.device
    if dtype not in _DTYPE or not bounds.is_cuda:
        raise TypeError("select_pages: bounds must be a float16 or bfloat16 device tensor")
    _need(bounds.dim() == 4 and bounds.shape[2] == 2 and bounds.is_contiguous() and not bounds.is_neg(), f,
          "bounds must be a contiguous [pages, kv_heads, 2, head_dim] tensor")
    q = _rows(f, "q", q, dtype, device)
    _check_ints(f, "table", table, 2, device)
    _check_ints(f, "lengths", lengths, 1, device)
    dev, qs, bs, ts = device.index, q.shape, bounds.shape, table.shape
    _need(qs[2] == bs[3], f, "q must be [sequences, heads, %d]" % bs[3])
    _need(ts[0] == qs[0] and lengths.shape[0] == qs[0], f, "table and lengths must have one row per sequence")
    pages, kv_heads, _, D = bs
    n, heads, _ = qs
    width = ts[1]
    if not 1 <= select <= 1 << 20:
        raise B.MarlinError("marlin_select_pages", 8)
    chosen = torch.empty((n, kv_heads, select), dtype=torch.int32, device=table.device)
    tokens = torch.empty_like(lengths, memory_format=_contiguous)
    stream = _raw_stream(dev)
    qt, tt = q.stride(), table.stride()
    args = (q.data_ptr(), qt[0], qt[1], bounds.data_ptr(), table.data_ptr(), tt[0], lengths.data_ptr(), chosen.data_ptr(),
            tokens.data_ptr())
    sizes = (n, heads, kv_heads, D, pages, page_size, width, select, _DTYPE[dtype])
    for nbytes in (0, B.marlin_select_pages_workspace_bytes(n, kv_heads, width)):
        buf = _workspace(f, dev, stream, workspace, nbytes)
        with torch.cuda.device(dev):
            status = B.lib().marlin_select_pages(B.pack_select_pages(*args, buf.data_ptr(), buf.numel(), *sizes), stream)
        if status != 5:
            break
    if status:
        raise B.MarlinError("marlin_select_pages", status)
    return chosen, tokens

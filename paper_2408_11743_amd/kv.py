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
makes the workspace).  There is no autograd formula (inference only).
"""
from __future__ import annotations

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
    f = float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _need(ok: bool, func: str, what: str) -> None:
    if not ok:
        raise ValueError("%s: %s" % (func, what))


def _rows(func: str, name: str, x: torch.Tensor, dtype) -> torch.Tensor:
    """x [rows, heads, head dim] as the kernels read it: channels contiguous, rows
    and heads at multiples of 16 bytes (any other view is copied)."""
    if x.dtype != dtype or not x.is_cuda:
        raise TypeError("%s: %s must be a device tensor of the cache's dtype" % (func, name))
    if x.dim() != 3:
        raise ValueError("%s: %s must be [tokens, heads, head_dim]" % (func, name))
    if x.is_neg():
        x = x.resolve_neg()
    s = x.stride()
    if s[2] != 1 or (s[0] | s[1]) & 7 or x.data_ptr() & 15:
        x = x.contiguous()
        if x.data_ptr() & 15 or x.stride(0) & 7 or x.stride(1) & 7:  # a dense view at an odd address or of one row
            x = x.clone(memory_format=torch.contiguous_format)
    return x


def _caches(func: str, k_cache: torch.Tensor, v_cache: torch.Tensor) -> tuple:
    dtype = k_cache.dtype
    if dtype not in _DTYPE or v_cache.dtype != dtype or not k_cache.is_cuda:
        raise TypeError("%s: the caches must be float16 or bfloat16 device tensors of one dtype" % func)
    shape = k_cache.shape
    if len(shape) != 4 or v_cache.shape != shape or not k_cache.is_contiguous() or not v_cache.is_contiguous():
        raise ValueError("%s: the caches must be contiguous [pages, kv_heads, page_size, head_dim]" % func)
    if k_cache.is_neg() or v_cache.is_neg():
        raise ValueError("%s: the caches must not be lazily negated views" % func)
    return shape


def _ints(func: str, name: str, x: torch.Tensor, dims: int) -> None:
    if x.dtype != torch.int32 or not x.is_cuda:
        raise TypeError("%s: %s must be an int32 device tensor" % (func, name))
    if x.dim() != dims or (x.stride(-1) != 1 and x.shape[-1] > 1):
        raise ValueError("%s: %s must have %d dimensions, the last one contiguous" % (func, name, dims))


def _workspace(index: int, device, stream: int, workspace, nbytes: int):
    if workspace is None:
        workspace = ops._default_ws.get((index, stream))
        if workspace is None:
            workspace = ops._default_ws.setdefault((index, stream), ops.Workspace(device))
    buf = workspace.buf
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
    f = "kv_append"
    pages, kv_heads, page_size, D = _caches(f, k_cache, v_cache)
    dtype, device = k_cache.dtype, k_cache.device
    q, k, v = _rows(f, "q", q, dtype), _rows(f, "k", k, dtype), _rows(f, "v", v, dtype)
    _ints(f, "table", table, 2)
    _ints(f, "lengths", lengths, 1)
    n, width = table.shape
    tokens, heads = q.shape[0], q.shape[1]
    _need(q.shape[2] == D and k.shape == (tokens, kv_heads, D) and v.shape == k.shape, f,
          "q, k and v must be [tokens, heads or kv_heads, %d]" % D)
    _need(lengths.shape[0] == n, f, "lengths must have one entry per row of table")
    _need(q.device == device and k.device == device and v.device == device and table.device == device
          and lengths.device == device and v_cache.device == device, f, "all tensors must be on one device")
    if starts is not None:
        _ints(f, "starts", starts, 1)
        _need(starts.shape[0] == n + 1 and starts.device == device, f,
              "starts must have one entry more than table has rows, on its device")
    else:
        _need(tokens == n, f, "without starts there is one token per row of table")
    rot = positions = 0
    if cos_sin is not None:
        if cos_sin.dtype != torch.float32:
            raise TypeError("kv_append: cos_sin must be float32")
        _need(cos_sin.dim() == 2 and cos_sin.is_contiguous() and cos_sin.device == device and not cos_sin.is_neg(), f,
              "cos_sin must be a contiguous [positions, rot] tensor on the cache's device")
        positions, rot = cos_sin.shape
    if bounds is not None:
        _need(bounds.dtype == dtype and bounds.shape == (pages, kv_heads, 2, D) and bounds.is_contiguous()
              and bounds.device == device and not bounds.is_neg(), f,
              "bounds must be a contiguous [pages, kv_heads, 2, head_dim] tensor of the cache's dtype and device")
    if out is None:
        out = torch.empty((tokens, heads, D), dtype=dtype, device=device)
    else:
        _need(out.shape == (tokens, heads, D) and out.dtype == dtype and out.device == device and out.is_contiguous()
              and not out.is_neg(), f, "out must be a contiguous tensor of q's shape, dtype and device")
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    status = B.lib().marlin_kv_append(B.pack_kv_append(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], out.data_ptr(),
        k_cache.data_ptr(), v_cache.data_ptr(), 0 if bounds is None else bounds.data_ptr(),
        0 if rot == 0 else cos_sin.data_ptr(), positions, rot, 1 if interleaved else 0, table.data_ptr(),
        table.stride(0), lengths.data_ptr(), 0 if starts is None else starts.data_ptr(), tokens, n, heads, kv_heads, D,
        pages, page_size, width, _DTYPE[dtype]), _raw_stream(device.index))
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
    f = "paged_attention"
    pages, kv_heads, page_size, D = _caches(f, k_cache, v_cache)
    dtype, device = k_cache.dtype, k_cache.device
    q = _rows(f, "q", q, dtype)
    per_head = table.dim() == 3
    _ints(f, "table", table, 3 if per_head else 2)
    _ints(f, "lengths", lengths, 1)
    n, heads, d = q.shape
    _need(d == D, f, "q must be [sequences, heads, %d]" % D)
    _need(table.shape[0] == n and lengths.shape[0] == n and (not per_head or table.shape[1] == kv_heads), f,
          "table must be [sequences, width] or [sequences, kv_heads, width] and lengths [sequences]")
    _need(q.device == device and v_cache.device == device and table.device == device and lengths.device == device, f,
          "all tensors must be on one device")
    if out is None:
        out = torch.empty((n, heads, D), dtype=dtype, device=device)
    else:
        _need(out.shape == (n, heads, D) and out.dtype == dtype and out.device == device and out.is_contiguous()
              and not out.is_neg(), f, "out must be a contiguous tensor of q's shape, dtype and device")
    lse = torch.empty((n, heads), dtype=torch.float32, device=device) if return_lse else None
    index = device.index
    stream = _raw_stream(index)
    buf = _workspace(index, device, stream, workspace, B.marlin_paged_attention_workspace_bytes(D))
    qs, ts = q.stride(), table.stride()
    status = B.lib().marlin_paged_attention(B.pack_paged_attention(
        q.data_ptr(), qs[0], qs[1], k_cache.data_ptr(), v_cache.data_ptr(), table.data_ptr(), ts[0],
        ts[1] if per_head else 0, lengths.data_ptr(), out.data_ptr(), 0 if lse is None else lse.data_ptr(),
        buf.data_ptr(), buf.numel(), n, heads, kv_heads, D, pages, page_size, table.shape[-1],
        1.0 / math.sqrt(D) if scale is None else scale, _DTYPE[dtype]), stream)
    if status:
        raise B.MarlinError("marlin_paged_attention", status)
    return (out, lse) if return_lse else out


def select_pages(q: torch.Tensor, bounds: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, page_size: int,
                 select: int, workspace: "ops.Workspace | None" = None):
    """The ``select`` pages of each sequence and kv head that by their bounds can hold
    the keys nearest the queries, the last page always among them
    (``marlin_select_pages``): (pages int32 [sequences, kv heads, select] in the
    order of their positions, tokens int32 [sequences]) for ``paged_attention``."""
    f = "select_pages"
    dtype, device = bounds.dtype, bounds.device
    if dtype not in _DTYPE or not bounds.is_cuda:
        raise TypeError("select_pages: bounds must be a float16 or bfloat16 device tensor")
    _need(bounds.dim() == 4 and bounds.shape[2] == 2 and bounds.is_contiguous() and not bounds.is_neg(), f,
          "bounds must be a contiguous [pages, kv_heads, 2, head_dim] tensor")
    pages, kv_heads, _, D = bounds.shape
    q = _rows(f, "q", q, dtype)
    _ints(f, "table", table, 2)
    _ints(f, "lengths", lengths, 1)
    n, heads, d = q.shape
    _need(d == D, f, "q must be [sequences, heads, %d]" % D)
    _need(table.shape[0] == n and lengths.shape[0] == n, f, "table and lengths must have one row per sequence")
    _need(q.device == device and table.device == device and lengths.device == device, f,
          "all tensors must be on one device")
    if not 1 <= select <= 1 << 20:
        raise B.MarlinError("marlin_select_pages", 8)
    chosen = torch.empty((n, kv_heads, select), dtype=torch.int32, device=device)
    tokens = torch.empty(n, dtype=torch.int32, device=device)
    index = device.index
    stream = _raw_stream(index)
    width = table.shape[1]
    buf = _workspace(index, device, stream, workspace, B.marlin_select_pages_workspace_bytes(n, kv_heads, width))
    qs = q.stride()
    status = B.lib().marlin_select_pages(B.pack_select_pages(
        q.data_ptr(), qs[0], qs[1], bounds.data_ptr(), table.data_ptr(), table.stride(0), lengths.data_ptr(),
        chosen.data_ptr(), tokens.data_ptr(), buf.data_ptr(), buf.numel(), n, heads, kv_heads, D, pages, page_size,
        width, select, _DTYPE[dtype]), stream)
    if status:
        raise B.MarlinError("marlin_select_pages", status)
    return chosen, tokens

"""Tensor helpers of the 8-bit key-value cache, of attention with a window or of several new
tokens over a cache of 8 or 16 bits, and of the page tables that both go by.

An 8-bit cache (``kv_cache8``) is a pair of float8_e4m3fn tensors [pages, kv heads, page size, head dim] and
float32 scales [pages, kv heads, 2, page size // 16]: an element is its code times the scale of its kv head
and block of 16 slots, of keys (0) or of values (1).  A step of one layer, of which the lengths, tables and lists never leave
the device, is

    starts, slots = assign_pages(table, lengths, new, free, free_count, page_size, tokens)
    q = kv_append8(q, k, v, k_cache, v_cache, scales, table, lengths, cos_sin, starts)
    o = cache_attention(q, k_cache, v_cache, table, lengths, scales, starts)

``cache_attention`` takes the 16-bit caches of ``kv_cache`` as well (without scales), behind ``kv_append``.

Without ``starts`` every row of the table has one new token, row b of q, k and v, at position lengths[b] - 1: a sequence that
``assign_pages`` gave none (``new[b]`` of 0, or no pages left) keeps its length, and its row would be written over its last token.
Where that can be, a decode step takes lengths of 0 for those, which the calls without ``starts`` pass over:

    starts, slots = assign_pages(table, lengths, ones, free, free_count, page_size, len(table))
    now = torch.where(starts[1:] > starts[:-1], lengths, 0)
    q = kv_append8(q, k, v, k_cache, v_cache, scales, table, now, cos_sin)
    o = cache_attention(q, k_cache, v_cache, table, now, scales)

What ``kv``'s functions do about arguments, streams, workspaces, graphs, gradients, modes and transforms, these do too.
"""
from __future__ import annotations

import ctypes
import math
import operator

import torch

from . import _binding as B
from . import kv, ops
from .kv import _DTYPE, _check_ints, _check_out, _contiguous, _empty_like, _into, _need, _no_tangents, _raw_stream, _rows, _watched

_E4M3 = torch.float8_e4m3fn
BLOCK = 16  # slots that share a scale


def kv_cache8(pages: int, kv_heads: int, page_size: int, head_dim: int, device="cuda"):
    """(k_cache, v_cache, scales) of an 8-bit cache, zero-filled: blocks that nothing has been appended to count as masked."""
    k, v = kv.kv_cache(pages, kv_heads, page_size, head_dim, torch.float16, "meta")
    k, v = (torch.zeros(x.shape, dtype=torch.uint8, device=device).view(_E4M3) for x in (k, v))
    return k, v, torch.zeros((*k.shape[:2], 2, k.shape[2] // BLOCK), dtype=torch.float32, device=device)


# As in kv: the common case goes to a native module, which does it or says None with nothing done.
_native = None


def _connect():
    global _native
    fast, handle = kv._native or kv._connect(), B.lib()
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
    fast.connect_cache(address(handle.marlin_kv_append8), address(handle.marlin_cache_attention),
                       address(handle.marlin_assign_pages))
    _native = fast
    return fast


def _check_cache8(func: str, k_cache, v_cache, scales) -> None:
    if k_cache.dtype != _E4M3 or v_cache.dtype != _E4M3 or not k_cache.is_cuda:
        raise TypeError("%s: the caches must be float8_e4m3fn device tensors" % func)
    _check_shapes(func, k_cache, v_cache)
    if scales.dtype != torch.float32:
        raise TypeError("%s: scales must be float32" % func)
    pages, kv_heads, page_size, _ = k_cache.shape
    _need(scales.shape == (pages, kv_heads, 2, page_size // BLOCK) and scales.is_contiguous() and scales.device == k_cache.device
          and not scales.is_neg(), func,
          "scales must be a contiguous [pages, kv_heads, 2, page_size // 16] tensor on the caches' device")


def _check_shapes(func: str, k_cache, v_cache) -> None:
    _need(k_cache.dim() == 4 and v_cache.shape == k_cache.shape and k_cache.is_contiguous() and v_cache.is_contiguous(),
          func, "the caches must be contiguous [pages, kv_heads, page_size, head_dim]")
    _need(v_cache.device == k_cache.device, func, "all tensors must be on one device")
    _need(not (k_cache.is_neg() or v_cache.is_neg()), func, "the caches must not be lazily negated views")


def kv_append8(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
               scales: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor, cos_sin: torch.Tensor | None = None,
               starts: torch.Tensor | None = None, interleaved: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """``kv_append`` into an 8-bit cache (``marlin_kv_append8``): returns the rotated queries.

    A block of 16 slots takes the least power of two (2^-40 .. 2^40) that brings its new keys, or values, of a kv head to
    448 at the most, and no less than its scale so far; codes of earlier tokens are rounded anew where it
    grew.  Infinities and NaN become NaN and do not count for the scale."""
    done = (_native or _connect()).kv_append8(q, k, v, k_cache, v_cache, scales, table, lengths, cos_sin, starts, interleaved, out)
    if done is not None:
        return done
    if _watched(q, k, v, k_cache, v_cache, scales, table, lengths, cos_sin, starts, out):
        y = torch.ops.marlin_mi355x.kv_append8(q, k, v, k_cache, v_cache, scales, table, lengths, cos_sin, starts, bool(interleaved))
        return _into("kv_append8", out, y, starts)
    return _kv_append8(q, k, v, k_cache, v_cache, scales, table, lengths, cos_sin, starts, interleaved, out)


def _kv_append8(q, k, v, k_cache, v_cache, scales, table, lengths, cos_sin, starts, interleaved, out):
    f, dtype, device = "kv_append8", q.dtype, k_cache.device
    _no_tangents(f, q, k, v, cos_sin)
    if dtype not in _DTYPE:
        raise TypeError("kv_append8: q, k and v must be float16 or bfloat16")
    _check_cache8(f, k_cache, v_cache, scales)
    q, k, v = (_rows(f, name, x, dtype, device, "of q's dtype") for name, x in (("q", q), ("k", k), ("v", v)))
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
        _need(starts.shape[0] == n + 1, f, "starts must have one entry more than table has rows")
    elif tokens != n:
        raise ValueError("kv_append8: without starts there is one token per row of table")
    positions = rot = 0
    if cos_sin is not None:
        if cos_sin.dtype is not torch.float32:
            raise TypeError("kv_append8: cos_sin must be float32")
        _need(cos_sin.dim() == 2 and cos_sin.is_contiguous() and cos_sin.device == device and not cos_sin.is_neg(), f,
              "cos_sin must be a contiguous [positions, rot] tensor on the cache's device")
        positions, rot = cos_sin.shape
    if out is None:
        out = _empty_like(q, memory_format=_contiguous)
    else:
        _check_out(f, out, (tokens, heads, D), dtype, device)
    qt, kt, vt = q.stride(), k.stride(), v.stride()
    with torch.cuda.device(dev):
        status = B.lib().marlin_kv_append8(B.pack_kv_append8(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), qt[0], qt[1], kt[0], kt[1], vt[0], vt[1], out.data_ptr(),
            k_cache.data_ptr(), v_cache.data_ptr(), scales.data_ptr(), cos_sin.data_ptr() if rot else 0, positions, rot,
            1 if interleaved else 0, table.data_ptr(), table.stride(0), lengths.data_ptr(),
            0 if starts is None else starts.data_ptr(), tokens, n, heads, kv_heads, D, pages, page_size, width,
            _DTYPE[dtype]), _raw_stream(dev))
    if status:
        raise B.MarlinError("marlin_kv_append8", status)
    return out


def _visible(func: str, window, sinks) -> tuple[int, int]:
    sinks = operator.index(sinks)
    if window is None:
        return 0, sinks
    window = operator.index(window)
    _need(window >= 1, func, "window must be None or at least 1")
    return window, sinks


def cache_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, table: torch.Tensor, lengths: torch.Tensor,
                    scales: torch.Tensor | None = None, starts: torch.Tensor | None = None, window: int | None = None,
                    sinks: int = 0, scale: float | None = None, return_lse: bool = False, out: torch.Tensor | None = None,
                    workspace: "ops.Workspace | None" = None):
    """Attention of new tokens, q [tokens, heads, head dim], over the cache (``marlin_cache_attention``): out like q, dense,
    and with ``return_lse`` (out, float32 [tokens, heads] logarithms of the softmax's sums).

    One token per sequence, or with ``starts`` int32 [sequences + 1] sequence b's rows are starts[b] .. starts[b + 1] - 1; the last
    has position lengths[b] - 1.  A token at position p attends to the positions up to p, with ``window`` to the last
    ``window`` of them and to the first ``sinks`` positions.  ``scales``: of an 8-bit cache.  ``table`` is [sequences, width] or,
    without starts, [sequences, kv heads, width].  ``scale`` defaults to 1 / sqrt(head dim).
    A token that sees nothing gives 0 and -inf; rows that belong to no sequence are left as they are (unset
    in a new ``out``)."""
    done = (_native or _connect()).cache_attention(q, k_cache, v_cache, table, lengths, scales, starts, window, sinks, scale, return_lse,
                                                   out, workspace)
    if done is not None:
        return done
    if _watched(q, k_cache, v_cache, table, lengths, scales, starts, out):
        window, sinks = _visible("cache_attention", window, sinks)
        o, lse = torch.ops.marlin_mi355x.cache_attention(q, k_cache, v_cache, table, lengths, scales, starts, window, sinks, scale)
        o = _into("cache_attention", out, o, starts)
        return (o, lse) if return_lse else o
    return _cache_attention(q, k_cache, v_cache, table, lengths, scales, starts, window, sinks, scale, return_lse, out, workspace)


def _cache_attention(q, k_cache, v_cache, table, lengths, scales, starts, window, sinks, scale, return_lse, out, workspace):
    f, dtype, device = "cache_attention", q.dtype, k_cache.device
    _no_tangents(f, q, k_cache, v_cache)
    if dtype not in _DTYPE:
        raise TypeError("cache_attention: q must be float16 or bfloat16")
    if scales is not None:
        _check_cache8(f, k_cache, v_cache, scales)
    else:
        if k_cache.dtype != dtype or v_cache.dtype != dtype or not k_cache.is_cuda:
            raise TypeError("cache_attention: without scales the caches must be device tensors of q's dtype")
        _check_shapes(f, k_cache, v_cache)
    window, sinks = _visible(f, window, sinks)
    q = _rows(f, "q", q, dtype, device, "float16 or bfloat16")
    per_head = table.dim() == 3 and starts is None
    _check_ints(f, "table", table, 3 if per_head else 2, device)
    _check_ints(f, "lengths", lengths, 1, device)
    dev, qs, cs, ts = device.index, q.shape, k_cache.shape, table.shape
    _need(qs[2] == cs[3], f, "q must be [tokens, heads, %d]" % cs[3])
    _need(lengths.shape[0] == ts[0] and (not per_head or ts[1] == cs[1]), f,
          "table must be [sequences, width] or, without starts, [sequences, kv_heads, width], and lengths [sequences]")
    pages, kv_heads, page_size, D = cs
    tokens, heads, _ = qs
    n = ts[0]
    if starts is not None:
        _check_ints(f, "starts", starts, 1, device)
        _need(starts.shape[0] == n + 1, f, "starts must have one entry more than table has rows")
    elif tokens != n:
        raise ValueError("cache_attention: without starts there is one token per row of table")
    if out is None:
        out = _empty_like(q, memory_format=_contiguous)
    else:
        _check_out(f, out, (tokens, heads, D), dtype, device)
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=device) if return_lse else None
    stream = _raw_stream(dev)
    qt, tt = q.stride(), table.stride()
    ptrs = (q.data_ptr(), qt[0], qt[1], k_cache.data_ptr(), v_cache.data_ptr(), 0 if scales is None else scales.data_ptr(),
            table.data_ptr(), tt[0], tt[1] if per_head else 0, lengths.data_ptr(), 0 if starts is None else starts.data_ptr(), tokens,
            window, sinks, out.data_ptr(), 0 if lse is None else lse.data_ptr())
    sizes = (n, heads, kv_heads, D, pages, page_size, ts[-1], 1.0 / math.sqrt(D) if scale is None else scale, _DTYPE[dtype])
    need = B.marlin_cache_attention_workspace_bytes(int(starts is not None), tokens, n, heads, kv_heads, D)
    for nbytes in (0, need):  # grown if the call says WORKSPACE_TOO_SMALL
        buf = kv._workspace(f, dev, stream, workspace, nbytes)
        with torch.cuda.device(dev):
            status = B.lib().marlin_cache_attention(B.pack_cache_attention(*ptrs, buf.data_ptr(), buf.numel(), *sizes), stream)
        if status != 5:
            break
    if status:
        raise B.MarlinError("marlin_cache_attention", status)
    return (out, lse) if return_lse else out


def assign_pages(table: torch.Tensor, lengths: torch.Tensor, new: torch.Tensor, free: torch.Tensor, free_count: torch.Tensor,
                 page_size: int, tokens: int, window: int | None = None, sinks: int = 0,
                 workspace: "ops.Workspace | None" = None, back: torch.Tensor | None = None):
    """The tables of a step (``marlin_assign_pages``): sequence b of ``table`` int32 [sequences, width] gets ``new[b]`` tokens, or ends
    where that is below 0.  Takes pages from, and gives them back to, ``free`` int32 [pages], whose
    first ``free_count`` (int32 [1]) entries are the free pages, and brings ``lengths`` up to date, all in place.
    Returns (starts int32 [sequences + 1], slots int64 [tokens]): the rows of each sequence's new tokens, and each
    token's page * page_size + slot, -1 behind the last.

    Sequences are served in their order while pages, room in the table and ``tokens`` rows last; one that is not gets no tokens in this
    step and keeps its length (its rows in ``starts`` are none; calls without ``starts`` have to be told: see the module's docstring).  With ``window`` the pages that a token sees neither through it nor among the
    first ``sinks`` positions are given back and their entries become -1.

    ``back`` int32 [sequences] takes tokens back first: drafted ones that were not accepted.  Lengths fall by it, and the pages that no token is
    left in are given back; the next tokens take the others' slots.  (What those had widened stays: the scale of an 8-bit block, a page's
    bounds.  Behind a window take back no more than the last call's tokens, as pages that earlier ones would see may be gone.)  A length that is lowered in another way loses the pages behind it, as entries behind a sequence's last page are overwritten without a
    look.  A page belongs to one sequence: it is given back with the first that names it."""
    done = (_native or _connect()).assign_pages(table, lengths, new, free, free_count, page_size, tokens, window, sinks, workspace, back)
    if done is not None:
        return done
    if _watched(table, lengths, new, free, free_count, back):
        window, sinks = _visible("assign_pages", window, sinks)
        return torch.ops.marlin_mi355x.assign_pages(table, lengths, new, free, free_count, page_size, tokens, window, sinks, back)
    return _assign_pages(table, lengths, new, free, free_count, page_size, tokens, window, sinks, workspace, back)


def _assign_pages(table, lengths, new, free, free_count, page_size, tokens, window, sinks, workspace, back):
    f, device = "assign_pages", table.device
    for name, x, dims in (("table", table, 2), ("lengths", lengths, 1), ("new", new, 1), ("free", free, 1), ("free_count", free_count, 1)):
        _check_ints(f, name, x, dims, device)
    if back is not None:
        _check_ints(f, "back", back, 1, device)
        _need(back.shape == lengths.shape, f, "back must have one entry per row of table")
    window, sinks = _visible(f, window, sinks)
    page_size, tokens = operator.index(page_size), operator.index(tokens)
    n, width = table.shape
    _need(lengths.shape[0] == n and new.shape[0] == n and free_count.shape[0] == 1, f,
          "lengths and new must have one entry per row of table, free_count one")
    _need(n <= 1 or table.stride(0) >= width, f, "the rows of table must not overlap")
    if not 0 <= tokens <= 1 << 24:
        raise B.MarlinError("marlin_assign_pages", 2)
    starts = torch.empty(n + 1, dtype=torch.int32, device=device)
    slots = torch.empty(tokens, dtype=torch.int64, device=device)
    dev = device.index
    stream = _raw_stream(dev)
    ptrs = (table.data_ptr(), table.stride(0), lengths.data_ptr(), new.data_ptr(), free.data_ptr(), free_count.data_ptr(),
            starts.data_ptr(), slots.data_ptr())
    for nbytes in (0, B.marlin_assign_pages_workspace_bytes(n)):
        buf = kv._workspace(f, dev, stream, workspace, nbytes)
        with torch.cuda.device(dev):
            status = B.lib().marlin_assign_pages(B.pack_assign_pages(
                *ptrs, buf.data_ptr(), buf.numel(), n, width, free.shape[0], page_size, tokens, window, sinks,
                0 if back is None else back.data_ptr()), stream)
        if status != 5:
            break
    if status:
        raise B.MarlinError("marlin_assign_pages", status)
    return starts, slots

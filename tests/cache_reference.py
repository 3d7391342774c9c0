"""Plain forms, on the CPU and from their definitions, of the 8-bit cache, of attention of any number of new tokens with a window, and
of the page tables; and the error bounds of the 16-bit results.

Attention is in 64 bits.  Its bounds count unit roundoffs as ``kv_reference`` does: a result is rounded once to its type, a weight once
at the most, everything else is fp32.  An 8-bit cache's scales enter the weights by a logarithm and a reciprocal of one ulp each: of
up to 40 in magnitude, 2^-18 absolute, so 2^-18 of a weight; 2^-16 covers both sides of the quotient.

Codes are whole numbers: their form repeats the definition's fp32 operations one by one, which leaves nothing to a bound.
"""
import math

import torch

from kv_reference import TINY, U

E4M3 = torch.float8_e4m3fn
BLOCK = 16


def held(cache, scales, which):
    """The cache's elements in 64 bits and, [pages, kv heads, page size], whether their scale is one."""
    P, H, ps, D = cache.shape
    if scales is None:
        return cache.double(), torch.ones(P, H, ps, dtype=torch.bool)
    s = scales.double()
    ok = ((s >= 2.0 ** -40) & (s <= 2.0 ** 40)).all(2)  # keys' and values'
    x = cache.float().double().view(P, H, ps // BLOCK, BLOCK, D) * s[:, :, which][..., None, None]
    return x.view(P, H, ps, D), ok.repeat_interleave(BLOCK, 2)


def attention(q, k_cache, v_cache, table, lengths, scales=None, starts=None, window=None, sinks=0, scale=None):
    """out, lse, the bounds of their errors, and which rows belong to a sequence.  Values that are not finite count where they are seen."""
    T, heads, D = q.shape
    pages, kv_heads, ps, _ = k_cache.shape
    scale = D ** -0.5 if scale is None else scale
    group = heads // kv_heads
    u, tiny = U[q.dtype], TINY[q.dtype]
    keys, fine = held(k_cache, scales, 0)
    values, _ = held(v_cache, scales, 1)
    out = torch.zeros(T, heads, D, dtype=torch.float64)
    lse = torch.full((T, heads), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    mine = torch.zeros(T, dtype=torch.bool)
    starts = list(range(len(lengths) + 1)) if starts is None else [int(x) for x in starts]
    extra = 0 if scales is None else 2.0 ** -16
    for b in range(len(lengths)):
        n = starts[b + 1] - starts[b]
        mine[starts[b]:starts[b + 1]] = True
        first = max(0, int(lengths[b])) - n
        for h in range(kv_heads):
            row = table[b, h] if table.dim() == 3 else table[b]
            j = torch.arange(max(0, min(first + n, len(row) * ps)))
            page = row[j // ps].long()
            ok = (page >= 0) & (page < pages)
            j, page = j[ok], page[ok]
            ok = fine[page, h, j % ps]
            j, page = j[ok], page[ok]
            if len(j) == 0 or n == 0:
                continue
            pos = first + torch.arange(n)[:, None]
            sees = j <= pos
            if window:
                sees &= (j > pos - window) | (j < sinks)
            K, V = keys[page, h, j % ps], values[page, h, j % ps]
            x = q[starts[b]:starts[b + 1], h * group:(h + 1) * group].double()  # [n, group, D]
            s = (torch.einsum("ngd,jd->ngj", x, K) * scale).masked_fill(~sees[:, None], -math.inf)
            m = s.amax(-1, keepdim=True)
            e = torch.where(sees[:, None], torch.exp(s - m), 0)
            e = torch.where(m == -math.inf, 0, e)
            total = e.sum(-1)
            some = total > 0
            plain = torch.where(torch.isfinite(V), V, 0)
            o = torch.einsum("ngj,jd->ngd", e, plain)
            for odd, what in ((V == math.inf, math.inf), (V == -math.inf, -math.inf), (torch.isnan(V), math.nan)):
                if odd.any():
                    o = torch.where(torch.einsum("nj,jd->nd", sees.double(), odd.double())[:, None] > 0, o + what, o)
            o = torch.where(some[..., None], o / total[..., None], 0)
            big = torch.einsum("ngd,jd->ngj", x.abs(), K.abs()).masked_fill(~sees[:, None], 0).amax(-1)
            top = s.masked_fill(~sees[:, None], 0).abs().amax(-1)
            off = D * 2.0 ** -24 * big * abs(scale) + 2.0 ** -21 * top
            spread = torch.einsum("ngj,jd->ngd", e, plain.abs()) / total[..., None]
            lost = sees.double() @ plain.abs()
            w = slice(starts[b], starts[b + 1]), slice(h * group, (h + 1) * group)
            out[w] = o
            lse[w] = torch.where(some, m[..., 0] + torch.log(total), -math.inf)
            tol[w] = torch.where(some[..., None], u * o.abs() + (u + 2 * off[..., None] + 2.0 ** -18 + extra) * spread + tiny +
                                 tiny * lost[:, None] / total[..., None], 0)
            tol_lse[w] = torch.where(some, off + 2.0 ** -21 * (1 + lse[w].abs()) + 2.0 ** -20 + extra, 0)
    return out, lse, tol, tol_lse, mine


# ---- the 8-bit append ----

def scale_of(a):
    """The least power of two, 2^-40 .. 2^40, with a <= 448 times it."""
    e = -40
    while e < 40 and a > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def encode(x, s):
    """fp32 x to codes of scale s: the nearest e4m3 number to x / s, ties to even."""
    y = (x * torch.tensor(1 / s, dtype=torch.float32)).clamp(-448, 448)
    y = torch.where(torch.isfinite(x), y, math.nan)
    return nearest(y.double())


def nearest(y):
    """64-bit y, at most 448 in magnitude, to the nearest e4m3 number (from their list), ties to even."""
    codes = torch.arange(127, dtype=torch.uint8)
    grid = codes.view(E4M3).float().double()
    a = y.abs().nan_to_num(0)
    hi = torch.searchsorted(grid, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    down, up = a - grid[lo], grid[hi] - a
    pick = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    pick = torch.where(torch.isnan(y), 127, pick)
    return (pick + 128 * (torch.signbit(y) & ~torch.isnan(y)).long()).to(torch.uint8)


def rotate32(x, cs, interleaved):
    """x [heads, D] fp32, rotated by a row of the table, each operation rounded to fp32."""
    rot = len(cs)
    y = x.clone()
    i = torch.arange(rot // 2)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    c, s, a, b = cs[:rot // 2], cs[rot // 2:], x[:, ia], x[:, ib]
    y[:, ia], y[:, ib] = a * c - b * s, b * c + a * s
    return y


def append8(k, v, k_cache, v_cache, scales, table, lengths, cos_sin=None, starts=None, interleaved=False):
    """The caches (uint8 codes) and scales after the call."""
    pages, H, ps, D = k_cache.shape
    codes = [x.view(torch.uint8).clone() for x in (k_cache, v_cache)]
    scales = scales.clone()
    starts = list(range(len(lengths) + 1)) if starts is None else [int(x) for x in starts]
    for b in range(len(lengths)):
        n = starts[b + 1] - starts[b]
        first = max(0, int(lengths[b])) - n
        blocks = {}
        for i in range(n):
            pos = first + i
            if pos < 0 or pos >= table.shape[1] * ps or (cos_sin is not None and pos >= len(cos_sin)):
                continue
            page = int(table[b, pos // ps])
            if 0 <= page < pages:
                blocks.setdefault(pos // BLOCK, []).append((pos, page, starts[b] + i))
        for block, rows in blocks.items():
            page, part, slot0 = rows[0][1], block * BLOCK % ps // BLOCK, block * BLOCK % ps
            for which, x in ((0, k), (1, v)):
                new = [x[t].float() for _, _, t in rows]
                if which == 0 and cos_sin is not None:
                    new = [rotate32(y, cos_sin[pos], interleaved) for y, (pos, _, _) in zip(new, rows)]
                new = torch.stack(new)  # [tokens, heads, D]
                older = max(0, rows[0][0] - block * BLOCK)
                for h in range(H):
                    mine = new[:, h]
                    s = scale_of(float(torch.where(torch.isfinite(mine), mine.abs(), 0).max()))
                    was = float(scales[page, h, which, part])
                    if older and 2.0 ** -40 <= was <= 2.0 ** 40:
                        if was > s:
                            s = was
                        elif s > was:
                            at = slice(slot0, slot0 + older)
                            old = codes[which][page, h, at].view(E4M3).float()
                            codes[which][page, h, at] = nearest((old * torch.tensor(was / s, dtype=torch.float32)).double())
                    scales[page, h, which, part] = s
                    for y, (pos, _, _) in zip(mine, rows):
                        codes[which][page, h, pos % ps] = encode(y, s)
    return codes[0], codes[1], scales


# ---- page tables ----

def assign_pages(table, lengths, new, free, count, page_size, tokens, window=None, sinks=0):
    """table, lengths, free, free_count after the call, starts and slots: sequence by sequence."""
    table, lengths, free = table.clone(), lengths.clone(), free.clone()
    B, width = table.shape
    pages, cap = len(free), width * page_size
    count = min(max(int(count), 0), pages)

    def names(x):
        return 0 <= int(x) < pages

    had = [min(max(int(n), 0), cap) for n in lengths]
    for b in range(B):
        back = []
        if new[b] < 0:
            back = [i for i in range(-(-had[b] // page_size)) if names(table[b, i])]
            lengths[b] = 0
        elif window:
            i = max(0, had[b] - window) // page_size - 1
            while i >= -(-sinks // page_size) and names(table[b, i]):
                back.insert(0, i)
                i -= 1
        for i in back:
            if count < pages:
                free[count] = table[b, i]
                count += 1
            table[b, i] = -1
    starts, slots, room, open_ = [0], [-1] * tokens, count, True
    for b in range(B):
        n = int(new[b])
        if n > 0 and had[b] + n <= cap:
            need = -(-(had[b] + n) // page_size) - -(-had[b] // page_size)
            open_ = open_ and need <= room and starts[-1] + n <= tokens  # the first that is not served ends it
            if open_:
                for i in range(-(-had[b] // page_size), -(-(had[b] + n) // page_size)):
                    room -= 1
                    table[b, i] = free[room]
                for i in range(n):
                    pos = had[b] + i
                    page = int(table[b, pos // page_size])
                    slots[starts[-1] + i] = page * page_size + pos % page_size if names(page) else -1
                lengths[b] = had[b] + n
                starts.append(starts[-1] + n)
                continue
        starts.append(starts[-1])
    return table, lengths, free, room, torch.tensor(starts, dtype=torch.int32), torch.tensor(slots, dtype=torch.int64)

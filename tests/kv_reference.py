"""Plain 64-bit forms of the paged key-value cache operators, on the CPU,
position by position from their definitions, and the error bounds of the 16-bit
results.

Unit roundoffs: a result is rounded once to its type (u: 2^-11 for float16,
2^-8 for bfloat16, half an ulp being at most u |x|), float16's subnormals have
an absolute half ulp of 2^-25, and everything before is fp32 (2^-24 an operation).
"""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}


def rows_of(table, b, kvh):
    return table[b, kvh] if table.dim() == 3 else table[b]


def attention(q, k_cache, v_cache, table, lengths, scale=None):
    """out, lse and the bounds of their errors (64 bits): all inputs on the CPU."""
    n, heads, D = q.shape
    pages, kv_heads, ps, _ = k_cache.shape
    scale = D ** -0.5 if scale is None else scale
    u, tiny = U[q.dtype], TINY[q.dtype]
    out = torch.zeros(n, heads, D, dtype=torch.float64)
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(n):
        length = min(max(int(lengths[b]), 0), table.shape[-1] * ps)
        pos = torch.arange(length)
        for h in range(heads):
            kvh = h // (heads // kv_heads)
            page = rows_of(table, b, kvh)[pos // ps].long()
            ok = (page >= 0) & (page < pages)
            page, slot = page[ok], (pos % ps)[ok]
            if len(page) == 0:
                continue
            x, keys = q[b, h].double(), k_cache[page, kvh, slot].double()
            values = v_cache[page, kvh, slot].double()
            s = (keys * x).sum(1) * scale
            m = s.max()
            if m == -math.inf:
                continue
            e = torch.exp(s - m)
            total = e.sum()
            out[b, h] = (e[:, None] * values).sum(0) / total
            lse[b, h] = m + torch.log(total)
            # a score: D products and sums in fp32, then a scaling and the exponent's argument
            off = D * 2.0 ** -24 * float((keys * x).abs().sum(1).max()) * abs(scale) + 2.0 ** -21 * float(s.abs().max())
            spread = (e[:, None] * values.abs()).sum(0) / total
            # the output's rounding; the weights' (u each, or an absolute one of subnormals, once per wave's maximum);
            # the scores' twice (numerator and sum); the fp32 sums'
            tol[b, h] = (u * out[b, h].abs() + (u + 2 * off + 2.0 ** -18) * spread + tiny
                         + tiny * values.abs().sum(0) / total)
            tol_lse[b, h] = off + 2.0 ** -21 * (1 + abs(float(lse[b, h]))) + 2.0 ** -20
    return out, lse, tol, tol_lse


def rotate(x, angles, rot, interleaved):
    """x [heads, D] and one row of the table, both 64-bit: rotated, and the largest term of each channel's sum."""
    y, big = x.clone(), x.abs()
    c, s = angles[:rot // 2], angles[rot // 2:]
    i = torch.arange(rot // 2)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    a, b = x[:, ia], x[:, ib]
    y[:, ia], y[:, ib] = a * c - b * s, b * c + a * s
    big[:, ia], big[:, ib] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, big


def append(q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, interleaved):
    """Rotated queries, keys and values by (page, slot): ({(page, slot): (k, v)}, q_out), each k and q with its
    error's bound.  Values are the inputs' own bits."""
    n = len(lengths)
    ps, pages = k_cache.shape[2], k_cache.shape[0]
    u, tiny = U[q.dtype], TINY[q.dtype]
    rot = 0 if cos_sin is None else cos_sin.shape[1]
    starts = list(range(n + 1)) if starts is None else [int(x) for x in starts]
    q_out, q_tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    put = {}
    for b in range(n):
        count = starts[b + 1] - starts[b]
        for i in range(count):
            t, pos = starts[b] + i, max(int(lengths[b]), 0) - count + i
            if pos < 0 or pos >= table.shape[1] * ps or (rot and pos >= cos_sin.shape[0]):
                continue
            page = int(table[b, pos // ps])
            if not 0 <= page < pages:
                continue
            got = []
            for x in (q[t], k[t]):
                x = x.double()
                y, big = rotate(x, cos_sin[pos].double(), rot, interleaved) if rot else (x, x.abs())
                tol = u * y.abs() + tiny + 2.0 ** -22 * big
                tol[:, rot:] = 0  # copied
                got.append((y, tol))
            (q_out[t], q_tol[t]), key = got
            put[page, pos % ps] = (key, v[t])
    return put, q_out, q_tol


def order(x):
    """16-bit floats as integers in the order -NaN < -inf < ... < -0 < 0 < ... < inf < NaN."""
    w = x.view(torch.int16).int()
    return torch.where(w < 0, w ^ 0x7FFF, w)


def select(q, bounds, table, lengths, ps, count):
    """chosen [n, kv heads, count] and lengths, from scores in 64 bits (exact where the inputs are small integers)."""
    n, heads, D = q.shape
    pages, kv_heads = bounds.shape[:2]
    group = heads // kv_heads
    chosen = torch.full((n, kv_heads, count), -1, dtype=torch.int32)
    tokens = torch.zeros(n, dtype=torch.int32)
    for b in range(n):
        length = min(max(int(lengths[b]), 0), table.shape[1] * ps)
        used = -(-length // ps)
        tokens[b] = length if used <= count else length - (used - count) * ps
        for h in range(kv_heads):
            best = list(range(used))
            if used > count:
                score = []
                for i in range(used):
                    page = int(table[b, i])
                    if not 0 <= page < pages:
                        score.append((-math.inf, 1))
                        continue
                    lo, hi = bounds[page, h].double()
                    x = q[b, h * group:(h + 1) * group].double()
                    s = (torch.clamp(x, max=0) * lo + torch.clamp(x, min=0) * hi).sum(1)
                    score.append((math.inf, 0) if torch.isnan(s).any() else (float(s.max()), 0))
                score[-1] = (math.inf, -1)
                best = sorted(sorted(range(used), key=lambda i: (-score[i][0], score[i][1], i))[:count])
            for i, at in enumerate(best):
                chosen[b, h, i] = table[b, at]
    return chosen, tokens

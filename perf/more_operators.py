"""Performance cases of the 8-bit key-value cache, of attention with a window and of several new
tokens over a cache, and of the tables that both go by.

Over the paged cache of ``operators.py`` (pages [pages, kv heads, page size, head dim], a table
[sequences, pages], lengths):

* append: new tokens, rotated by their positions, into a cache of 8-bit floating-point elements with
  a scale for each kv head and block of 16 slots, of keys and of values (scales [pages, kv heads, 2, page size / 16]);
* attend: attention of one new token per sequence, over a cache of 8 or 16 bits, of everything or of the last
  ``window`` positions and the first ``sinks``;
* prompt: the same of several new tokens per sequence, each of which sees the positions up to its own;
* pages: the pages of a step's new tokens are taken from a list of free ones, those of ended sequences and those that
  no window sees any more are given back; starts and slots of the new tokens.

"step" is all of it as a decode step of an 8-bit cache runs it.  ``run`` computes them in elementary torch operations in
fp32 (``own`` false) or by this package's entry points (``own`` true).

Values: activations N(0, 1), some key channels four times larger, values with a per-channel offset.  Tables are random
permutations; entries that no token uses are -1.  The sizes of a case are the same for every seed, in another order.
"""
import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
LARGEST = 64 * 32768 * 8 * 128  # keys of the largest listed case, in elements
SCORES = 8192 * 8192 * 32  # scores of the largest prompts, whole and padded
BLOCK = 16  # slots that share a scale
LEAST, MOST = 2.0 ** -40, 2.0 ** 40  # scales


def _case(kind, B, hq, hkv, D, ps, dtype, lo, hi, name=None, **more):
    """lo, hi: tokens of the sequences before the call; new: the most new ones."""
    case = {"kind": kind, "B": B, "hq": hq, "hkv": hkv, "D": D, "ps": ps, "dtype": dtype, "bits": 8, "lo": lo, "hi": hi,
            "new": 1, "least": 1, "window": 0, "sinks": 0, "rot": D, "interleaved": False, "zeros": False, "lse": False}
    case.update(more)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # single-stream decode of a 4096-wide layer: launch latency and host time are what counts
        _case("append", 1, 32, 8, 128, 16, "f16", 1000, 1000, name="append8_b1"),
        # prompts of 1 to 4096 tokens in one call, half of them behind what is cached already
        _case("append", 24, 64, 8, 128, 32, "bf16", 0, 700, name="append8_prompts", new=4096, interleaved=True),
        # an ordinary decode batch of a 4096-wide layer, with the logarithms of the sums
        _case("attend", 16, 32, 8, 128, 16, "f16", 500, 4000, name="attend8_b16", lse=True),
        # the largest: a full batch of long contexts
        _case("attend", 64, 64, 8, 128, 64, "bf16", 32767, 32767, name="attend8_b64_long"),
        # ragged long contexts of which a token sees a window and the first four, and sequences without any
        _case("attend", 32, 64, 8, 128, 32, "f16", 300, 60000, name="window_b32", bits=16, window=4096, sinks=4, zeros=True),
        # one long prompt of a 4096-wide layer
        _case("prompt", 1, 32, 8, 128, 16, "f16", 0, 0, name="prompt_8k", bits=16, new=8192, least=8192),
        # prompts of 1 to 2048 tokens, half of them behind what is cached, through a window and sinks
        _case("prompt", 4, 64, 8, 128, 64, "bf16", 100, 2000, name="prompt_window", bits=16, new=2048, window=1024, sinks=4),
        # chunks of long prompts over an 8-bit cache
        _case("prompt", 4, 32, 8, 128, 32, "f16", 15000, 16384, name="prompt8_chunks", new=512, least=512),
        # up to four drafted tokens of each sequence are looked over at once
        _case("prompt", 32, 32, 8, 128, 16, "f16", 300, 8000, name="draft8_b32", new=4, least=4, lse=True),
        # the tables of a decode step: most sequences get a token, some end, windows leave pages behind
        _case("pages", 128, 1, 1, 64, 16, "f16", 1, 2500, name="pages_b128", window=1024, sinks=4),
        # the tables of prompts for a large batch
        _case("pages", 512, 1, 1, 64, 32, "f16", 0, 4000, name="pages_prompts", new=4096),
        # tables, append and attention, as a decode step of narrow heads runs them
        _case("step", 32, 40, 40, 64, 16, "bf16", 1, 2500, name="step8_b32_d64"),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    while True:
        kind = rng.choices(["append", "attend", "prompt", "pages", "step"], [20, 25, 30, 12, 13])[0]
        D = rng.choice([64, 96, 128, 128, 128, 256])
        hkv = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
        hq = hkv * rng.choice([g for g in (1, 2, 4, 5, 8, 12, 16, 32) if hkv * g <= 128])
        ps, dtype = rng.choice([16, 32, 64, 128, 256]), rng.choice(["f16", "bf16"])
        more = {"bits": rng.choice([8, 8, 16]) if kind == "prompt" else 8, "interleaved": rng.random() < 0.3,
                "zeros": kind == "attend" and rng.random() < 0.25, "rot": rng.choice([D, D, D // 2])}
        if rng.random() < 0.4 and kind != "append":
            more.update(window=_log(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 64]))
            if kind == "attend":
                more["bits"] = rng.choice([8, 16])
        if kind in ("attend", "prompt"):
            more["lse"] = rng.random() < 0.5
        B = _log(rng, 1, 256 if kind in ("attend", "step") else 2048 if kind == "pages" else 64)
        lo = _log(rng, 1, 8192) - 1
        hi = max(lo, _log(rng, 16, 65536))
        if kind == "prompt" or kind in ("append", "pages") and rng.random() < 0.5:
            more["new"] = _log(rng, 2, 8192)
            more["least"] = rng.choice([1, more["new"]])
        if kind == "append" and "new" in more:
            lo, hi = 0, rng.randint(0, 2000)
        case = _case(kind, B, hq, hkv, D, ps, dtype, lo, hi, **more)
        n, width, most = sum(_lengths(case)), _width(case), max(_new(case))
        room = LARGEST // (8 if kind in ("append", "prompt", "step") else 1)
        if kind == "pages":
            if n <= 4_000_000 and B * width <= 4_000_000:
                return case
        elif n * hkv * D <= room and B * width * ps * hkv * D <= LARGEST and sum(_new(case)) * (hq + 2 * hkv) * D <= 2 ** 29 and \
                (kind == "append" or B * most * hq * width * ps <= SCORES):
            return case


# ---- what a case's sequences are ----

def _spread(lo, hi, n):
    """n numbers from lo to hi, spread over their logarithm; the last is hi."""
    a, b = math.log(lo + 1), math.log(hi + 1)
    return [round(math.exp(b if n == 1 else a + (b - a) * i / (n - 1))) - 1 for i in range(n)]


def _new(case):
    """New tokens of each sequence; -1 where it ends."""
    got = [max(1, n) for n in _spread(case["least"], case["new"], case["B"])]
    if case["kind"] == "pages":
        return [-1 if i % 16 == 5 else 0 if i % 16 == 9 else n for i, n in enumerate(got)]
    return got


def _cached(case):
    got = _spread(case["lo"], case["hi"], case["B"])
    if case["new"] > 1 and case["least"] == 1:  # every other prompt is the sequence's first
        got = [n if i % 2 else 0 for i, n in enumerate(got)]
    if case["zeros"]:  # no tokens at all, the new one aside, which _lengths leaves out
        got = [0 if i % 8 == 3 else n for i, n in enumerate(got)]
    return got


def _lengths(case):
    """Tokens of each sequence, the new ones included."""
    return [0 if case["zeros"] and i % 8 == 3 else c + max(0, n) for i, (c, n) in enumerate(zip(_cached(case), _new(case)))]


def _width(case):
    return max(1, max(-(-(c + max(0, n)) // case["ps"]) for c, n in zip(_cached(case), _new(case))))


def _seen(case, length, new):
    """(keys that some new token sees, pairs of a token and a key that it sees)"""
    W, S = case["window"], case["sinks"]
    first = length - new  # position of the first new token
    if not W or length <= W:
        return length, new * first + new * (new + 1) // 2
    low = max(first - W + 1, 0)
    keys = length - low + min(S, low)
    pairs = sum(min(p + 1, W) + min(S, max(0, p + 1 - W)) for p in range(first, length))
    return keys, pairs


def work(case):
    B, hq, hkv, D, ps = (case[k] for k in ("B", "hq", "hkv", "D", "ps"))
    lengths, new, kind = _lengths(case), _new(case), case["kind"]
    nbytes = flops = 0
    if kind in ("append", "step"):
        tokens = sum(n for n, m in zip(new, lengths) if m)
        blocks = sum((m - 1) // BLOCK - (m - n) // BLOCK + 1 for n, m in zip(new, lengths) if m)
        nbytes += 2 * tokens * (2 * hq + 2 * hkv) * D + tokens * 2 * hkv * D + 4 * tokens * case["rot"] + 8 * blocks * hkv + 12 * B
        flops += tokens * (3 * (hq + hkv) * case["rot"] + 4 * hkv * D)
    if kind in ("attend", "prompt", "step"):
        seen = [_seen(case, m, n) if m else (0, 0) for n, m in zip(new, lengths)]
        size = 2 * (1 if case["bits"] == 8 else 2) * D + (8 / BLOCK if case["bits"] == 8 else 0)
        nbytes += int(sum(s[0] for s in seen) * hkv * size) + 4 * sum(-(-s[0] // ps) for s in seen) + 8 * B
        nbytes += 2 * 2 * sum(new) * hq * D + (4 * sum(new) * hq if case["lse"] else 0)
        flops += sum(s[1] for s in seen) * hq * 4 * D
    if kind in ("pages", "step"):
        some = [max(0, n) for n in new]
        nbytes += 16 * B + 8 * sum(some) + 8 * sum(-(-m // ps) - -(-(m - n) // ps) for n, m in zip(some, lengths))
        flops += 8 * B + 4 * sum(some)
    return {"bytes": nbytes, "flops": flops}


# ---- inputs ----

def _quantise(x):
    """x [pages, kv heads, page size, D] to codes and scales [pages, kv heads, page size / 16]."""
    P, H, ps, D = x.shape
    x = x.float().view(P, H, ps // BLOCK, BLOCK * D)
    s = _scale_of(x.abs().amax(-1))
    return (x / s[..., None]).to(torch.float8_e4m3fn).view(P, H, ps, D), s


def _scale_of(a):
    """The least power of two, 2^-40 to 2^40, with a <= 448 times it."""
    m, e = torch.frexp(a)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(-40, 40)
    return torch.ldexp(torch.ones_like(a), torch.where(a == 0, -40, e))


def prepare(case, seed):
    B, hq, hkv, D, ps = (case[k] for k in ("B", "hq", "hkv", "D", "ps"))
    dt, dev, kind = DTYPES[case["dtype"]], "cuda", case["kind"]
    g = torch.Generator(device=dev).manual_seed(int(seed))
    order = random.Random(int(seed))

    def randn(*shape):
        return torch.randn(shape, dtype=dt, device=dev, generator=g)

    rows = list(zip(_lengths(case), _new(case), _cached(case)))
    order.shuffle(rows)
    lengths, new, cached = ([r[i] for r in rows] for i in range(3))
    width = _width(case)
    paged = kind in ("pages", "step")  # the new tokens' pages are still to be found
    used = torch.tensor([-(-n // ps) for n in (cached if paged else lengths)], device=dev)
    pages = sum(-(-n // ps) for n in lengths) + 3
    at = torch.randperm(pages, device=dev, generator=g).to(torch.int32)
    i = torch.arange(width, device=dev)
    have = i < used[:, None]
    n_used = int(used.sum())
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    table[have] = at[:n_used]
    state = {"case": case, "tokens": sum(max(0, n) for n in new)}
    if paged:
        n_free = pages - n_used
        if case["window"]:  # earlier steps gave back what their windows had left behind
            gone = have & (i < ((torch.tensor(cached, device=dev) - case["window"] - 1).clamp(min=0) // ps)[:, None])
            gone &= i >= -(-case["sinks"] // ps)
            back = table[gone]
            table[gone] = -1
        else:
            back = table[:0].view(-1)
        # one array holds what a step changes, so that it can be put back for the next pass
        flat = torch.cat([table.view(-1), torch.tensor(cached, dtype=torch.int32, device=dev), at[n_used:], back,
                          at[:n_used - len(back)], torch.tensor([n_free + len(back)], dtype=torch.int32, device=dev)])
        state["before"], state["flat"] = flat, flat.clone()
        names, sizes = ("table", "lengths", "free", "free_count"), (B * width, B, pages, 1)
        state.update(zip(names, state["flat"].split(sizes)))
        state["table"] = state["table"].view(B, width)
        state["new"] = torch.tensor(new, dtype=torch.int32, device=dev)
    else:
        state["table"] = table
        state["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=dev)
        if case["new"] > 1:
            state["starts"] = torch.tensor([0] + new, device=dev).cumsum(0).to(torch.int32)
    if kind == "pages":
        return state

    loud = 1 + 3 * (torch.rand(D, device=dev, generator=g) < 0.05).to(dt)  # some key channels are larger
    k_cache, v_cache = randn(pages, hkv, ps, D), randn(pages, hkv, ps, D)
    k_cache *= loud
    v_cache += 0.5 * randn(D)
    state["scales"] = None
    if case["bits"] == 8:
        k_cache, ks = _quantise(k_cache)
        v_cache, vs = _quantise(v_cache)
        state["scales"] = torch.stack([ks, vs], 2)
    state["k_cache"], state["v_cache"] = k_cache, v_cache
    tokens = sum(new)
    if kind in ("append", "step"):
        # one projection gives all three: q, k and v are slices of its rows
        qkv = randn(tokens, (hq + 2 * hkv) * D)
        state["q"] = qkv[:, :hq * D].view(tokens, hq, D)
        state["k"] = qkv[:, hq * D:(hq + hkv) * D].view(tokens, hkv, D)
        state["v"] = qkv[:, (hq + hkv) * D:].view(tokens, hkv, D)
        state["k"] *= loud
        rot = case["rot"]
        angle = torch.arange(max(lengths), device=dev, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        state["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    else:
        state["q"] = randn(tokens, hq, D)
    return state


# ---- the plain forms ----

def _rotate(x, cs, rot, interleaved):
    """x [tokens, heads, D] in fp32, its first `rot` channels rotated by cs [tokens, rot] (cosines, then sines)."""
    c, s = cs[:, None, :rot // 2], cs[:, None, rot // 2:]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _token_rows(state):
    """Sequence and position of each new token."""
    lengths = state["lengths"].long()
    token = torch.arange(state["q"].shape[0], device=lengths.device)
    if "starts" not in state:
        return token, lengths - 1
    starts = state["starts"].long()
    seq = torch.searchsorted(starts[1:], token, right=True)
    return seq, lengths[seq] - starts[seq + 1] + token


def _put(cache, scales, x, block, slot, older, ps):
    """x [tokens, kv heads, D] in fp32 to slots of blocks (page * ps / 16 + block of the page) that hold `older` tokens."""
    P, H, _, D = cache.shape
    per = ps // BLOCK
    blocks, at = torch.unique(block, return_inverse=True)
    a = torch.zeros(len(blocks), H, device=x.device).index_reduce_(0, at, x.abs().amax(-1), "amax")
    n = torch.zeros_like(blocks).scatter_(0, at, older)
    page, part = blocks // per, blocks % per
    old = scales[page, :, part]
    s = torch.where(n[:, None] > 0, torch.maximum(old, _scale_of(a)), _scale_of(a))
    codes = cache.view(torch.uint8).view(P, H, per, BLOCK, D)
    have = codes[page, :, part].view(torch.float8_e4m3fn).float()  # [blocks, heads, 16, D]
    again = (have * (old / s)[:, :, None, None]).to(torch.float8_e4m3fn)
    keep = torch.arange(BLOCK, device=x.device) < n[:, None]
    codes[page, :, part] = torch.where(keep[:, None, :, None], again.view(torch.uint8), codes[page, :, part])
    scales[page, :, part] = s
    y = (x / s[at][..., None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[page[at], :, part[at], slot] = y


def _plain_append(state):
    case, scales = state["case"], state["scales"]
    q, k, v, ps, rot = state["q"], state["k"], state["v"], case["ps"], case["rot"]
    seq, pos = _token_rows(state)
    cs = state["cos_sin"][pos]
    q_out = _rotate(q.float(), cs, rot, case["interleaved"]).to(q.dtype)
    k_new = _rotate(k.float(), cs, rot, case["interleaved"])
    page = state["table"][seq, pos // ps].long()
    block = page * (ps // BLOCK) + pos % ps // BLOCK
    first = pos if "starts" not in state else state["lengths"].long()[seq] - (state["starts"][1:] - state["starts"][:-1]).long()[seq]
    older = (first - pos // BLOCK * BLOCK).clamp(min=0)
    _put(state["k_cache"], scales[:, :, 0], k_new, block, pos % BLOCK, older, ps)
    _put(state["v_cache"], scales[:, :, 1], v.float(), block, pos % BLOCK, older, ps)
    return q_out


def _read(cache, scales, at, head):
    """fp32 [B, kv heads, positions, D] of the pages `at` [B, 1, width]."""
    B, _, width = at.shape
    _, H, ps, D = cache.shape
    if scales is None:
        return cache[at, head].view(B, H, width * ps, D).float()
    x = cache.view(torch.uint8)[at, head].view(torch.float8_e4m3fn).float()
    return x.view(B, H, -1, BLOCK, D).mul_(scales[at, head].view(B, H, -1, 1, 1)).view(B, H, width * ps, D)


def _plain_attend(state, q):
    case, table, scales = state["case"], state["table"], state["scales"]
    hkv, W = case["hkv"], case["window"]
    T, hq, D = q.shape
    B, group = table.shape[0], hq // hkv
    seq, pos = _token_rows(state)
    first = torch.arange(B, device=q.device) if "starts" not in state else state["starts"][:-1].long()
    row = torch.arange(T, device=q.device) - first[seq]
    n = max(1, case["new"])
    rows = torch.zeros(B, n, hq, D, device=q.device)
    rows[seq, row] = q.float()
    where = torch.full((B, n), -1, dtype=torch.int64, device=q.device)
    where[seq, row] = pos
    head = torch.arange(hkv, device=q.device)[:, None]
    at = table.clamp(min=0).long()[:, None]
    keys = _read(state["k_cache"], None if scales is None else scales[:, :, 0], at, head)
    L = keys.shape[2]
    rows = rows.view(B, n, hkv, group, D).permute(0, 2, 1, 3, 4).reshape(B * hkv, n * group, D)
    s = torch.matmul(rows, keys.view(B * hkv, L, D).transpose(1, 2)).view(B, hkv, n, group, L).mul_(1 / math.sqrt(D))
    del keys
    j = torch.arange(L, device=q.device)
    p = where[:, :, None]
    off = j > p
    if W:
        off |= (j <= p - W) & (j >= case["sinks"])
    s.masked_fill_(off[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = s.sub_(m.clamp(min=-1e30)).exp_()
    total = e.sum(-1, keepdim=True)
    values = _read(state["v_cache"], None if scales is None else scales[:, :, 1], at, head)
    o = torch.matmul(e.view(B * hkv, n * group, L), values.view(B * hkv, L, D)).view(B, hkv, n, group, D)
    o = torch.where(total > 0, o / total, 0).permute(0, 2, 1, 3, 4).reshape(B, n, hq, D)[seq, row].to(q.dtype)
    if not case["lse"]:
        return [o]
    return [o, (m + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(B, n, hq)[seq, row]]


def _plain_pages(state):
    case = state["case"]
    table, lengths, free, count, new = (state[k] for k in ("table", "lengths", "free", "free_count", "new"))
    ps, tokens, W = case["ps"], state["tokens"], case["window"]
    i = torch.arange(table.shape[1], device=table.device)
    n = lengths.long().clamp(0, table.shape[1] * ps)
    a, ends = new.long(), (new < 0)[:, None]
    have = (n + ps - 1) // ps
    named = (table >= 0) & (table < len(free))
    back = ends & named & (i < have[:, None])
    if W:  # from the window's lower end back to the first entry that names no page
        left = (i >= -(-case["sinks"] // ps)) & (i < ((n - W).clamp(min=0) // ps)[:, None])
        stop = torch.where(left & ~named, i, -1).amax(1, keepdim=True)
        back |= ~ends & left & (i > stop)
    given = table[back]
    free[count + torch.arange(len(given), device=table.device)] = given
    table[back] = -1
    room = count.long() + len(given)
    fits = (a > 0) & (n + a <= table.shape[1] * ps)
    want = (n + a + ps - 1) // ps
    need = torch.where(fits, want - have, 0)
    upto = need.cumsum(0)
    served = fits & (upto <= room) & (torch.where(fits, a, 0).cumsum(0) <= tokens)
    got = torch.where(served, a, 0)
    take = served[:, None] & (i >= have[:, None]) & (i < want[:, None])
    rank = (upto - need - have)[:, None] + i
    table[take] = free[(room - 1 - rank)[take]]
    count.copy_(room - torch.where(served, need, 0).sum())
    starts = torch.cat([got.new_zeros(1), got.cumsum(0)])
    t = torch.arange(tokens, device=table.device)
    seq = torch.searchsorted(starts[1:], t, right=True).clamp(max=len(n) - 1)
    pos = n[seq] + t - starts[seq]
    page = table[seq, (pos // ps).clamp(max=table.shape[1] - 1)].long()
    slots = torch.where((t < starts[-1]) & (page >= 0), page * ps + pos % ps, -1)
    lengths.copy_(torch.where(ends[:, 0], 0, n + got))
    return starts.to(torch.int32), slots


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    q, starts, slots = state.get("q"), state.get("starts"), None
    window = case["window"] or None
    if own:
        import paper_2408_11743_amd as mk
        table, lengths = state["table"], state["lengths"]
        if kind in ("pages", "step"):
            state["flat"].copy_(state["before"])
            starts, slots = mk.assign_pages(table, lengths, state["new"], state["free"], state["free_count"], case["ps"],
                                            state["tokens"], window=window, sinks=case["sinks"])
        if kind in ("append", "step"):
            q = mk.kv_append8(q, state["k"], state["v"], state["k_cache"], state["v_cache"], state["scales"], table, lengths,
                              cos_sin=state["cos_sin"], starts=state.get("starts"), interleaved=case["interleaved"])
        if kind in ("attend", "prompt", "step"):
            got = mk.cache_attention(q, state["k_cache"], state["v_cache"], table, lengths, scales=state["scales"],
                                     starts=state.get("starts"), window=window, sinks=case["sinks"], return_lse=case["lse"])
            got = list(got) if case["lse"] else [got]
    else:
        if kind in ("pages", "step"):
            state["flat"].copy_(state["before"])
            starts, slots = _plain_pages(state)
        if kind in ("append", "step"):
            q = _plain_append(state)
        if kind in ("attend", "prompt", "step"):
            got = _plain_attend(state, q)
    cache = [state.get(k) for k in ("k_cache", "v_cache", "scales")]
    tables = [starts, slots, state["table"], state["lengths"], state.get("free"), state.get("free_count")]
    if kind == "pages":
        return tables
    if kind == "append":
        return [q] + cache
    return got + [q] + cache + tables if kind == "step" else got


# ---- the definitions in 64 bits, sequence by sequence ----

def exact(case, seed):
    kind = case["kind"]
    if kind == "pages":
        return None
    s = prepare(case, seed)
    hq, hkv, D, ps, rot = (case[k] for k in ("hq", "hkv", "D", "ps", "rot"))
    q, dev, before = s["q"].double(), s["q"].device, kind == "step"
    if before:  # as the tables' form leaves them; whole numbers are compared elsewhere
        _plain_pages(s)
    table, lengths = s["table"], s["lengths"].tolist()
    starts = s["starts"].tolist() if "starts" in s else list(range(len(lengths) + 1))
    out = []
    kc, vc = s["k_cache"], s["v_cache"]
    P = kc.shape[0]
    if kind in ("append", "step"):
        if kc.numel() * 16 > 8 << 30:
            return None
        kc, vc, scales = kc.double(), vc.double(), s["scales"].double()
        q_out = torch.zeros_like(q)
        half = rot // 2
        c = torch.arange(half, device=dev)
        ia, ib = (2 * c, 2 * c + 1) if case["interleaved"] else (c, c + half)
        for b, n in enumerate(lengths):
            t = torch.arange(starts[b], starts[b + 1], device=dev)
            pos = t - starts[b + 1] + n
            w = torch.complex(s["cos_sin"][pos, :half].double(), s["cos_sin"][pos, half:].double())[:, None]
            turned = []
            for x in (q[t], s["k"][t].double()):
                z = torch.complex(x[..., ia], x[..., ib]) * w
                x = x.clone()
                x[..., ia], x[..., ib] = z.real, z.imag
                turned.append(x)
            q_out[t] = turned[0]
            first = n - len(t)
            low = first // BLOCK * BLOCK  # whole blocks from here on
            page = table[b, torch.arange(low, -(-n // BLOCK) * BLOCK, BLOCK, device=dev) // ps].long()
            part = torch.arange(low, -(-n // BLOCK) * BLOCK, BLOCK, device=dev) % ps // BLOCK
            for which, cache, x in ((0, kc, turned[1]), (1, vc, s["v"][t].double())):
                cells = cache.view(P, hkv, ps // BLOCK, BLOCK, D)
                kept = cells[page, :, part] * scales[page, :, which, part][..., None, None]  # [blocks, heads, 16, D]
                kept = kept.transpose(1, 2).reshape(-1, hkv, D)
                mine = torch.zeros_like(kept)
                mine[first - low:n - low] = x
                blocks = mine.view(-1, BLOCK, hkv, D)
                new = _scale_of(blocks.abs().amax((1, 3)))
                if first > low:
                    new[0] = torch.maximum(new[0], scales[page[0], :, which, part[0]])
                held = kept.clone()
                held[first - low:n - low] = x
                codes = held.view(-1, BLOCK, hkv, D) / new[:, None, :, None]
                keep = torch.arange(len(page) * BLOCK, device=dev).view(-1, BLOCK) >= n - low  # slots behind the last token
                codes = torch.where(keep[..., None, None], cells[page, :, part].transpose(1, 2), _e4m3(codes))
                cells[page, :, part] = codes.transpose(1, 2)
                scales[page, :, which, part] = new
        q = q_out
        out = [q, kc, vc, scales]
        if kind == "append":
            return out
    o = torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=dev)
    group = hq // hkv
    for b, n in enumerate(lengths):
        t = torch.arange(starts[b], starts[b + 1], device=dev)
        if n == 0 or len(t) == 0:
            continue
        pos = t - starts[b + 1] + n
        low = max(0, int(pos[0]) - case["window"] + 1) if case["window"] else 0
        j = torch.arange(n, device=dev)
        j = j[(j >= low) | (j < case["sinks"])]
        p = pos[:, None].expand(-1, group).reshape(-1, 1)
        off = j > p
        if case["window"]:
            off |= (j <= p - case["window"]) & (j >= case["sinks"])
        page, slot = table[b, j // ps].long(), j % ps
        for h in range(hkv):
            keys, values = kc[page, h, slot].double(), vc[page, h, slot].double()
            if s["scales"] is not None:
                sc = (scales if before else s["scales"])[page, h]  # [keys, 2, page size / 16]
                keys *= sc[torch.arange(len(j), device=dev), 0, slot // BLOCK].double()[:, None]
                values *= sc[torch.arange(len(j), device=dev), 1, slot // BLOCK].double()[:, None]
            rows = q[t, h * group:(h + 1) * group].reshape(-1, D)
            x = torch.mm(rows, keys.t().contiguous()).mul_(D ** -0.5).masked_fill_(off, -math.inf)
            lse[t, h * group:(h + 1) * group] = torch.logsumexp(x, -1).view(-1, group)
            o[t, h * group:(h + 1) * group] = torch.mm(torch.softmax(x, -1), values).view(-1, group, D)
    got = [o, lse] if case["lse"] else [o]
    return got + out + [None] * 6 if before else got


def _e4m3(x):
    """x in 64 bits, rounded to four bits of significand (three below 2^-6, and fewer), ties to even."""
    e = torch.frexp(x).exponent.clamp(min=-5)
    unit = torch.ldexp(torch.ones_like(x), e - 4)
    return (torch.round(x / unit) * unit).clamp(-448, 448)

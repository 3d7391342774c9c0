"""Performance cases of the key-value cache operators: what one attention layer of
a served model asks for between its 4-bit projections.

Three operators, over one paged cache (k_cache and v_cache [pages, kv heads,
page size, head dim], a page table [sequences, pages] and the sequences'
lengths):

* append: the new tokens' queries and keys are rotated by their positions, the
  keys and values go to their pages, and (where the cache keeps them) each
  touched page's bounds, the smallest and largest key per channel, are updated;
* attend: attention of one new token per sequence over its cached keys and values;
* sparse: pages are scored by the largest product their bounds allow with the
  heads of the new token, the best ones of each kv head are chosen (the last
  page always), and the token attends to those alone.

"step" is an append of one token per sequence and the attention over it, as a
decode step runs them.  ``run`` computes them in elementary torch operations in
fp32 (``own`` false) or by this package's entry points (``own`` true).

Values: activations N(0, 1), some key channels four times larger, as trained
projections have them; values with a per-channel offset.  Where pages are to be
chosen, half as many pages as are chosen hold tokens that the query looks
for (attention is concentrated; that is what makes choosing sound), and the rest is noise.
Page tables are random permutations; slots and table entries that no token uses hold
older finite values and -1.  The lengths of a case are the same for every seed, in another order.
"""
import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
MAX_KV_BYTES = 64 * 32768 * 8 * 128 * 4  # keys and values of the largest listed case


def _case(kind, B, hq, hkv, D, ps, dtype, lo, hi, name=None, **more):
    case = {"kind": kind, "B": B, "hq": hq, "hkv": hkv, "D": D, "ps": ps, "dtype": dtype, "lo": lo, "hi": hi,
            "new": 1, "bounds": False, "interleaved": False, "rot": D, "zeros": False, "lse": False, "select": 0}
    case.update(more)
    if kind == "sparse":
        case["bounds"] = True
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # single-stream decode of a 4096-wide layer: launch latency and host time are what counts
        _case("append", 1, 32, 8, 128, 16, "f16", 1000, 1000, name="append_b1"),
        # a full decode batch of an 8192-wide layer whose cache keeps page bounds
        _case("append", 128, 64, 8, 128, 64, "bf16", 1, 2048, name="append_b128_bounds", bounds=True),
        # prompts of 1 to 4096 tokens in one call, some behind what is cached already, neighbouring channels paired
        _case("append", 24, 64, 8, 128, 32, "f16", 0, 700, name="append_prompts", new=4096, bounds=True, interleaved=True),
        # the first tokens of a single-stream chat, one kv head per query head
        _case("attend", 1, 32, 32, 128, 16, "f16", 77, 77, name="attend_b1_short"),
        # an ordinary decode batch of a 4096-wide layer, with the logarithms of the sums
        _case("attend", 16, 32, 8, 128, 16, "f16", 500, 4001, name="attend_b16", lse=True),
        # one sequence with a very long context
        _case("attend", 1, 64, 8, 128, 64, "bf16", 131071, 131071, name="attend_b1_long"),
        # ragged: one to 16384 tokens, and sequences without any
        _case("attend", 128, 64, 8, 128, 32, "f16", 1, 16384, name="attend_ragged_b128", zeros=True),
        # wide heads that share two kv heads
        _case("attend", 20, 16, 2, 256, 128, "bf16", 100, 9001, name="attend_d256_b20"),
        # the largest: a full batch of long contexts
        _case("attend", 64, 64, 8, 128, 64, "f16", 32768, 32768, name="attend_b64_long"),
        # append and attention, as a decode step of narrow heads runs them
        _case("step", 32, 40, 40, 64, 16, "bf16", 1, 2500, name="step_b32_d64"),
        # a long context read through its 64 best pages, and a ragged batch of them
        _case("sparse", 1, 32, 8, 128, 16, "f16", 65001, 65001, name="sparse_b1_long", select=64),
        _case("sparse", 32, 64, 8, 128, 32, "bf16", 300, 60000, name="sparse_b32", select=64),
    ]


def _log(rng, lo, hi):
    return round(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def draw(rng):
    while True:
        kind = rng.choices(["append", "prompts", "attend", "step", "sparse"], [15, 15, 40, 10, 20])[0]
        D = rng.choice([64, 96, 128, 128, 128, 256])
        hkv = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
        hq = hkv * rng.choice([g for g in (1, 2, 4, 5, 8, 12, 16, 32) if hkv * g <= 128])
        ps, dtype = rng.choice([16, 32, 64, 128, 256]), rng.choice(["f16", "bf16"])
        more = {"interleaved": rng.random() < 0.3, "bounds": rng.random() < 0.5, "zeros": rng.random() < 0.25,
                "rot": rng.choice([D, D, D // 2])}
        if kind == "prompts":
            B = _log(rng, 1, 64)
            case = _case("append", B, hq, hkv, D, ps, dtype, 0, rng.randint(0, 2000), new=_log(rng, 2, 8192), **more)
            if 4 * sum(_new(case)) * (hq + 2 * hkv) * D > 2 ** 31:
                continue
        else:
            B = _log(rng, 1, 256)
            lo = _log(rng, 1, 8192)
            hi = max(lo, _log(rng, 16, 131072))
            if kind == "attend":
                more["lse"] = rng.random() < 0.5
            if kind == "sparse":
                more["select"] = _log(rng, 2, 256)
                more["zeros"] = False
            case = _case(kind, B, hq, hkv, D, ps, dtype, lo, hi, **more)
        if 4 * sum(_lengths(case)) * hkv * D <= MAX_KV_BYTES // (8 if kind in ("append", "prompts") else 1) and \
                B * _width(case) * ps * hkv * D * 4 <= MAX_KV_BYTES:
            return case


# ---- what a case's sequences are ----

def _spread(lo, hi, n):
    """n lengths from lo to hi, spread over their logarithm; the last is hi."""
    a, b = math.log(lo + 1), math.log(hi + 1)
    return [round(math.exp(b if n == 1 else a + (b - a) * i / (n - 1))) - 1 for i in range(n)]


def _new(case):
    """New tokens of each sequence."""
    return [1] * case["B"] if case["new"] == 1 else [max(1, n) for n in _spread(1, case["new"], case["B"])]


def _lengths(case):
    """Tokens of each sequence, the new ones included."""
    got = _spread(case["lo"], case["hi"], case["B"])
    if case["new"] > 1:  # every other prompt is the sequence's first; the others follow a cached one
        return [n + (p if i % 2 else 0) for i, (p, n) in enumerate(zip(got, _new(case)))]
    got = [max(1, n) for n in got]
    return [0 if case["zeros"] and i % 8 == 3 else n for i, n in enumerate(got)]


def _width(case):
    """Pages a sequence's row of the table has room for."""
    return max(1, max(-(-n // case["ps"]) for n in _lengths(case)))


def work(case):
    B, hq, hkv, D, ps = (case[k] for k in ("B", "hq", "hkv", "D", "ps"))
    lengths, new = _lengths(case), _new(case)
    pages = [-(-n // ps) for n in lengths]
    tokens = sum(n for n, m in zip(new, lengths) if m)
    nbytes = flops = 0
    if case["kind"] in ("append", "step"):
        nbytes += 2 * tokens * 2 * (hq + 2 * hkv) * D + 4 * tokens * case["rot"] + 8 * B
        flops += 3 * tokens * (hq + hkv) * case["rot"]
        if case["bounds"]:
            first = [(m - n) // ps for n, m in zip(new, lengths) if m]
            nbytes += sum((m - 1) // ps - f + 1 for f, m in zip(first, (m for m in lengths if m))) * 2 * hkv * 2 * D * 2
    if case["kind"] == "sparse":
        nbytes += sum(pages) * hkv * 2 * D * 2 + 4 * sum(pages) + 2 * B * hq * D
        flops += sum(pages) * hq * 4 * D
        short = [(min(case["select"], p) - 1) * ps + (n - 1) % ps + 1 for n, p in zip(lengths, pages)]
        nbytes += sum(short) * hkv * D * 4 + 2 * B * hq * D
        flops += sum(short) * hq * 4 * D
    if case["kind"] in ("attend", "step"):
        nbytes += sum(lengths) * hkv * D * 4 + 4 * sum(pages) + 4 * B + 2 * B * hq * D * 2 + (4 * B * hq if case["lse"] else 0)
        flops += sum(lengths) * hq * 4 * D
    return {"bytes": nbytes, "flops": flops}


# ---- inputs ----

def prepare(case, seed):
    B, hq, hkv, D, ps = (case[k] for k in ("B", "hq", "hkv", "D", "ps"))
    dt, dev = DTYPES[case["dtype"]], "cuda"
    g = torch.Generator(device=dev).manual_seed(int(seed))
    order = random.Random(int(seed))

    def randn(*shape):
        return torch.randn(shape, dtype=dt, device=dev, generator=g)

    rows = list(zip(_lengths(case), _new(case)))
    order.shuffle(rows)
    lengths, new = [r[0] for r in rows], [r[1] for r in rows]
    used = [-(-n // ps) for n in lengths]
    pages, width = sum(used) + 3, _width(case)
    at = torch.randperm(pages, device=dev, generator=g)[:sum(used)].to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    n_used = torch.tensor(used, device=dev)
    table[torch.arange(width, device=dev) < n_used[:, None]] = at

    loud = 1 + 3 * (torch.rand(D, device=dev, generator=g) < 0.05).to(dt)  # some key channels are larger
    k_cache, v_cache = randn(pages, hkv, ps, D), randn(pages, hkv, ps, D)
    if case["kind"] != "sparse":
        k_cache *= loud
    v_cache += 0.5 * randn(D)
    state = {"case": case, "k_cache": k_cache, "v_cache": v_cache, "table": table,
             "lengths": torch.tensor(lengths, dtype=torch.int32, device=dev), "bounds": None}
    tokens = sum(new)
    if case["kind"] == "append" and tokens > B:
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        state["starts"] = torch.tensor(starts, dtype=torch.int32, device=dev)
    if case["kind"] in ("append", "step"):
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
    elif case["kind"] == "attend":
        state["q"] = randn(B, hq, D)
    else:  # the heads of a group look for one thing each sequence's planted pages hold
        look = randn(B, hkv, D)
        state["q"] = (look[:, :, None] + 0.5 * randn(B, hkv, hq // hkv, D)).reshape(B, hq, D)
        plant = torch.rand((B, hkv, width), device=dev, generator=g)
        share = (case["select"] / 2 / n_used.clamp(min=1)).clamp(max=0.5)
        plant = (plant < share[:, None, None]) & (torch.arange(width, device=dev) < n_used[:, None])[:, None]
        b, h, p = plant.nonzero(as_tuple=True)
        strength = 7 / math.sqrt(D) + 5 / math.sqrt(D) * torch.rand((len(b), ps, 1), device=dev, generator=g)
        where = table[b, p].long()
        k_cache[where, h] = (k_cache[where, h] + strength * look[b, h][:, None]).to(dt)
    if case["bounds"]:
        b, p = (table >= 0).nonzero(as_tuple=True)
        # appending: of what is cached before the new tokens come; a page that has nothing yet holds an older page's
        have = torch.tensor([n - m if "k" in state else n for n, m in zip(lengths, new)], device=dev)
        state["bounds"] = randn(pages, hkv, 2, D)
        state["bounds"][table[b, p].long()] = _bounds(k_cache, table[b, p].long(), have[b] - p * ps)
    return state


def _bounds(k_cache, pages, valid):
    """[pages, kv heads, 2, head dim]: smallest and largest key of each page's first `valid` slots."""
    keys = k_cache[pages]
    off = torch.arange(k_cache.shape[2], device=keys.device) >= valid.clamp(min=1)[:, None]
    off = off[:, None, :, None]
    return torch.stack([keys.masked_fill(off, math.inf).amin(2), keys.masked_fill(off, -math.inf).amax(2)], 2)


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


def _plain_append(state):
    case, k_cache, v_cache = state["case"], state["k_cache"], state["v_cache"]
    q, k, v, table, lengths = (state[n] for n in ("q", "k", "v", "table", "lengths"))
    ps, dt = case["ps"], k_cache.dtype
    T, B = q.shape[0], lengths.shape[0]
    token = torch.arange(T, device=q.device)
    if "starts" in state:
        seq = torch.searchsorted(state["starts"][1:], token, right=True)
        pos = lengths[seq] - state["starts"][seq + 1] + token
    else:
        seq, pos = token, lengths - 1
    ok = pos >= 0  # a sequence without tokens takes none; its query is zero
    pos = pos.clamp(min=0).long()
    cs = state["cos_sin"][pos]
    q_out = _rotate(q.float(), cs, case["rot"], case["interleaved"]).masked_fill(~ok[:, None, None], 0).to(dt)
    k_new = _rotate(k.float(), cs, case["rot"], case["interleaved"]).to(dt)
    seq, pos, k_new, v_new = seq[ok], pos[ok], k_new[ok], v[ok]
    page = table[seq, pos // ps].long()
    k_cache[page, :, pos % ps] = k_new
    v_cache[page, :, pos % ps] = v_new
    if state["bounds"] is None:
        return q_out, k_cache, v_cache
    left = lengths[seq] - pos // ps * ps
    state["bounds"][page] = _bounds(k_cache, page, left) if "starts" not in state else \
        _bounds_of_touched(state, page, left)
    return q_out, k_cache, v_cache, state["bounds"]


def _bounds_of_touched(state, page, left):
    """As many tokens of a prompt share a page, each page is looked at once."""
    pages, at = torch.unique(page, return_inverse=True)
    first = torch.zeros(len(pages), dtype=left.dtype, device=left.device).scatter_(0, at, left)
    return _bounds(state["k_cache"], pages, first)[at]


def _plain_attend(q, k_cache, v_cache, table, lengths, lse):
    B, hq, D = q.shape
    hkv = k_cache.shape[1]
    if table.dim() == 2:
        table = table[:, None].expand(-1, hkv, -1)
    head = torch.arange(hkv, device=q.device)[:, None]
    at = table.clamp(min=0).long()
    n = at.shape[2] * k_cache.shape[2]
    keys = k_cache[at, head].view(B * hkv, n, D).float()
    s = torch.matmul(q.float().view(B * hkv, hq // hkv, D), keys.transpose(1, 2)).view(B, hq, n) / math.sqrt(D)
    del keys
    s = s.masked_fill(torch.arange(n, device=q.device) >= lengths[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m.clamp(min=-1e30))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B * hkv, hq // hkv, n), v_cache[at, head].view(B * hkv, n, D).float()).view(B, hq, D)
    o = torch.where(total > 0, o / total, 0).to(q.dtype)
    return (o, (m + torch.log(total)).squeeze(-1)) if lse else o


def _plain_select(q, bounds, table, lengths, ps, select):
    B, hq, D = q.shape
    hkv = bounds.shape[1]
    pages = (lengths + ps - 1) // ps
    box = bounds[table.clamp(min=0).long()].float().permute(0, 2, 4, 3, 1)  # [B, kv heads, D, 2, pages]
    qf = q.float().view(B, hkv, hq // hkv, D)
    score = torch.matmul(qf.clamp(min=0), box[:, :, :, 1].contiguous()) + torch.matmul(qf.clamp(max=0), box[:, :, :, 0].contiguous())
    score = score.amax(2)
    i = torch.arange(table.shape[1], device=q.device)
    score = score.masked_fill(i == pages[:, None, None] - 1, math.inf).masked_fill(i >= pages[:, None, None], -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :select].sort(-1).values
    chosen = torch.gather(table[:, None].expand(-1, hkv, -1), 2, best)
    return chosen, torch.where(pages > select, lengths - (pages - select) * ps, lengths)


def run(state):
    case, q = state["case"], state["q"]
    k_cache, v_cache, table, lengths = (state[n] for n in ("k_cache", "v_cache", "table", "lengths"))
    kind, lse = case["kind"], case["lse"]
    if own:
        import paper_2408_11743_amd as mk
        if kind in ("append", "step"):
            q = mk.kv_append(q, state["k"], state["v"], k_cache, v_cache, table, lengths, cos_sin=state["cos_sin"],
                             starts=state.get("starts"), interleaved=case["interleaved"], bounds=state["bounds"])
            if kind == "append":
                return [q, k_cache, v_cache] + ([] if state["bounds"] is None else [state["bounds"]])
        if kind == "sparse":
            table, lengths = mk.select_pages(q, state["bounds"], table, lengths, case["ps"], case["select"])
        o = mk.paged_attention(q, k_cache, v_cache, table, lengths, return_lse=lse)
    else:
        if kind in ("append", "step"):
            got = _plain_append(state)
            if kind == "append":
                return list(got)
            q = got[0]
        if kind == "sparse":
            table, lengths = _plain_select(q, state["bounds"], table, lengths, case["ps"], case["select"])
        o = _plain_attend(q, k_cache, v_cache, table, lengths, lse)
    if kind == "sparse":
        return [o, lengths]
    if kind == "step":
        return [o, q, k_cache, v_cache] + ([] if state["bounds"] is None else [state["bounds"]])
    return list(o) if lse else [o]


# ---- the definitions in 64 bits, sequence by sequence ----

def exact(case, seed):
    s = prepare(case, seed)
    hq, hkv, D, ps, rot = (case[k] for k in ("hq", "hkv", "D", "ps", "rot"))
    dev = s["q"].device
    lengths, q = s["lengths"].tolist(), s["q"].double()
    kind = case["kind"]
    out = []
    if kind in ("append", "step"):
        if s["k_cache"].numel() * 16 > 6 << 30 and kind == "append":
            return None
        starts = s["starts"].tolist() if "starts" in s else list(range(len(lengths) + 1))
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        bounds = None if s["bounds"] is None else s["bounds"].double()
        q_out = torch.zeros_like(q)
        half = rot // 2
        j = torch.arange(half, device=dev)
        ia, ib = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + half)
        for b, n in enumerate(lengths):
            t = torch.arange(starts[b], starts[b + 1], device=dev)
            if n == 0:
                continue
            pos = t - starts[b + 1] + n
            w = torch.complex(s["cos_sin"][pos, :half].double(), s["cos_sin"][pos, half:].double())[:, None]
            for x, y in ((q[t], q_out), (s["k"][t].double(), None)):
                z = torch.complex(x[..., ia], x[..., ib]) * w
                x = x.clone()
                x[..., ia], x[..., ib] = z.real, z.imag
                if y is not None:
                    y[t] = x
            at = s["table"][b, pos // ps].long()
            kc[at, :, pos % ps], vc[at, :, pos % ps] = x, s["v"][t].double()
            if bounds is not None:
                for p in range(int(pos[0]) // ps, (n - 1) // ps + 1):
                    keys = kc[s["table"][b, p], :, :min(ps, n - p * ps)]
                    bounds[s["table"][b, p]] = torch.stack([keys.amin(1), keys.amax(1)], 1)
        out, q = [q_out, kc, vc] + ([] if bounds is None else [bounds]), q_out
        if kind == "append":
            return out
        s["k_cache"], s["v_cache"] = kc, vc
    o = torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=dev)
    for b, n in enumerate(lengths):
        used = -(-n // ps)
        pages = s["table"][b, :used].long()
        for h in range(hkv):
            if n == 0:
                continue
            mine, heads = pages, slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            left = n - (used - 1) * ps
            if kind == "sparse" and used > case["select"]:
                lo, hi = s["bounds"][pages, h].double().unbind(1)
                x = q[b, heads][:, None]
                score = torch.where(x > 0, x * hi, x * lo).sum(-1).amax(0)
                score[-1] = math.inf
                mine = pages[torch.topk(score, case["select"]).indices.sort().values]
            total = (len(mine) - 1) * ps + left
            keys = s["k_cache"][mine, h].reshape(-1, D)[:total].double()
            values = s["v_cache"][mine, h].reshape(-1, D)[:total].double()
            logits = torch.mm(q[b, heads], keys.t().contiguous()) * D ** -0.5
            o[b, heads] = torch.mm(torch.softmax(logits, -1), values)
            lse[b, heads] = torch.logsumexp(logits, -1)
    if kind == "step":
        return [o] + out
    return [o, None] if kind == "sparse" else [o, lse] if case["lse"] else [o]

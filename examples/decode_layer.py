"""One attention layer of a served model: 4-bit projections, the paged key-value
cache between them, prompts and then decode steps as a HIP graph.

    python examples/decode_layer.py [--sequences 16] [--steps 32] [--select 64 | --bits 8 --window 256 --sinks 4]

The layer's qkv projection is one 4-bit matrix; its output rows are handed to
``kv_append`` as they lie (q, k and v are slices), which rotates them and
fills the pages, which ``assign_pages`` has given to the sequences.  The prompts attend
by ``cache_attention``; a decode step is pages, projection, append, attention, projection.  With
--select the attention reads the most promising pages only, with --bits 8 the cache is in 8 bits, and with --window
a token sees the last ones and --sinks first ones, and pages behind them go to other tokens.  The graph is
captured once: tables and lengths live on the device, so its replays follow the
sequences as they grow, and pass over one that there are no pages for.  Weights and prompts are random.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2408_11743_amd as mk  # noqa: E402


class Attention(torch.nn.Module):
    def __init__(self, hidden, heads, kv_heads, head_dim, positions, generator):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim

        def linear(n_out, n_in):
            w = torch.randn(n_out, n_in, device="cuda", generator=generator) / n_in ** 0.5
            return mk.MarlinLinear.from_float(w.half(), ratios=(1.0,))
        self.qkv = linear((heads + 2 * kv_heads) * head_dim, hidden)
        self.out = linear(hidden, heads * head_dim)
        self.register_buffer("cos_sin", mk.rotation_table(positions, head_dim))

    def forward(self, x, cache, starts=None, lengths=None, select=0):
        """x [tokens, hidden]: with ``starts`` each sequence's new tokens, or one of every sequence, but those with a 0 in ``lengths``."""
        k_cache, v_cache, extra = cache["pages"]  # scales in 8 bits, else bounds
        seen = dict(window=cache["window"], sinks=cache["sinks"])
        table, eight = cache["table"], k_cache.dtype == torch.float8_e4m3fn
        lengths = cache["lengths"] if lengths is None else lengths
        rows = self.qkv(x).view(x.shape[0], -1, self.head_dim)
        q, k, v = rows.split([self.heads, self.kv_heads, self.kv_heads], 1)
        if eight:
            q = mk.kv_append8(q, k, v, k_cache, v_cache, extra, table, lengths, self.cos_sin, starts=starts)
        else:
            q = mk.kv_append(q, k, v, k_cache, v_cache, table, lengths, self.cos_sin, starts=starts, bounds=extra)
        if select and starts is None:
            table, lengths = mk.select_pages(q, extra, table, lengths, k_cache.shape[2], select)
            o = mk.paged_attention(q, k_cache, v_cache, table, lengths)
        else:
            o = mk.cache_attention(q, k_cache, v_cache, table, lengths, scales=extra if eight else None, starts=starts, **seen)
        return self.out(o.flatten(1))


def make_cache(sequences, room, page_size, kv_heads, head_dim, bits=16, window=None, sinks=0):
    """Pages for `room` tokens of each sequence, all of them free."""
    width = -(-room // page_size)
    pages = sequences * width
    made = (mk.kv_cache8(pages, kv_heads, page_size, head_dim) if bits == 8 else
            mk.kv_cache(pages, kv_heads, page_size, head_dim, bounds=True))

    def ints(*shape, value=0):
        return torch.full(shape, value, dtype=torch.int32, device="cuda")
    return {"pages": made, "table": ints(sequences, width, value=-1), "lengths": ints(sequences), "window": window, "sinks": sinks,
            "free": torch.arange(pages, dtype=torch.int32, device="cuda"), "free_count": ints(1, value=pages)}


def give_pages(cache, new, tokens):
    """To ``new[b]`` tokens of every sequence, ``tokens`` in all; returns the tokens' first rows."""
    return mk.assign_pages(cache["table"], cache["lengths"], new, cache["free"], cache["free_count"], cache["pages"][0].shape[2], tokens,
                           cache["window"], cache["sinks"])[0]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("sequences", 16),
                        ("prompt", 1000), ("steps", 32), ("page-size", 16), ("select", 0), ("bits", 16), ("window", 0), ("sinks", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    if a.bits not in (8, 16) or (a.select and (a.bits == 8 or a.window)):
        ap.error("--bits is 8 or 16, and --select goes with neither 8 bits nor a window")
    g = torch.Generator(device="cuda").manual_seed(0)
    room = a.prompt + a.steps + 8
    layer = Attention(a.hidden, a.heads, a.kv_heads, a.head_dim, room, g)
    cache = make_cache(a.sequences, room, a.page_size, a.kv_heads, a.head_dim, a.bits, a.window or None, a.sinks)

    # prompts of different lengths, one after another in the rows of x
    new = torch.linspace(max(1, a.prompt // 4), a.prompt, a.sequences).int()
    tokens = int(new.sum())
    starts = give_pages(cache, new.cuda(), tokens)
    x = layer(torch.randn(tokens, a.hidden, device="cuda", generator=g).half(), cache, starts)
    x = x[(starts[1:] - 1).long()]  # the last tokens'

    # a step adds a token to every sequence; the layer's output is the next step's input
    one = torch.ones_like(cache["lengths"])

    def step():
        starts = give_pages(cache, one, a.sequences)
        lengths = torch.where(starts[1:] > starts[:-1], cache["lengths"], 0)  # of those that got pages
        x.copy_(torch.nn.functional.normalize(layer(x, cache, lengths=lengths, select=a.select).float(), dim=1).mul_(a.hidden ** 0.5))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()  # makes the stream's workspace
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()

    # the first replay against the same step run eagerly
    state = [x] + [cache[name] for name in ("table", "lengths", "free", "free_count")]
    before = [y.clone() for y in state]
    graph.replay()
    replayed = x.clone()
    for y, old in zip(state, before):
        y.copy_(old)
    step()
    same = torch.equal(x, replayed)

    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
    torch.cuda.synchronize()
    us = (time.perf_counter() - t) / a.steps * 1e6
    print("%d sequences of %d to %d tokens: %.1f us a step, replayed and eager steps %s" % (
        a.sequences, int(cache["lengths"].min()), int(cache["lengths"].max()), us, "agree" if same else "DIFFER"), flush=True)
    return same and bool(torch.isfinite(x).all())


if __name__ == "__main__":
    sys.exit(0 if main() else 1)

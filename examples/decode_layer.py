"""One attention layer of a served model: 4-bit projections, the paged key-value
cache between them, prompts and then decode steps as a HIP graph.

    python examples/decode_layer.py [--sequences 16] [--steps 32] [--select 64]

The layer's qkv projection is one 4-bit matrix; its output rows are handed to
``kv_append`` as they lie (q, k and v are slices), which rotates them and
fills the pages.  A decode step is projection, append, attention, projection; with
--select the attention reads the most promising pages only.  The graph is
captured once: the lengths live on the device, so its replays follow the
sequences as they grow.  Weights and prompts are random.
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

    def forward(self, x, cache, starts=None, select=0):
        """x [tokens, hidden]: one new token per sequence, or with ``starts`` prompts, of which the last
        token's output is returned."""
        k_cache, v_cache, bounds = cache["pages"]
        rows = self.qkv(x).view(x.shape[0], -1, self.head_dim)
        q, k, v = rows.split([self.heads, self.kv_heads, self.kv_heads], 1)
        q = mk.kv_append(q, k, v, k_cache, v_cache, cache["table"], cache["lengths"], self.cos_sin, starts=starts,
                         bounds=bounds)
        if starts is not None:
            q = q[(starts[1:] - 1).long()]
        table, lengths = cache["table"], cache["lengths"]
        if select:
            table, lengths = mk.select_pages(q, bounds, table, lengths, k_cache.shape[2], select)
        o = mk.paged_attention(q, k_cache, v_cache, table, lengths)
        return self.out(o.flatten(1))


def make_cache(sequences, room, page_size, kv_heads, head_dim):
    """Pages for `room` tokens of each sequence, dealt out in turn."""
    width = -(-room // page_size)
    table = torch.arange(sequences * width, dtype=torch.int32, device="cuda").view(width, sequences).t().contiguous()
    return {"pages": mk.kv_cache(sequences * width, kv_heads, page_size, head_dim, bounds=True), "table": table,
            "lengths": torch.zeros(sequences, dtype=torch.int32, device="cuda")}


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("hidden", 4096), ("heads", 32), ("kv-heads", 8), ("head-dim", 128), ("sequences", 16),
                        ("prompt", 1000), ("steps", 32), ("page-size", 16), ("select", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    room = a.prompt + a.steps + 8
    layer = Attention(a.hidden, a.heads, a.kv_heads, a.head_dim, room, g)
    cache = make_cache(a.sequences, room, a.page_size, a.kv_heads, a.head_dim)

    # prompts of different lengths, one after another in the rows of x
    new = torch.linspace(max(1, a.prompt // 4), a.prompt, a.sequences).int()
    starts = torch.cat([new.new_zeros(1), new.cumsum(0, dtype=torch.int32)]).cuda()
    cache["lengths"] += new.cuda()
    x = layer(torch.randn(int(new.sum()), a.hidden, device="cuda", generator=g).half(), cache, starts)

    # a step adds a token to every sequence; the layer's output is the next step's input
    def step():
        cache["lengths"].add_(1)
        x.copy_(torch.nn.functional.normalize(layer(x, cache, select=a.select).float(), dim=1).mul_(a.hidden ** 0.5))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()  # makes the stream's workspace
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()

    # the first replay against the same step run eagerly
    before = x.clone(), cache["lengths"].clone()
    graph.replay()
    replayed = x.clone()
    x.copy_(before[0])
    cache["lengths"].copy_(before[1])
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

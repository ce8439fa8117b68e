"""Long-running streams served by the stream operators together: glue only.

A pool that drains leaves few sequences that answer for long: their layers look through a window with sinks, what falls
behind it is given up, a prompt that is answered several ways is forked, and the step is bound by its weights, kept in
four bits (or in eight, which many rows multiply faster), and by its cache, which may be kept in four bits too.  `Streams`
runs the attention half of such layers (x + Wo attention(rope(Wqkv x)), without norms) over one tensor of pools and one book
of pages:

    extend -> copy_pages -> window_plan -> for every layer: w4_linear, rope_append, window_attention, w4_linear -> trim
                                                            (w8_linear)                               (w8_linear)

    python -m paper_2411_16102_amd.streams [--prompts 2 --answers 4 --prompt-tokens 3000 --tokens 32 --layers 8]
                                           [--cache-group 64] [--weight-bits 8]
"""
from __future__ import annotations

import argparse
from typing import Sequence

import numpy as np

from . import workloads as W
from .binding import W8Rows, W8Weight


class Streams:
    """Sequences over `n_pages` pages of every layer, each of up to the layer's max_positions tokens (positions count from a sequence's
    first token).  weights: (Wqkv, Wo) of each layer, from Layer.w4_pack or in 8-bit integers (W8Weight, or what Layer.w8_quantize
    gives).  cache: Kv4(group) for pages in four bits."""

    def __init__(self, api, layer, weights, n_pages: int, window: int, sinks: int, cache=None):
        import torch
        self.torch, self.layer, self.weights, self.cache = torch, layer, list(weights), cache
        self.window, self.sinks = window, sinks
        self.pages = api.Pages(n_pages)
        size, kind = (layer.page_bytes() // 2, torch.bfloat16) if cache is None else (layer.page_bytes(cache), torch.uint8)
        self.pools = torch.zeros((len(self.weights), n_pages * size), device="cuda:%d" % layer.device, dtype=kind)
        self.plan = None

    def batch(self, ids, rows) -> W.Batch:
        """The step in which sequence ids[i] has rows[i] rows at its end (their room is there already)."""
        start, pages = self.pages.tables(ids)
        none, n = np.zeros(0, dtype=np.int32), len(ids)
        return W.Batch(page_size=16, n_seq=n, n_prefill=0, n_rows=int(np.sum(rows)), row_start=np.concatenate([[0], np.cumsum(rows)]).astype(np.int32),
                       kv_len=self.pages.lengths(ids).astype(np.int32), page_start=start, page_ids=pages, n_nodes=0, node_parent=none,
                       node_page_start=np.zeros(1, dtype=np.int32), node_page_ids=none, node_seq_first=none, node_seq_count=none,
                       seq_leaf_node=np.full(n, -1, dtype=np.int32), n_pages=self.pages.n_pages)

    def linear(self, x, weight):
        return self.layer.w8_linear(x, weight) if isinstance(weight, W8Rows) else self.layer.w4_linear(x, weight)

    def step(self, ids: Sequence[int], rows: Sequence[int], x):
        """x: bf16 [sum(rows), d_model], the rows of ids[0] first.  What the layers make of it, [sum(rows), d_model]."""
        lay = self.layer
        src, dst = self.pages.extend(ids, rows)
        lay.copy_pages(self.pools, src, dst, cache=self.cache)
        batch = self.batch(ids, rows)
        if self.plan is None:
            self.plan = lay.window_plan(batch, self.window, self.sinks, cache=self.cache)
        else:
            self.plan.update(batch, self.window, self.sinks)
        x = self.layers(x)
        self.pages.trim(ids, self.window, self.sinks)
        return x

    def layers(self, x):
        """The planned step's layers."""
        lay = self.layer
        for (w_qkv, w_o), pool in zip(self.weights, self.pools):
            q = lay.rope_append(self.plan, self.linear(x, w_qkv), pool)
            x = x + self.linear(lay.window_attention(self.plan, q, pool, out=q), w_o)
        return x

    def compact(self) -> int:
        """Moves the live pages to the front of every pool; how many there are."""
        src, dst, live = self.pages.compact()
        self.layer.copy_pages(self.pools, src, dst, cache=self.cache)
        return live


def synthetic_weights(layer, n_layers: int, group: int = 128, seed: int = 0, bits: int = 4):
    """Seeded weights (Wqkv, Wo) of unit gain for each layer, in 4 bits, laid out, or in 8."""
    import torch
    dev, gen = "cuda:%d" % layer.device, torch.Generator(device="cuda:%d" % layer.device).manual_seed(seed)
    s, out = layer.shape, []
    wide = s.n_q_heads * s.head_dim
    for _ in range(n_layers):
        pair = []
        for n, k in ((s.n_qkv, s.d_model), (s.d_model, wide)):
            if bits == 8:
                q = torch.randint(-127, 128, (n, k), dtype=torch.int8, device=dev, generator=gen)
                pair.append(W8Weight(q, torch.full((n,), (k * 5418.0) ** -0.5, device=dev)))  # (-127 .. 127 has a variance of 5418 nearly)
                continue
            packed = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device=dev, generator=gen)
            scales = torch.full((n, k // group), (k * 21.25) ** -0.5, dtype=torch.bfloat16, device=dev)  # (0 .. 15 has a variance of 21.25)
            zeros = torch.randint(7, 9, (n, k // group), dtype=torch.uint8, device=dev, generator=gen)
            pair.append(layer.w4_pack(packed, scales, zeros))
        out.append(tuple(pair))
    return out


def main(argv=None):
    import torch

    from . import load
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("prompts", 2), ("answers", 4), ("prompt-tokens", 3000), ("tokens", 32), ("layers", 8), ("window", 1024), ("sinks", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache-group", type=int, choices=(32, 64, 128), help="a cache in four bits, with two numbers for so many channels")
    ap.add_argument("--weight-bits", type=int, default=4, choices=(4, 8))
    a = ap.parse_args(argv)
    api = load()
    shape = W.LLAMA3_8B
    layer = api.Layer(shape, device=0)
    n_pages = a.prompts * (-(-a.prompt_tokens // 16) + a.answers * (-(-a.tokens // 16) + 1))
    st = Streams(api, layer, synthetic_weights(layer, a.layers, bits=a.weight_bits), n_pages, a.window, a.sinks,
                 cache=api.Kv4(a.cache_group) if a.cache_group else None)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = lambda n: torch.randn((n, shape.d_model), device="cuda", generator=gen).to(torch.bfloat16)
    prompts = st.pages.open(a.prompts)
    # the first prompt also builds whatever a first call builds
    for p in prompts:
        e0, e1 = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        e0.record()
        st.step([p], [a.prompt_tokens], rows(a.prompt_tokens))
        e1.record()
    answers = np.concatenate([prompts, st.pages.fork(prompts, a.answers - 1)])
    events, inputs = [], [rows(len(answers)) for _ in range(a.tokens)]
    for x in inputs:
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        e[0].record()
        st.step(answers, [1] * len(answers), x)
        e[1].record()
        events.append(e)
    live = st.compact()
    torch.cuda.synchronize()
    ms = sorted(b.elapsed_time(c) for b, c in events)
    print("weights in %d bits, cache in %d" % (a.weight_bits, 4 if a.cache_group else 16))
    print("prompt of %d rows, %d layers: %.3f ms" % (a.prompt_tokens, a.layers, e0.elapsed_time(e1)))
    print("step of %d rows, %d layers: %.3f ms (median of %d; %.1f us a layer)" % (len(answers), a.layers, ms[len(ms) // 2], len(ms), 1e3 * ms[len(ms) // 2] / a.layers))
    print("%d of %d pages live after compaction" % (live, n_pages))


if __name__ == "__main__":
    main()

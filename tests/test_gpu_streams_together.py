"""The stream operators run together (`paper_2411_16102_amd.streams`) against float64 layers over dense histories.

Tolerance: what a layer rounds to bf16 is its products (rows of qkv, of o), its turned queries and keys, its probabilities, its attention and
its sum, at most eight roundings on the way to an element of x, each of at most 2^-8 of what it rounds (root mean square below 2^-8 / sqrt(3)) and
of values no larger than x's own size here; over two layers sixteen of them: 4 * 2^-8 / sqrt(3) < 1e-2 of the norm."""
import numpy as np
import pytest

from oracle import stream as OS
from paper_2411_16102_amd import workloads as W

pytestmark = pytest.mark.gpu


class Dense:
    """The same layers in 64 bits; a sequence is its keys and values of every layer."""

    def __init__(self, shape, weights, window, sinks):
        self.s, self.weights, self.window, self.sinks, self.kv = shape, weights, window, sinks, {}

    def step(self, ids, rows, x):
        s, at = self.s, 0
        hq, hkv, dh = s.n_q_heads, s.n_kv_heads, s.head_dim
        axis, out = np.zeros(dh // 2, dtype=np.int64), []
        for i, n in zip(ids, rows):
            h = x[at:at + n].astype(np.float64)
            at += n
            past = self.kv.setdefault(i, [(np.zeros((0, hkv, dh)), np.zeros((0, hkv, dh))) for _ in self.weights])
            first = len(past[0][0])
            for l, (w_qkv, w_o) in enumerate(self.weights):
                qkv = OS.w4_linear(h, *w_qkv).reshape(n, -1, dh)
                turned = OS.rope_axes(qkv[:, :hq + hkv], np.arange(first, first + n)[None], axis, s.rope_theta)
                past[l] = (np.concatenate([past[l][0], turned[:, hq:]]), np.concatenate([past[l][1], qkv[:, hq + hkv:]]))
                o, _ = OS.window_attention(turned[:, :hq], past[l][0], past[l][1], first, self.window, self.sinks)
                h = h + OS.w4_linear(o.reshape(n, -1), *w_o)
            out.append(h)
        return np.concatenate(out)

    def fork(self, parent, child):
        self.kv[child] = list(self.kv[parent])


@pytest.mark.parametrize("group,window,sinks", [(64, 24, 3), (32, 1, 0), (128, 70, 20)])
def test_streams_follow_dense_layers(lib, group, window, sinks):
    import torch
    from paper_2411_16102_amd.streams import Streams
    rng = np.random.default_rng([group, window])
    shape = W.LayerShape(256, 8, 2, 64, 256)
    layer = lib.Layer(shape, device=0)
    laid, plain = [], []
    for _ in range(2):
        pair = []
        for n, k in ((shape.n_qkv, 256), (256, 512)):
            w, z = rng.integers(0, 16, (n, k)).astype(np.uint8), rng.integers(6, 10, (n, k // group)).astype(np.uint8)
            scale = W.f32_to_bf16_bits(np.full((n, k // group), (22.0 * k) ** -0.5, dtype=np.float32))
            laid.append(layer.w4_pack(torch.from_numpy(w[:, 0::2] | (w[:, 1::2] << 4)).cuda(), torch.from_numpy(scale.view(np.int16)).cuda().view(torch.bfloat16),
                                      torch.from_numpy(z).cuda()))
            pair.append((w, W.bf16_bits_to_f32(scale), z))
        plain.append(tuple(pair))
    st, ref = Streams(lib, layer, [tuple(laid[:2]), tuple(laid[2:])], 48, window, sinks), Dense(shape, plain, window, sinks)

    def step(ids, rows):
        bits = W.f32_to_bf16_bits(rng.standard_normal((int(np.sum(rows)), 256)).astype(np.float32))
        got = st.step(ids, rows, torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)).float().cpu().numpy()
        want = ref.step([int(i) for i in ids], rows, W.bf16_bits_to_f32(bits))
        assert np.isfinite(got).all()
        assert np.linalg.norm(got - want) <= 1e-2 * np.linalg.norm(want)

    prompts = st.pages.open(2)
    step(prompts, [41, 17])
    children = st.pages.fork(prompts, 2)
    for i, c in enumerate(children):
        ref.fork(int(prompts[i // 2]), int(c))
    ids = np.concatenate([prompts, children])
    for t in range(20):
        step(ids, [1 + (t + i) % 2 for i in range(len(ids))])
        if t == 9:
            st.pages.free(ids[:1])
            del ref.kv[int(ids[0])]
            ids = ids[1:]
            free = st.pages.stats()["free"]
            assert st.compact() == 48 - free
    # the pages in front of the window, but for the sinks', are given up
    start, pages = st.pages.tables(ids)
    for i, n in enumerate(st.pages.lengths(ids)):
        held = np.flatnonzero(pages[start[i]:start[i + 1]] >= 0)
        needed = {t // 16 for t in range(n) if t > n - window or t < sinks}
        assert needed <= set(held.tolist()) <= needed | {n // 16}

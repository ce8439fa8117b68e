"""Streams with weights in eight bits and a cache in four (`paper_2411_16102_amd.streams`): every operator of every layer of every step, on what it was given,
against float64 over dense histories that are kept of the same rows.

Tolerances: a product of 8-bit integers is off by its last rounding, 2^-8 of each result; one of 4-bit weights, and attention, round factors
and results, 2^-8 / 3^(1/2) twice over for errors spread evenly: 5e-3 of the norm.  Codes are the definition's but for keys at a border that another
angle's last bit moves by one: such a key is off by a scale, one among thousands of numbers that a norm is of."""
import numpy as np
import pytest

from oracle import bits as OB, stream as OS
from paper_2411_16102_amd import workloads as W

pytestmark = pytest.mark.gpu
WINDOW, SINKS = 70, 20


def _host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _near(got, want, limit):
    assert np.isfinite(got).all()
    assert np.linalg.norm(got - want) <= limit * np.linalg.norm(want), np.linalg.norm(got - want) / np.linalg.norm(want)


def make_streams(lib, shape, bits, group, n_pages, seed=0):
    """(Streams with two layers, their weights in float64 form)."""
    import torch
    from paper_2411_16102_amd.streams import Streams
    rng, layer, laid, plain = np.random.default_rng(seed), lib.Layer(shape, device=0), [], []
    wide = shape.n_q_heads * shape.head_dim
    for _ in range(2):
        pairs = []
        for n, k in ((shape.n_qkv, shape.d_model), (shape.d_model, wide)):
            if bits == 8:
                w, s = rng.integers(-127, 128, (n, k)).astype(np.int8), ((0.5 + rng.random(n)) * (5418.0 * k) ** -0.5).astype(np.float32)
                pairs.append((lib.W8Weight(torch.from_numpy(w).cuda(), torch.from_numpy(s).cuda()), (w, s)))
            else:
                w, z = rng.integers(0, 16, (n, k)).astype(np.uint8), rng.integers(6, 10, (n, k // 64)).astype(np.uint8)
                s = W.f32_to_bf16_bits(np.full((n, k // 64), (22.0 * k) ** -0.5, dtype=np.float32))
                pairs.append((layer.w4_pack(torch.from_numpy(w[:, 0::2] | (w[:, 1::2] << 4)).cuda(), torch.from_numpy(s.view(np.int16)).cuda().view(torch.bfloat16),
                                            torch.from_numpy(z).cuda()), (w, W.bf16_bits_to_f32(s), z)))
        laid.append(tuple(p[0] for p in pairs))
        plain.append(tuple(p[1] for p in pairs))
    return Streams(lib, layer, laid, n_pages, WINDOW, SINKS, cache=lib.Kv4(group) if group else None), plain


class Followed:
    """A step's layers, each operator checked on what it is given; kv[id][layer]: a sequence's keys and values as its cache keeps them."""

    def __init__(self, streams, plain, bits, group):
        self.st, self.plain, self.bits, self.group, self.kv = streams, plain, bits, group, {}

    def linear(self, x, weight, plain):
        got = self.st.linear(x, weight)
        want = OB.w8_linear(_host(x), *plain) if self.bits == 8 else OS.w4_linear(_host(x), *plain)
        _near(_host(got), want, 2.0 ** -8 if self.bits == 8 else 5e-3)
        return got

    def kept(self, v):
        bits = W.f32_to_bf16_bits(v.astype(np.float32))
        return OB.kv4_values(v.astype(np.float32), self.group)[0] if self.group else W.bf16_bits_to_f32(bits).astype(np.float64)

    def __call__(self, ids, rows, x):
        st, s = self.st, self.st.layer.shape
        hq, hkv, dh = s.n_q_heads, s.n_kv_heads, s.head_dim
        none = np.zeros((0, hkv, dh))
        for l, ((w_qkv, w_o), plain) in enumerate(zip(st.weights, self.plain)):
            qkv = self.linear(x, w_qkv, plain[0])
            q = st.layer.rope_append(st.plan, qkv, st.pools[l])
            q_host, given = _host(q), _host(qkv).reshape(len(qkv), -1, dh)
            out = st.layer.window_attention(st.plan, q, st.pools[l], out=q)
            at, turned_q, want = 0, [], []
            for i, n in zip(ids, rows):
                past = self.kv.setdefault(int(i), [(none, none) for _ in st.weights])
                first = len(past[l][0])
                part = given[at:at + n]
                turned = OS.rope_axes(part[:, :hq + hkv], np.arange(first, first + n)[None], np.zeros(dh // 2, dtype=np.int64), s.rope_theta)
                past[l] = tuple(np.concatenate([p, self.kept(v)]) for p, v in zip(past[l], (turned[:, hq:], part[:, hq + hkv:])))
                turned_q.append(turned[:, :hq].reshape(n, -1))
                want.append(OS.window_attention(q_host[at:at + n].reshape(n, hq, dh), *past[l], first, st.window, st.sinks)[0].reshape(n, -1))
                at += n
            _near(q_host, np.concatenate(turned_q), 2.0 ** -8)
            _near(_host(out), np.concatenate(want), 5e-3)
            x = x + self.linear(out, w_o, plain[1])
        return x


@pytest.mark.parametrize("bits,group,heads,dh", [(8, 32, (8, 2), 64), (8, 64, (4, 4), 64), (8, 128, (8, 2), 128), (4, 32, (6, 2), 128), (8, None, (8, 1), 64)])
def test_steps_of_streams(lib, bits, group, heads, dh):
    import torch
    shape = W.LayerShape(256, *heads, dh, 256)
    st, plain = make_streams(lib, shape, bits, group, 64)
    follow = Followed(st, plain, bits, group)
    rng = np.random.default_rng(dh)

    def step(ids, rows):
        x = torch.from_numpy(W.f32_to_bf16_bits(rng.standard_normal((int(np.sum(rows)), 256)).astype(np.float32)).view(np.int16)).cuda().view(torch.bfloat16)
        inner, st.layers = st.layers, lambda x: follow(ids, rows, x)
        try:
            st.step(ids, rows, x)
        finally:
            st.layers = inner

    prompts = st.pages.open(2)
    step(prompts, [141, 17])
    children = st.pages.fork(prompts, 2)
    for i, c in enumerate(children):
        follow.kv[int(c)] = [tuple(p) for p in follow.kv[int(prompts[i // 2])]]
    ids = np.concatenate([prompts, children])
    for t in range(12):
        step(ids, [1 + (t + i) % 3 for i in range(len(ids))])
        if t == 5:
            st.pages.free(ids[:1])
            ids = ids[1:]
            assert st.compact() == 64 - st.pages.stats()["free"]


def test_layers_in_a_graph(lib):
    # the layers of a planned step, captured: replays append the same rows to the same places
    import torch
    st, _ = make_streams(lib, W.LayerShape(256, 8, 2, 64, 256), 8, 32, 64)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = lambda n: torch.randn((n, 256), device="cuda", generator=gen).to(torch.bfloat16)
    ids = st.pages.open(3)
    st.step(ids, [90, 40, 3], rows(133))
    x = rows(6)
    st.step(ids, [1, 4, 1], x)
    want, pools = st.layers(x), st.pools.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        got = st.layers(x)
    for fresh in (None, rows(6), rows(6)):
        if fresh is not None:
            x.copy_(fresh)
            want = st.layers(x)
            pools = st.pools.clone()
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(st.pools, pools)
        assert torch.equal(st.layers(x), want)


def test_steps_on_another_stream(lib):
    import torch
    both = [make_streams(lib, W.LayerShape(256, 8, 2, 64, 256), 8, 64, 64)[0] for _ in range(2)]
    gen = torch.Generator(device="cuda").manual_seed(2)
    inputs = [torch.randn((n, 256), device="cuda", generator=gen).to(torch.bfloat16) for n in (120, 5, 2, 9, 2)]
    torch.cuda.synchronize()
    results, other = [], torch.cuda.Stream()
    for st, stream in zip(both, (torch.cuda.current_stream(), other)):
        with torch.cuda.stream(stream):
            ids = st.pages.open(2)
            results.append([st.step(ids, [len(x) - 1, 1], x) for x in inputs])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*results)) and torch.equal(both[0].pools, both[1].pools)


def test_weights_from_rows(lib):
    # weights that Layer.w8_quantize made are those of their integers
    import torch
    from paper_2411_16102_amd.streams import Streams
    layer, gen = lib.Layer(W.LayerShape(256, 8, 2, 64, 256), device=0), torch.Generator(device="cuda").manual_seed(3)
    s = layer.shape
    rows = [layer.w8_quantize((0.06 * torch.randn((n, k), device="cuda", generator=gen)).to(torch.bfloat16)) for n, k in ((s.n_qkv, 256), (256, 512))]
    both = [Streams(lib, layer, [tuple(pair)], 16, WINDOW, SINKS, cache=lib.Kv4(64)) for pair in (rows, [lib.W8Weight(r.q, r.scales) for r in rows])]
    for n in (50, 1, 4):
        x = torch.randn((n, 256), device="cuda", generator=gen).to(torch.bfloat16)
        results = []
        for st in both:
            ids = [0] if n != 50 else st.pages.open(1)
            results.append(st.step(ids, [n], x))
        assert torch.equal(*results) and torch.isfinite(results[0]).all()

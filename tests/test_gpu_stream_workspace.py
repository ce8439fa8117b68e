"""The 4-bit products and the products of the blended step share a context's partial sums and arrival counters: calls of both kinds,
in turn on one context, give bit for bit what each gives on a context of its own (their sums are added up in a fixed order)."""
import numpy as np
import pytest

from paper_2411_16102_amd import workloads as W
from stream_cases import make_batch

pytestmark = pytest.mark.gpu


def test_both_kinds_of_products_in_turn(lib):
    import torch
    from paper_2411_16102_amd import binding
    gen = torch.Generator(device="cuda").manual_seed(7)
    new = lambda *shape, std=1.0: (std * torch.randn(shape, device="cuda", generator=gen)).to(torch.bfloat16)
    s = W.LLAMA3_8B
    d, wide, f = s.d_model, s.n_q_heads * s.head_dim, s.d_ffn
    batch = make_batch([(1, 100 + 3 * i) for i in range(61)])
    keep = [new(s.n_qkv, d, std=d ** -0.5), new(d, wide, std=wide ** -0.5), new(2 * f, d, std=d ** -0.5), new(d, f, std=f ** -0.5), new(d), new(d)]
    x = new(61, d)
    a, b = new(700, 2048), new(4096, 2048)
    owner = lib.Layer(s, device=0)
    pool = new(batch.n_pages * owner.page_bytes() // 2)
    dev = binding.DeviceState(binding.Weights(*[t.data_ptr() for t in keep]), keep, x, pool, batch.n_pages)
    weights = []  # outputs shared by workgroups: tiles of 64 rows, slices of 16
    for n, k, group in ((4200, 5120, 64), (4096, 14336, 128), (1000, 8192, 32)):
        packed = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=gen)
        weights.append(owner.w4_pack(packed, new(n, k // group, std=0.02)))
    rows = [(61, 0), (4, 1), (16, 2), (30, 0)]
    inputs = [new(m, weights[i].k) for m, i in rows]

    def step(layer):
        assert layer.gemm_division("down", 61)[1] > 1 and layer.gemm_division("qkv", 61)[1] > 1
        return layer.blend_step(dev, batch)

    def shared(layer):  # tiles that workgroups share, with arrival counters
        layer.set_gemm_tiles(6)
        out = layer.gemm_nt(a, b)
        layer.set_gemm_tiles(0)
        return out

    calls = [step, shared] + [lambda layer, i=i, m=m: layer.w4_linear(inputs[m], weights[i]) for m, (_, i) in enumerate(rows)]
    want = []
    for call in calls:
        alone = lib.Layer(s, device=0)
        want.append(call(alone).clone())
        torch.cuda.synchronize()
        alone.close()
    order = np.random.default_rng(3)
    for turn in range(6):
        for i in [int(i) for i in order.permutation(len(calls))] * 2:
            assert torch.equal(calls[i](owner), want[i]), "call %d in turn %d" % (i, turn)

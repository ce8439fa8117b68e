"""The Python calls of the stream operators on the GPU: what they refuse, and where their results are allocated."""
import numpy as np
import pytest

from paper_2411_16102_amd import workloads as W
from stream_cases import make_batch

pytestmark = pytest.mark.gpu
SHAPE = W.LayerShape(256, 8, 2, 64, 256)


def test_host_tensors_are_refused(lib):
    import torch
    layer = lib.Layer(SHAPE, device=0)
    batch = make_batch([(1, 40), (3, 20)])
    plan = layer.window_plan(batch, 8)
    zeros = lambda *shape, **kw: torch.zeros(shape, dtype=torch.bfloat16, **kw)
    q, qkv, pool = zeros(4, 512), zeros(4, SHAPE.n_qkv), zeros(batch.n_pages * layer.page_bytes() // 2)
    packed, scales = torch.zeros((16, 64), dtype=torch.uint8), zeros(16, 2)
    weight = layer.w4_pack(packed.cuda(), scales.cuda())
    for call in (lambda: layer.window_attention(plan, q, pool.cuda()), lambda: layer.window_attention(plan, q.cuda(), pool),
                 lambda: layer.window_attention(plan, q.cuda(), pool.cuda(), out=q), lambda: layer.rope_append(plan, qkv, pool.cuda()),
                 lambda: layer.rope_append(plan, qkv.cuda(), pool), lambda: layer.rope_append(plan, qkv.cuda(), pool.cuda(), q=q),
                 lambda: layer.w4_pack(packed, scales.cuda()), lambda: layer.w4_pack(packed.cuda(), scales),
                 lambda: layer.w4_linear(zeros(2, 128), weight), lambda: layer.w4_linear(zeros(2, 128, device="cuda"), weight, out=zeros(2, 16)),
                 lambda: layer.copy_pages([pool], [0], [1]), lambda: layer.compact_pages([pool.cuda(), pool], [0, 2])):
        with pytest.raises(ValueError, match=" on cpu"):
            call()


def test_results_of_calls_on_another_stream(lib):
    # results that the calls allocate belong to the side stream: equal to those of the current one, and their memory
    # does not go back to the current stream's when they are dropped
    import torch
    layer = lib.Layer(SHAPE, device=0)
    batch = make_batch([(1, 3000), (200, 700), (1, 0)])
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *shape: torch.randn(shape, device="cuda", generator=gen).to(torch.bfloat16)
    pool, qkv, x = new(batch.n_pages * layer.page_bytes() // 2), new(batch.n_rows, SHAPE.n_qkv), new(40, 256)
    packed, scales = torch.randint(0, 256, (520, 128), dtype=torch.uint8, device="cuda", generator=gen), new(520, 4)
    plan = layer.window_plan(batch, 500, 4)

    def results(stream=None):
        q = layer.rope_append(plan, qkv, pool, stream=stream)
        weight = layer.w4_pack(packed, scales, stream=stream)
        return [q, layer.window_attention(plan, q, pool, stream=stream), weight.data, layer.w4_linear(x, weight, stream=stream)]

    want = results()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        got = results(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        places, sizes = [t.data_ptr() for t in got], [t.shape for t in got]
        types = [t.dtype for t in got]
        del got
        again = [torch.empty(s, dtype=d, device="cuda") for s, d in zip(sizes, types)]
        assert not set(places) & {t.data_ptr() for t in again}


def test_single_rows_and_columns_at_any_stride(lib):
    import torch
    layer = lib.Layer(SHAPE, device=0)
    batch = make_batch([(1, 300)])
    new = lambda *shape: torch.randn(shape, device="cuda").to(torch.bfloat16)
    row = lambda t: t.reshape(-1, 1).clone().t()
    pool, qkv, x = new(batch.n_pages * layer.page_bytes() // 2), new(1, SHAPE.n_qkv), new(1, 256)
    assert row(qkv).stride() == (1, 1)
    plan = layer.window_plan(batch, 100, 4)
    weight = layer.w4_pack(torch.randint(0, 256, (77, 128), dtype=torch.uint8, device="cuda"), new(77, 4))
    q = layer.rope_append(plan, qkv, pool)
    out, y = layer.window_attention(plan, q, pool), layer.w4_linear(x, weight)
    assert torch.equal(layer.rope_append(plan, row(qkv), pool, q=row(q)), q)
    mine = row(qkv)
    layer.rope_append(plan, mine, pool, q=mine[:, :512])
    assert torch.equal(mine[:, :512], q) and torch.equal(mine[:, 512:], qkv[:, 512:])
    mine = row(q)
    assert torch.equal(layer.window_attention(plan, mine, pool, out=mine), out)
    assert torch.equal(layer.w4_linear(row(x), weight, out=row(y)), y)
    one = layer.w4_pack(torch.randint(0, 256, (1, 128), dtype=torch.uint8, device="cuda"), new(1, 4))
    xs, ys = new(5, 256), torch.zeros((1, 5), dtype=torch.bfloat16, device="cuda")
    assert torch.equal(layer.w4_linear(xs, one, out=ys.t()), layer.w4_linear(xs, one))

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

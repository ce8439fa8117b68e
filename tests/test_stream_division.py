"""How planned steps of streams are divided (host only): the kernels' paths that a batch takes, by its lengths."""
import numpy as np
import pytest

from paper_2411_16102_amd import binding, workloads as W
from stream_cases import make_batch

WHOLE = 1 << 30  # a window that sees everything: a stream's pages are its length's


def streams(*runs):
    """(how many, pages) each; the last pages are not all full."""
    return make_batch([(1, 16 * pages - i % 7) for n, pages in runs for i in range(n)])


# KV heads, streams, wavefronts that share a unit's pages, whether units are cut and joined: every kernel of single tokens
SHARED = [(8, [(200, 12)], 1, False), (8, [(255, 4), (1, 200)], 1, True), (4, [(100, 33)], 2, False), (1, [(1, 400)], 2, True),
          (1, [(250, 66)], 4, False), (1, [(32, 400)], 4, True), (1, [(200, 130)], 8, False), (1, [(48, 600)], 8, True)]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("hkv,runs,waves,cut", SHARED)
def test_wavefronts_of_a_unit(hkv, runs, waves, cut, dh):
    layer = binding.Layer(W.LayerShape(256, 2 * hkv, hkv, dh, 256), device=-1)
    d = layer.window_plan(streams(*runs), WHOLE).division()
    assert (d.waves, d.split_rows > 0, d.wide_blocks) == (waves, cut, 0)


@pytest.mark.parametrize("hkv,dh,runs,cut", [
    # one old stream among many young ones: whole it would outlast them all
    (8, 128, [(255, 4), (1, 100)], True), (8, 64, [(255, 4), (1, 100)], True), (8, 128, [(255, 32), (1, 256)], True), (8, 64, [(255, 32), (1, 256)], True),
    (16, 128, [(255, 4), (1, 200)], True), (8, 128, [(255, 64), (1, 512)], True), (8, 128, [(511, 8), (1, 256)], True),
    # batches of equal streams fill the chip whole, and so do those whose longest ends with the others
    (8, 128, [(256, 64)], False), (8, 64, [(256, 64)], False), (8, 128, [(512, 16)], False), (8, 128, [(128, 64), (128, 40)], False)])
def test_long_streams_among_many(hkv, dh, runs, cut):
    layer = binding.Layer(W.LayerShape(256, 2 * hkv, hkv, dh, 256), device=-1)
    d = layer.window_plan(streams(*runs), WHOLE).division()
    longest = max(pages for _, pages in runs)
    assert (d.split_rows > 0) == cut
    assert d.longest_pages <= longest // 2 if cut else d.longest_pages == longest
    if cut:
        # only streams that are longer than a unit
        assert d.split_rows <= sum(n for n, pages in runs if pages > d.longest_pages)

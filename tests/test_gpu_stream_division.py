"""Window attention on every way that single tokens are divided: wavefronts that share a unit's pages, whole and joined from memory."""
import pytest

from paper_2411_16102_amd import workloads as W
from test_gpu_stream import _attention
from test_stream_division import SHARED, WHOLE, streams

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("hkv,runs,waves,cut", SHARED)
def test_wavefronts_of_a_unit(lib, hkv, runs, waves, cut, dh):
    shape = W.LayerShape(256, 2 * hkv, hkv, dh, 256)
    _, plan, *_ = _attention(lib, shape, streams(*runs), WHOLE, 0, seed=waves)
    d = plan.division()
    assert (d.waves, d.split_rows > 0) == (waves, cut)

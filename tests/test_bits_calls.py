"""The operators of fewer bits without a GPU: their definition against other formulas, how steps and products are divided, and what is refused, by the
Python calls before the library is reached and by the library."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import bits as OB
from paper_2411_16102_amd import binding, workloads as W
from stream_cases import make_batch

SHAPE = W.LayerShape(256, 8, 2, 64, 256)
FOUR = binding.Kv4(32)


class Asked:
    """The library, but for the calls that would launch something: those are kept in `calls`."""
    NAMES = ("bs_window_attention", "bs_rope_append", "bs_kv4_pack", "bs_kv4_unpack", "bs_kv4_copy_pages", "bs_kv4_compact", "bs_kv_copy_pages", "bs_kv_compact",
             "bs_w8_quantize", "bs_w8_linear", "bs_w8_linear_rows")

    def __init__(self, lib):
        self._lib, self.calls = lib, []

    def __getattr__(self, name):
        if name not in self.NAMES:
            return getattr(self._lib, name)

        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


class Stream:
    cuda_stream = 0


@pytest.fixture(autouse=True)
def _streams_in_name(monkeypatch):
    from contextlib import nullcontext
    monkeypatch.setattr(torch.cuda, "stream", nullcontext)


def make_layer(shape=SHAPE):
    layer = binding.Layer(shape, device=-1)
    layer.lib = Asked(layer.lib)
    return layer


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def u8(n):
    return torch.zeros(n, dtype=torch.uint8)


# ---- the definitions --------------------------------------------------------------------------
def test_no_value_is_further_than_half_a_scale():
    rng = np.random.default_rng(0)
    for scale in (1.0, 1e-30, 1e30):
        v = W.round_to_bf16((scale * rng.standard_normal((500, 128)) * np.exp(rng.standard_normal((500, 1)))).astype(np.float32))
        for group in (32, 64, 128):
            s, mid = OB.kv4_numbers(v, group)
            kept, size = OB.kv4_values(v, group)
            per = np.repeat(s.astype(np.float64), group, axis=-1)
            assert (np.abs(kept - v) <= 0.5 * per * (1 + 1e-6)).all() and (size >= np.abs(kept) * (1 - 1e-12)).all()
            # and no scale is much more than it has to be: 1 / 15 of the span, mid's rounding and its own
            span = v.reshape(500, -1, group).max(-1) - v.reshape(500, -1, group).min(-1)
            assert (s <= (span / 15 + 2.0 ** -8 * np.abs(mid) / 7) * (1 + 2.0 ** -7) + 2.0 ** -126).all()


def test_what_is_kept_as_it_is():
    for value in (0.0, 3.0, -1.5, 2.0 ** -133, 3.0e38):
        v = W.round_to_bf16(np.full((1, 64), value, dtype=np.float32))
        assert (OB.kv4_values(v, 32)[0] == v).all()
    v = np.arange(-8, 8, dtype=np.float32).repeat(4)[None]     # sixteen values at equal distances
    assert (OB.kv4_values(v, 64)[0] == v).all()
    bad = v.copy()
    bad[0, 3] = np.inf
    assert np.isnan(OB.kv4_values(bad, 32)[0][0, :32]).all() and not np.isnan(OB.kv4_values(bad, 32)[0][0, 32:]).any()


def test_rows_of_integers():
    x = np.float32([[127.0, -63.5, 0.5, 1.5, 0, 0, 0, 0], [0] * 8, [1, 2, np.nan, 0, 0, 0, 0, 0], [1e-38] * 8])
    q, s = OB.w8_rows(x)
    assert s[0] == 1.0 and q[0].tolist() == [127, -64, 0, 2, 0, 0, 0, 0] and not q[1].any() and s[1] == np.float32(2.0 ** -100) / np.float32(127)
    assert np.isnan(s[2]) and not q[2].any() and not q[3].any()
    y = OB.w8_linear(x[:2], np.ones((3, 8), dtype=np.int8), np.float32([1, 2, 0]))
    np.testing.assert_array_equal(y, [[65.0, 130.0, 0.0], [0.0, 0.0, 0.0]])


# ---- sizes and plans ---------------------------------------------------------------------------
@pytest.mark.parametrize("heads,dh,group,size", [(2, 64, 64, 2 * (1024 + 128)), (2, 64, 32, 2 * (1024 + 256)), (8, 128, 128, 8 * (2048 + 128)), (1, 128, 32, 2048 + 512)])
def test_page_sizes(heads, dh, group, size):
    assert binding.Layer(W.LayerShape(256, heads, heads, dh, 256), device=-1).page_bytes(binding.Kv4(group)) == size


@pytest.mark.parametrize("group", [0, 16, 33, 128, -64, 1 << 40])
def test_other_groups_are_refused(group):
    layer, cache = make_layer(), binding.Kv4(group)
    for call in (lambda: layer.page_bytes(cache), lambda: layer.window_plan(make_batch([(1, 40)]), 8, cache=cache),
                 lambda: layer.kv4_pack(bf16(1, 16, 2, 64), bf16(1, 16, 2, 64), cache, stream=Stream), lambda: layer.kv4_unpack(u8(0), cache, stream=Stream),
                 lambda: layer.copy_pages(u8(0).view(1, 0), [], [], stream=Stream, cache=cache)):
        with pytest.raises(ValueError):
            call()
    assert not layer.lib.calls


def test_the_library_refuses_other_caches():
    layer = binding.Layer(SHAPE, device=-1)
    plan = layer.window_plan(make_batch([(1, 40)]), 8, cache=FOUR)
    lib = layer.lib
    for bits, group in ((4, 0), (4, 128), (4, 48), (8, 32), (16, 32), (2, 32), (0, 0)):
        assert lib.bs_window_cache(plan.h, bits, group) < 0 and "bs_window_cache" in layer.last_error()
    assert plan.division().pages == 1                      # (a refused change leaves the plan)
    assert lib.bs_window_cache(plan.h, 16, 0) == 0
    with pytest.raises(binding.BlendStepError, match="nothing is planned"):
        plan.division()                                    # (a change ends it)
    assert lib.bs_window_cache(None, 4, 32) < 0 and lib.bs_kv4_page_bytes(None, 32) == 0 and lib.bs_kv4_page_bytes(layer.h, 48) == 0


def test_host_only_contexts_and_bad_arguments_are_errors():
    layer = binding.Layer(SHAPE, device=-1)
    lib, h, none = layer.lib, layer.h, None
    p = C.c_void_p(1 << 20)
    for rc in (lib.bs_kv4_pack(h, p, p, p, 1, 32, none), lib.bs_kv4_unpack(h, p, p, p, 1, 32, none), lib.bs_w8_quantize(h, p, 64, 1, 64, p, p, none),
               lib.bs_w8_linear(h, p, p, p, p, 1, 1, 64, p, 1, none), lib.bs_w8_linear_rows(h, p, 64, p, p, 1, 1, 64, p, 1, none, none)):
        assert rc < 0 and "host-only" in layer.last_error()
    assert lib.bs_kv4_copy_pages(h, none, 1, 1, 48, none, none, 0, none) < 0 and "48" in layer.last_error()
    assert lib.bs_kv4_compact(h, none, 1, 1, 48, none, 0, none, none, none) < 0
    for f, n in ((lib.bs_kv4_pack, 7), (lib.bs_kv4_unpack, 7), (lib.bs_w8_quantize, 8), (lib.bs_w8_linear, 11), (lib.bs_w8_linear_rows, 12), (lib.bs_kv4_copy_pages, 9),
                 (lib.bs_kv4_compact, 10)):
        assert f(*[None if t is C.c_void_p else 0 for t in f.argtypes]) < 0 and len(f.argtypes) == n
    r = [C.c_int32() for _ in range(3)]
    for m, n, k in ((0, 5, 64), (5, 0, 64), (5, 5, 8), (5, 5, 72), (5, 5, 1 << 20), (1 << 40, 5, 64)):
        assert lib.bs_w8_division(h, m, n, k, *(C.byref(v) for v in r)) < 0
    assert lib.bs_w8_division(h, 1, 1, 16, None, None, None) < 0
    assert lib.bs_w8_scratch_bytes(0, 64) == lib.bs_w8_scratch_bytes(2, 4096) == 0 and lib.bs_w8_scratch_bytes(5, 4096) == 32 + 5 * 4096


def test_a_step_over_either_cache_names_the_same_pages():
    layer = binding.Layer(W.LLAMA3_70B, device=-1)
    for seqs, window, sinks in (([(1, 900), (1, 33), (3, 70)], 1000, 0), ([(400, 900), (1, 2000), (0, 5)], 300, 20), ([(700, 700)], 50, 0)):
        four, sixteen = (layer.window_plan(make_batch(seqs), window, sinks, cache=c) for c in (binding.Kv4(64), None))
        a, b = four.division(), sixteen.division()
        assert min(a.pages, b.pages) > 0 and a.units + a.wide_blocks > 0 and (a.pages == b.pages or a.wide_blocks != b.wide_blocks)


@pytest.mark.parametrize("rows,kv,window", [(1, 100, 20), (300, 400, 10)])
def test_pages_given_up_that_a_row_sees_are_refused(rows, kv, window):
    layer = make_layer()
    first = (kv - rows - window + 1) // 16          # the first page that the first row sees
    layer.window_plan(make_batch([(rows, kv)], given_up={0: range(first)}), window, cache=FOUR)
    with pytest.raises(binding.BlendStepError, match="given up"):
        layer.window_plan(make_batch([(rows, kv)], given_up={0: [first]}), window, cache=FOUR)


# ---- pools --------------------------------------------------------------------------------------
def test_pools_of_the_other_kind_are_refused():
    layer = make_layer()
    batch = make_batch([(1, 40), (2, 20)])
    four, sixteen = layer.window_plan(batch, 8, cache=FOUR), layer.window_plan(batch, 8)
    size = layer.page_bytes(FOUR)
    good4, good16 = u8(batch.n_pages * size), bf16(batch.n_pages * layer.page_bytes() // 2)
    q, qkv = bf16(3, 512), bf16(3, SHAPE.n_qkv)
    for plan, pool in ((four, good16), (sixteen, good4), (four, good4[:-1]), (four, good4.view(torch.int8)), (four, u8(2 * good4.numel())[::2])):
        with pytest.raises(ValueError, match="pool"):
            layer.window_attention(plan, q, pool, stream=Stream)
        with pytest.raises(ValueError, match="pool"):
            layer.rope_append(plan, qkv, pool, stream=Stream)
    assert not layer.lib.calls
    layer.window_attention(four, q, good4, stream=Stream)
    layer.rope_append(four, qkv, good4, stream=Stream)
    layer.window_attention(sixteen, q, good16, stream=Stream)
    assert len(layer.lib.calls) == 3


@pytest.mark.parametrize("k,v", [((2, 16, 2, 64), (3, 16, 2, 64)), ((2, 16, 64), (2, 16, 64)), ((2, 8, 2, 64), (2, 8, 2, 64)), ((2, 16, 2, 32), (2, 16, 2, 32))])
def test_shapes_of_conversions(k, v):
    layer = make_layer()
    with pytest.raises(ValueError, match="kv4_pack"):
        layer.kv4_pack(bf16(*k), bf16(*v), FOUR, stream=Stream)
    with pytest.raises(ValueError, match="kv4_pack"):
        layer.kv4_pack(torch.zeros(2, 16, 2, 64), torch.zeros(2, 16, 2, 64), FOUR, stream=Stream)
    with pytest.raises(ValueError, match="kv4_pack"):
        layer.kv4_pack(bf16(2, 16, 64, 2).transpose(2, 3), bf16(2, 16, 2, 64), FOUR, stream=Stream)
    size = layer.page_bytes(FOUR)
    for pool in (u8(size + 1), u8(2 * size)[::2], torch.zeros(size, dtype=torch.int8)):
        with pytest.raises(ValueError, match="kv4_unpack"):
            layer.kv4_unpack(pool, FOUR, stream=Stream)
    assert not layer.lib.calls
    assert layer.kv4_pack(bf16(2, 16, 2, 64), bf16(2, 16, 2, 64), FOUR, stream=Stream).numel() == 2 * size
    assert tuple(layer.kv4_unpack(u8(3 * size), FOUR, stream=Stream)[1].shape) == (3, 16, 2, 64) and len(layer.lib.calls) == 2


def test_copies_count_pages_of_their_cache():
    layer = make_layer()
    size = layer.page_bytes(FOUR)
    with pytest.raises(ValueError, match="uint8"):
        layer.copy_pages(bf16(2, size), [0], [1], stream=Stream, cache=FOUR)
    with pytest.raises(ValueError, match="bf16"):
        layer.copy_pages(torch.zeros((2, 6 * size), dtype=torch.uint8), [0], [1], stream=Stream)
    pools = torch.zeros((2, 6 * size), dtype=torch.uint8)
    layer.copy_pages(pools, [0], [1], stream=Stream, cache=FOUR)
    layer.copy_pages(list(pools), [0], [1], stream=Stream, cache=FOUR)
    layer.compact_pages(pools, [5, 3], stream=Stream, cache=FOUR)
    assert [(n, a[2], a[3], a[4]) for n, a in layer.lib.calls] == [("bs_kv4_copy_pages", 2, 6, 32)] * 2 + [("bs_kv4_compact", 2, 6, 32)]


# ---- 8-bit products ------------------------------------------------------------------------------
def weight(n, k):
    return binding.W8Weight(torch.zeros((n, k), dtype=torch.int8), torch.zeros(n))


def test_integers_and_scales_belong_together():
    q = torch.zeros((4, 32), dtype=torch.int8)
    for a, b in ((q.to(torch.uint8), torch.zeros(4)), (q, torch.zeros(3)), (q, torch.zeros(4, dtype=torch.bfloat16)), (q, torch.zeros(4, 1)), (q.t(), torch.zeros(32)),
                 (q[0], torch.zeros(32)), (q, torch.zeros(8)[::2])):
        with pytest.raises(ValueError):
            binding.W8Weight(a, b)
    binding.W8Weight(q, torch.zeros(4))


def test_products_check_their_rows():
    layer, w = make_layer(), weight(5, 32)
    for x in (bf16(3, 48), torch.zeros(3, 32), bf16(32), bf16(32, 3).t(), bf16(1, 3, 32)):
        with pytest.raises(ValueError):
            layer.w8_linear(x, w, stream=Stream)
    for out in (bf16(3, 4), bf16(2, 5), torch.zeros(3, 5), bf16(5, 3).t()):
        with pytest.raises(ValueError, match="out"):
            layer.w8_linear(bf16(3, 32), w, out=out, stream=Stream)
    with pytest.raises(ValueError):
        layer.w8_quantize(bf16(32, 3).t(), stream=Stream)
    assert not layer.lib.calls
    assert tuple(layer.w8_linear(bf16(3, 32), w, stream=Stream).shape) == (3, 5)
    rows = layer.w8_quantize(bf16(7, 40)[:, :32], stream=Stream)
    layer.w8_linear(rows, w, out=bf16(7, 9)[:, 2:7], stream=Stream)
    layer.w8_linear(bf16(9, 64)[::3, :32], w, stream=Stream)
    layer.w8_linear(bf16(1, 32).expand(1, 32), w, stream=Stream)
    names = [n for n, _ in layer.lib.calls]
    assert names == ["bs_w8_linear_rows", "bs_w8_quantize", "bs_w8_linear", "bs_w8_linear_rows", "bs_w8_linear_rows"]
    assert layer.lib.calls[1][1][2] == 40 and layer.lib.calls[2][1][9] == 9 and layer.lib.calls[3][1][2] == 192


def test_tensors_on_other_devices_are_refused(monkeypatch):
    class Elsewhere:
        """A tensor of another device, in name."""
        def __init__(self, t):
            self.t = t

        def __getattr__(self, name):
            return getattr(self.t, name)

        def get_device(self):
            return 3
    layer = make_layer()
    for call in (lambda: layer.w8_quantize(Elsewhere(bf16(2, 32)), stream=Stream), lambda: layer.w8_linear(Elsewhere(bf16(2, 32)), weight(5, 32), stream=Stream),
                 lambda: layer.w8_linear(bf16(2, 32), weight(5, 32), out=Elsewhere(bf16(2, 5)), stream=Stream),
                 lambda: layer.kv4_unpack(Elsewhere(u8(layer.page_bytes(FOUR))), FOUR, stream=Stream),
                 lambda: layer.kv4_pack(bf16(1, 16, 2, 64), Elsewhere(bf16(1, 16, 2, 64)), FOUR, stream=Stream),
                 lambda: layer.copy_pages([Elsewhere(u8(0))], [], [], stream=Stream, cache=FOUR)):
        with pytest.raises(ValueError, match="layer on device"):
            call()
    assert not layer.lib.calls


def test_every_kind_of_tile_is_reached():
    layer, seen = binding.Layer(SHAPE, device=-1), set()
    for m, n, k in ((9, 2857, 3952), (1, 5123, 7728), (51, 412, 4352), (20, 13329, 2368), (53, 15186, 2432), (678, 1071, 5008), (1090, 4091, 4080), (845, 18071, 2880), (433, 17789, 10000),
                    (1123, 9151, 4160), (2166, 13634, 20416)):
        rows, outputs, ranges = layer.w8_division(m, n, k)
        seen.add((rows, outputs))
        assert ranges >= 1 and (rows > 32 or ranges == 1)
    assert seen >= {(16, 16), (16, 32), (32, 16), (32, 32), (64, 128), (128, 128), (192, 128), (128, 256), (160, 256), (192, 256), (256, 256)}, seen


def test_every_kind_of_tile_takes_ranges_too():
    layer, seen = binding.Layer(SHAPE, device=-1), set()
    for m, n, k in ((127, 465, 3616), (340, 1133, 7376), (133, 5923, 7760), (199, 8826, 5952), (799, 2509, 7696), (541, 6409, 11040), (995, 5415, 10832)):
        rows, outputs, ranges = layer.w8_division(m, n, k)
        assert ranges > 1
        seen.add((rows, outputs))
    assert seen == {(64, 128), (128, 128), (192, 128), (128, 256), (160, 256), (192, 256), (256, 256)}, seen


def test_streams_take_weights_from_rows():
    from types import SimpleNamespace

    from paper_2411_16102_amd.streams import Streams
    q, s = torch.zeros((4, 32), dtype=torch.int8), torch.zeros(4)
    st = Streams.__new__(Streams)
    st.layer = SimpleNamespace(w8_linear=lambda x, w: "eight", w4_linear=lambda x, w: "four")
    assert [st.linear(None, w) for w in (binding.W8Rows(q, s), binding.W8Weight(q, s), binding.W4Weight)] == ["eight", "eight", "four"]


@pytest.mark.parametrize("hq,hkv,dh,group,seqs,window,units,blocks,waves,pages", [
    (32, 8, 128, 128, [(700, 2200)] * 6, 1 << 20, 0, 132, 1, 15444), (32, 8, 128, 64, [(700, 2200)] * 6, 1 << 20, 0, 132, 1, 15444),
    (32, 8, 128, 32, [(700, 2200)] * 6, 1 << 20, 1050, 0, 1, 121932), (32, 8, 128, 128, [(300, 2200)] * 3, 1 << 20, 225, 0, 1, 28941),
    (32, 8, 128, 128, [(400, 2200)] * 4 + [(1, 2000)] * 40, 1 << 20, 40, 52, 4, 11600), (64, 8, 128, 128, [(500, 900)] * 5, 1 << 20, 0, 160, 1, 6640),
    (32, 8, 64, 64, [(700, 2200)] * 6, 1 << 20, 0, 132, 1, 15444), (32, 8, 64, 32, [(900, 2200)] * 6, 500, 0, 174, 1, 6078),
    (16, 16, 128, 64, [(1000, 3000)] * 4, 1 << 20, 0, 32, 1, 5148), (16, 16, 128, 64, [(200, 300)] * 4, 64, 52, 0, 2, 360),
    (48, 8, 128, 128, [(2000, 2000), (5, 900)], 1 << 20, 0, 101, 1, 6407)])
def test_which_kind_of_work_longer_segments_are(hq, hkv, dh, group, seqs, window, units, blocks, waves, pages):
    # as both kinds and every division of either are expected to take; a plan may leave out what it knows to be longer
    layer = binding.Layer(W.LayerShape(256, hq, hkv, dh, 256), device=-1)
    d = layer.window_plan(make_batch(seqs), window, 4, cache=binding.Kv4(group)).division()
    assert (d.units, d.wide_blocks, d.waves, d.pages) == (units, blocks, waves, pages)


def test_plans_leave_out_what_is_longer():
    # four segments of 4096 rows: as units of four rows each they name eight times the pages (without looking at these 1.2 ms a plan, with them 4.7; over the
    # cache in bf16 2.7)
    import time
    layer, batch = binding.Layer(W.LLAMA3_8B, device=-1), make_batch([(4096, 12000)] * 4)
    plans = [layer.window_plan(batch, 1 << 20, cache=c) for c in (binding.Kv4(128), None)]
    times = [[], []]
    for _ in range(8):
        for plan, t in zip(plans, times):
            start = time.perf_counter()
            plan.update(batch, 1 << 20)
            t.append(time.perf_counter() - start)
    assert min(times[0]) < min(times[1])

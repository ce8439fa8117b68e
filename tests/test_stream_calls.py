"""What the Python calls of the stream operators check before the library is reached, on contexts without a device.

A layer here is host-only (CPU tensors are then those of its device) and its library is one that writes down what it
is asked, so that a call that passes the checks is seen and nothing runs."""
import numpy as np
import pytest
import torch

from paper_2411_16102_amd import binding, workloads as W
from stream_cases import make_batch

SHAPE = W.LayerShape(256, 8, 2, 64, 256)


class Asked:
    """The library, but for the calls that would launch something: those are kept in `calls` and answer `rc`."""

    def __init__(self, lib, rc=0):
        self._lib, self.rc, self.calls = lib, rc, []

    def __getattr__(self, name):
        if name not in ("bs_window_attention", "bs_rope_append", "bs_w4_pack", "bs_w4_linear", "bs_kv_copy_pages", "bs_kv_compact"):
            return getattr(self._lib, name)

        def call(*args):
            self.calls.append((name, args))
            return self.rc
        return call


class Stream:
    """A stream in name: contexts without a device use none."""
    cuda_stream = 0


@pytest.fixture(autouse=True)
def _streams_in_name(monkeypatch):
    from contextlib import nullcontext
    monkeypatch.setattr(torch.cuda, "stream", nullcontext)


def make_layer(shape=SHAPE, rc=0):
    layer = binding.Layer(shape, device=-1)
    layer.lib = Asked(layer.lib, rc)
    return layer


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


# ---- plans of other layers ------------------------------------------------------------------
@pytest.mark.parametrize("other", [W.LayerShape(256, 4, 4, 128, 256), W.LayerShape(256, 8, 1, 64, 256), W.LayerShape(256, 4, 1, 128, 256),
                                   W.LayerShape(256, 8, 2, 64, 256, rope_theta=10000.0)])
def test_plans_of_layers_with_other_shapes_are_refused(other):
    # (the queries of all of these are as wide as the layer's: their pages, their groups or their angles differ)
    layer, owner = make_layer(), make_layer(other)
    batch = make_batch([(1, 40), (3, 20)])
    plan = owner.window_plan(batch, 8)
    pool = bf16(batch.n_pages * max(layer.page_bytes(), owner.page_bytes()))
    with pytest.raises(ValueError, match="another device, or with other heads"):
        layer.window_attention(plan, bf16(4, 512), pool, stream=Stream)
    with pytest.raises(ValueError, match="another device, or with other heads"):
        layer.rope_append(plan, bf16(4, SHAPE.n_qkv), pool, stream=Stream)
    assert not layer.lib.calls and not owner.lib.calls


def test_plans_of_layers_on_other_devices_are_refused():
    layer, owner = make_layer(), make_layer()
    batch = make_batch([(1, 40)])
    plan, pool = owner.window_plan(batch, 8), bf16(batch.n_pages * layer.page_bytes() // 2)
    layer.window_attention(plan, bf16(1, 512), pool, stream=Stream)  # (a layer of the same kind: its plan is as good)
    assert len(layer.lib.calls) == 1
    owner._plan_key = (1,) + owner._plan_key[1:]  # as if it had been made on device 1
    with pytest.raises(ValueError, match="another device"):
        layer.window_attention(plan, bf16(1, 512), pool, stream=Stream)
    assert len(layer.lib.calls) == 1


def test_the_message_of_a_plans_error_is_the_plans():
    layer, owner = binding.Layer(SHAPE, device=-1), binding.Layer(SHAPE, device=-1)
    batch = make_batch([(1, 40)])
    plan, pool = owner.window_plan(batch, 8), bf16(batch.n_pages * layer.page_bytes() // 2)
    with pytest.raises(binding.BlendStepError, match="host-only context"):
        layer.window_attention(plan, bf16(1, 512), pool, stream=Stream)
    with pytest.raises(binding.BlendStepError, match="host-only context"):
        layer.rope_append(plan, bf16(1, SHAPE.n_qkv), pool, stream=Stream)


# ---- plans and contexts that end --------------------------------------------------------------
class Ends:
    """The library, with the order in which contexts (True) and plans (False) end."""

    def __init__(self, lib):
        self._lib, self.order = lib, []

    def __getattr__(self, name):
        if name not in ("bs_destroy", "bs_window_destroy"):
            return getattr(self._lib, name)

        def call(h):
            self.order.append(name == "bs_destroy")
            if not all(self.order):  # (a plan that outlives its context must not be ended through it)
                getattr(self._lib, name)(h)
        return call


@pytest.mark.parametrize("how", ["layer first", "plan first", "dropped", "a cycle", "a cycle that was closed"])
def test_plans_end_before_their_layer(how):
    import gc
    layer = binding.Layer(SHAPE, device=-1)
    ends = layer.lib = Ends(layer.lib)
    plans = [layer.window_plan(make_batch([(1, 40)]), 8) for _ in range(2)]
    if how.startswith("a cycle"):
        layer.plans = plans
    if how in ("layer first", "a cycle that was closed"):
        layer.close()
    elif how == "plan first":
        for p in plans:
            p.close()
        layer.close()
    if not how.startswith("a cycle"):
        for p in plans:
            p.close()
        p = None
    del layer, plans
    gc.collect()
    assert ends.order == [False, False, True]


def test_a_closed_layers_plans_raise():
    layer = binding.Layer(SHAPE, device=-1)
    batch = make_batch([(1, 40)])
    plan = layer.window_plan(batch, 8)
    gone = layer.window_plan(batch, 8)
    gone.close()
    gone.close()
    with pytest.raises(ValueError, match="closed"):
        gone.division()
    assert plan.division().pages == 1
    layer.close()
    for call in (lambda: plan.update(batch, 8), lambda: plan.division(), lambda: layer.window_plan(batch, 8),
                 lambda: layer.window_attention(plan, bf16(1, 512), bf16(3 * 16 * 256), stream=Stream),
                 lambda: layer.rope_append(plan, bf16(1, SHAPE.n_qkv), bf16(3 * 16 * 256), stream=Stream)):
        with pytest.raises(ValueError, match="closed"):
            call()
    plan.close()
    layer.close()


# ---- tensors of other devices --------------------------------------------------------------------
def test_tensors_of_other_devices_are_refused():
    layer = make_layer()
    layer.device = 0  # as a layer of the first GPU: the tensors below are the host's
    batch = make_batch([(1, 40), (3, 20)])
    own = make_layer()
    plan = own.window_plan(batch, 8)
    plan.layer = layer
    q, qkv, pool = bf16(4, 512), bf16(4, SHAPE.n_qkv), bf16(batch.n_pages * layer.page_bytes() // 2)
    packed, scales, zeros = torch.zeros((16, 64), dtype=torch.uint8), bf16(16, 2), torch.zeros((16, 2), dtype=torch.uint8)
    weight = own.w4_pack(packed, scales, zeros, stream=Stream)
    calls = (lambda l: l.window_attention(plan, q, pool, stream=Stream), lambda l: l.window_attention(plan, q, pool, out=q, stream=Stream),
             lambda l: l.rope_append(plan, qkv, pool, stream=Stream), lambda l: l.rope_append(plan, qkv, pool, q=q, stream=Stream),
             lambda l: l.w4_pack(packed, scales, stream=Stream), lambda l: l.w4_pack(packed, scales, zeros, stream=Stream),
             lambda l: l.w4_linear(bf16(2, 128), weight, stream=Stream), lambda l: l.w4_linear(bf16(2, 128), weight, out=bf16(2, 16), stream=Stream),
             lambda l: l.copy_pages(pool.view(1, -1), [0], [1], stream=Stream), lambda l: l.copy_pages([pool, pool], [0], [1], stream=Stream),
             lambda l: l.compact_pages([pool], [0, 2], stream=Stream), lambda l: l.compact_pages(pool.view(1, -1), [0, 2], stream=Stream))
    for call in calls:
        with pytest.raises(ValueError, match=" on cpu"):
            call(layer)
    assert not layer.lib.calls
    # the same calls on a layer of their own device are asked
    plan.layer = own
    own.lib.calls.clear()
    for call in calls:
        call(own)
    assert len(own.lib.calls) == len(calls)


def test_every_tensor_of_a_call_is_looked_at():
    # one of them elsewhere is enough
    layer = make_layer()
    batch = make_batch([(1, 40)])
    plan = layer.window_plan(batch, 8)
    pool, far = bf16(batch.n_pages * layer.page_bytes() // 2), lambda *shape: Elsewhere(bf16(*shape))
    weight = layer.w4_pack(torch.zeros((16, 64), dtype=torch.uint8), bf16(16, 2), stream=Stream)
    there = binding.W4Weight(Elsewhere(weight.data), weight.n, weight.k, weight.group, weight.with_zeros)
    u8 = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    layer.lib.calls.clear()
    for call in (lambda: layer.window_attention(plan, far(1, 512), pool, stream=Stream), lambda: layer.window_attention(plan, bf16(1, 512), Elsewhere(pool), stream=Stream),
                 lambda: layer.window_attention(plan, bf16(1, 512), pool, out=far(1, 512), stream=Stream),
                 lambda: layer.rope_append(plan, far(1, SHAPE.n_qkv), pool, stream=Stream), lambda: layer.rope_append(plan, bf16(1, SHAPE.n_qkv), Elsewhere(pool), stream=Stream),
                 lambda: layer.rope_append(plan, bf16(1, SHAPE.n_qkv), pool, q=far(1, 512), stream=Stream),
                 lambda: layer.w4_pack(Elsewhere(u8(16, 64)), bf16(16, 2), u8(16, 2), stream=Stream), lambda: layer.w4_pack(u8(16, 64), far(16, 2), u8(16, 2), stream=Stream),
                 lambda: layer.w4_pack(u8(16, 64), bf16(16, 2), Elsewhere(u8(16, 2)), stream=Stream),
                 lambda: layer.w4_linear(far(2, 128), weight, stream=Stream), lambda: layer.w4_linear(bf16(2, 128), there, stream=Stream),
                 lambda: layer.w4_linear(bf16(2, 128), weight, out=far(2, 16), stream=Stream),
                 lambda: layer.copy_pages([pool, Elsewhere(pool)], [0], [1], stream=Stream), lambda: layer.compact_pages([pool, Elsewhere(pool)], [0], stream=Stream)):
        with pytest.raises(ValueError, match=" on cuda:3"):
            call()
    assert not layer.lib.calls


class Elsewhere:
    """A tensor that says it is on another device."""

    def __init__(self, t):
        self._t, self.device = t, torch.device("cuda", 3)

    def __getattr__(self, name):
        return getattr(self._t, name)

    def get_device(self):
        return 3


# ---- results on another stream ------------------------------------------------------------------
class Allocating(torch.Tensor):
    """A tensor that writes down under which stream memory like its own is asked for."""
    current, asked = None, []

    def new_empty(self, *args, **kw):
        Allocating.asked.append(Allocating.current)
        return self.as_subclass(torch.Tensor).new_empty(*args, **kw)


def test_results_are_allocated_for_the_stream_of_the_call(monkeypatch):
    from contextlib import contextmanager

    @contextmanager
    def under(stream):
        Allocating.current = stream
        yield
        Allocating.current = None
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(binding, "_current_stream", lambda device: 0)
    monkeypatch.setattr(Allocating, "asked", [])
    layer = make_layer()
    batch = make_batch([(1, 40)])
    plan, pool = layer.window_plan(batch, 8), bf16(batch.n_pages * layer.page_bytes() // 2)
    mine = lambda t: t.as_subclass(Allocating)
    weight = layer.w4_pack(torch.zeros((16, 64), dtype=torch.uint8), bf16(16, 2))
    for stream in (Stream, None):
        Allocating.asked.clear()
        layer.window_attention(plan, mine(bf16(1, 512)), pool, stream=stream)
        layer.rope_append(plan, mine(bf16(1, SHAPE.n_qkv)), pool, stream=stream)
        layer.w4_pack(mine(torch.zeros((16, 64), dtype=torch.uint8)), bf16(16, 2), stream=stream)
        layer.w4_linear(mine(bf16(2, 128)), weight, stream=stream)
        assert Allocating.asked == [stream] * 4


# ---- strides that no element uses ---------------------------------------------------------------
def row(k, offset=0):
    """A row of k elements, contiguous, whose stride along the rows is one."""
    t = torch.zeros((offset + k, 1), dtype=torch.bfloat16)[offset:].t()
    assert t.is_contiguous() and t.stride() == (1, 1)
    return t


def test_the_stride_of_a_single_row_is_not_looked_at():
    layer = make_layer()
    batch = make_batch([(1, 40)])
    plan, pool = layer.window_plan(batch, 8), bf16(batch.n_pages * layer.page_bytes() // 2)
    calls = layer.lib.calls
    q, out = row(512), row(512)
    layer.window_attention(plan, q, pool, out=out, stream=Stream)
    layer.window_attention(plan, q, pool, out=q, stream=Stream)
    layer.window_attention(plan, q, pool, out=bf16(1, 512), stream=Stream)
    for _, (_, _, q_stride, _, out_stride, _, _) in calls:
        assert q_stride >= 512 and out_stride >= 512 and q_stride % 8 == 0 and out_stride % 8 == 0
    assert calls[1][1][2] == calls[1][1][4], "in place with one stride"
    calls.clear()
    qkv = row(SHAPE.n_qkv)
    layer.rope_append(plan, qkv, pool, stream=Stream)
    layer.rope_append(plan, qkv, pool, q=qkv[:, :512], stream=Stream)
    layer.rope_append(plan, bf16(1, SHAPE.n_qkv), pool, q=row(512), stream=Stream)
    for _, (_, _, stride, _, q_stride, _, _) in calls:
        assert stride >= SHAPE.n_qkv and q_stride >= 512 and stride % 8 == 0 and q_stride % 8 == 0
    assert calls[1][1][1] == calls[1][1][3] and calls[1][1][2] == calls[1][1][4], "in place with one stride"
    calls.clear()
    weight = layer.w4_pack(torch.zeros((17, 64), dtype=torch.uint8), bf16(17, 2), stream=Stream)
    layer.w4_linear(row(128), weight, out=row(17), stream=Stream)
    stride, out_stride = calls[-1][1][2], calls[-1][1][10]
    assert stride >= 128 and stride % 8 == 0 and out_stride >= 17
    # rows that are not contiguous in themselves, and strides of several rows, are refused as before
    for bad in (lambda: layer.window_attention(plan, bf16(1, 1024)[:, ::2], pool, stream=Stream), lambda: layer.w4_linear(bf16(1, 256)[:, ::2], weight, stream=Stream),
                lambda: layer.w4_linear(bf16(2, 128), weight, out=bf16(17, 2).t(), stream=Stream)):
        with pytest.raises(ValueError):
            bad()


def test_the_stride_of_a_single_column_is_not_looked_at():
    layer = make_layer()
    weight = layer.w4_pack(torch.zeros((1, 64), dtype=torch.uint8), bf16(1, 2), stream=Stream)
    out = bf16(1, 5).t()
    assert out.shape == (5, 1) and out.stride() == (1, 5)
    layer.w4_linear(bf16(5, 128), weight, out=out, stream=Stream)
    assert layer.lib.calls[-1][1][10] == 1
    layer.w4_linear(bf16(0, 128), weight, out=bf16(1, 0).t(), stream=Stream)


# ---- numbers that do not fit ----------------------------------------------------------------------
BIG = 1 << 32


def test_numbers_beyond_32_bits_are_refused():
    p = binding.Pages(20)
    ids = p.open(2)
    p.extend(ids, [5, 17])
    for call in (lambda: binding.Pages(BIG + 3), lambda: p.open(BIG + 1), lambda: p.fork(ids, BIG + 1), lambda: p.fork(ids, (1 << 31) - 1), lambda: p.extend(ids, BIG + 1),
                 lambda: p.extend(ids, np.array([1, BIG + 1])), lambda: p.extend(ids, np.array([1.0, 1.5])), lambda: p.extend(ids, [0.5, 1]),
                 lambda: p.extend(ids.astype(np.int64) + BIG, 1), lambda: p.free(np.array([BIG])), lambda: p.tables(np.array([-BIG])), lambda: p.fork(np.array([np.nan]), 1)):
        with pytest.raises(ValueError):
            call()
    assert p.lengths(ids).tolist() == [5, 17] and p.stats() == {"free": 17, "sequences": 2}
    # whole numbers of any type are taken
    p.extend(ids.astype(np.int64), np.array([1.0, 2.0]))
    p.extend([int(i) for i in ids], np.uint8(3))
    p.extend(ids, 1)
    assert p.lengths(ids).tolist() == [10, 23]


def test_tables_and_positions_beyond_32_bits_are_refused():
    layer = make_layer()
    pool = bf16(4 * layer.page_bytes() // 2)
    for call in (lambda: layer.copy_pages([pool], np.array([BIG]), [1], stream=Stream), lambda: layer.copy_pages([pool], [0], np.array([BIG + 1]), stream=Stream),
                 lambda: layer.compact_pages([pool], np.array([BIG + 1]), stream=Stream), lambda: layer.compact_pages([pool], [0.5], stream=Stream)):
        with pytest.raises(ValueError):
            call()
    assert not layer.lib.calls
    batch = make_batch([(2, 40)])
    for bad in (np.full((1, 2), BIG), np.full((1, 2), 0.5)):
        with pytest.raises(ValueError):
            layer.window_plan(batch, 8, positions=bad, axis_of_pair=np.zeros(32))
    layer.window_plan(batch, 8, positions=np.full((1, 2), 7.0), axis_of_pair=np.zeros(32))


def test_windows_and_sinks_beyond_every_length():
    layer = make_layer()
    batch = make_batch([(1, 1000)])
    for window, sinks, pages in ((BIG + 5, 0, 63), (BIG, 0, 63), (1 << 31, 0, 63), (16, BIG, 63), (16, BIG + 3, 63), (8, 0, 1), (np.int64(17), np.int64(0), 2)):
        assert layer.window_plan(batch, window, sinks).division().pages == pages
    for window, sinks in ((5 - BIG, 0), (16, 3 - BIG)):
        with pytest.raises(binding.BlendStepError, match="at least"):
            layer.window_plan(batch, window, sinks)
    p = binding.Pages(63)
    ids = p.open(1)
    p.extend(ids, 1000)
    for window, sinks in ((BIG + 5, 0), (BIG, 0), (16, BIG), (16, BIG + 3)):
        p.trim(ids, window, sinks)
        assert (p.tables(ids)[1] >= 0).all()
    with pytest.raises(binding.BlendStepError, match="at least"):
        p.trim(ids, 5 - BIG, 0)
    p.trim(ids, 16, 0)
    assert (p.tables(ids)[1] >= 0).sum() == 2


# ---- laid-out weights --------------------------------------------------------------------------------
def test_weights_with_less_memory_than_their_layout_are_refused():
    layer = make_layer()
    w = layer.w4_pack(torch.zeros((17, 64), dtype=torch.uint8), bf16(17, 2), torch.zeros((17, 2), dtype=torch.uint8), stream=Stream)
    size = layer.lib.bs_w4_bytes(17, 128, 64, 1)
    assert w.data.numel() == size
    binding.W4Weight(w.data, 17, 128, 64, True)
    binding.W4Weight(w.data, 17, 128, 64, False)
    binding.W4Weight(bf16(size // 2), 17, 128, 64, True)
    for data, n, k in ((w.data[:-1], 17, 128), (w.data, 33, 128), (w.data, 17, 256), (torch.zeros(2 * size, dtype=torch.uint8)[::2], 17, 128)):
        with pytest.raises(ValueError, match="laid-out weight"):
            binding.W4Weight(data, n, k, 64, True)

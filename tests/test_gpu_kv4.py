"""A cache in four bits on the GPU against its definition in float64.

Tolerances, from the arithmetic.  Of bf16 inputs the codes are exact: values that are read back equal the definition's, rounded to
bf16 once (relative 2^-8).  Attention: probabilities, and probabilities times scale, are rounded to bf16 before their
products (2^-8 of the sum of p (|mid| + |scale (c - 8)|)), the output once more; sums in 32 bits carry up to 31 scale p for each token and are off
by 2^-24 of that for each of the steps a token passes through, at most one for each 32 tokens of its unit."""
import numpy as np
import pytest

from oracle import bits as OB, stream as OS
from paper_2411_16102_amd import workloads as W
from stream_cases import make_batch

pytestmark = pytest.mark.gpu
U = 2.0 ** -8

# query heads, KV heads, head size, group
SHAPES = [(8, 2, 128, 128), (8, 2, 128, 64), (16, 1, 128, 32), (8, 2, 64, 64), (4, 4, 64, 32), (6, 2, 128, 64), (3, 1, 64, 32), (14, 2, 128, 32),
          (16, 4, 128, 64), (32, 8, 128, 128), (32, 8, 64, 32), (12, 4, 64, 64), (8, 4, 128, 32)]


def make_layer(lib, hq, hkv, dh, **kw):
    return lib.Layer(W.LayerShape(256, hq, hkv, dh, 256, **kw), device=0)


def to_gpu(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def to_host(t):
    return t.float().cpu().numpy().astype(np.float64)


def _bits(rng, shape, scale=1.0):
    return W.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


def _kept_bits(v, group):
    return W.f32_to_bf16_bits(OB.kv4_values(v, group)[0].astype(np.float32))


def _equal_or_nan(a, b):
    return (a == b) | (np.isnan(a) & np.isnan(b))


# ---- what a cache keeps ------------------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,dh,group", SHAPES)
def test_what_is_kept(lib, hq, hkv, dh, group):
    layer, rng = make_layer(lib, hq, hkv, dh), np.random.default_rng(dh + group)
    shape = (5, 16, hkv, dh)
    k = _bits(rng, shape) if hkv > 1 else _bits(rng, shape, 1e-20)
    v = W.f32_to_bf16_bits((rng.standard_normal(shape) * np.exp(20 * rng.standard_normal(shape[:3]))[..., None]).astype(np.float32))
    # equal values, zeros, two values, whole numbers (halfway between codes), one far value, and what is no number
    k[0, 0] = W.f32_to_bf16_bits(np.full((hkv, dh), 3.0, dtype=np.float32))
    k[0, 1] = 0
    k[0, 2] = W.f32_to_bf16_bits(rng.integers(0, 2, (hkv, dh)).astype(np.float32))
    k[0, 3:12] = W.f32_to_bf16_bits(rng.integers(-8, 23, (9, hkv, dh)).astype(np.float32))
    k[0, 12, :, 5] = W.f32_to_bf16_bits(np.float32([1000.0]))[0]
    k[0, 13, :, 1] = 0x7FC0
    k[0, 14, :, dh - 1] = 0xFF80
    v[1, 0, :, ::2], v[1, 0, :, 1::2] = 0x7F7F, 0xFF7F     # the largest numbers of either sign: further apart than 32 bits say
    v[1, 1] = W.f32_to_bf16_bits(np.full((hkv, dh), 2.0 ** -133, dtype=np.float32))
    cache = lib.Kv4(group)
    pool = layer.kv4_pack(to_gpu(k), to_gpu(v), cache)
    assert pool.numel() == 5 * layer.page_bytes(cache) and layer.page_bytes(cache) == hkv * (16 * dh + 128 * dh // group)
    for got, bits in zip(layer.kv4_unpack(pool, cache), (k, v)):
        got, want = to_host(got), W.bf16_bits_to_f32(_kept_bits(W.bf16_bits_to_f32(bits), group)).astype(np.float64)
        assert _equal_or_nan(got, want).all(), "%d of %d" % ((~_equal_or_nan(got, want)).sum(), got.size)
        # no value is further than half a scale from what is kept (and its rounding)
        x = W.bf16_bits_to_f32(bits)
        scale = np.repeat(OB.kv4_numbers(x, group)[0].astype(np.float64), group, axis=-1)
        near = ~np.isnan(scale)
        assert (np.abs(got - x)[near] <= (scale * 0.5 * (1 + 1e-6) + U * np.abs(want))[near]).all()
    assert np.isnan(to_host(layer.kv4_unpack(pool, cache)[0])[0, 13]).any() and (to_host(layer.kv4_unpack(pool, cache)[0])[0, 1] == 0).all()


def test_pages_of_zero_bytes_stand_for_zeros(lib):
    import torch
    layer, cache = make_layer(lib, 8, 2, 64), lib.Kv4(32)
    k, v = layer.kv4_unpack(torch.zeros(3 * layer.page_bytes(cache), dtype=torch.uint8, device="cuda"), cache)
    assert not k.any() and not v.any() and tuple(k.shape) == (3, 16, 2, 64)
    k, v = layer.kv4_unpack(torch.zeros(0, dtype=torch.uint8, device="cuda"), cache)
    assert tuple(k.shape) == (0, 16, 2, 64) and layer.kv4_pack(k, v, cache).numel() == 0


def test_more_pages_than_a_launch_has_are_refused(lib):
    import ctypes as C
    import torch
    layer = make_layer(lib, 8, 2, 64)
    t = torch.zeros(64, dtype=torch.uint8, device="cuda")
    for f in (layer.lib.bs_kv4_pack, layer.lib.bs_kv4_unpack):
        for n in (1 << 24, 1 << 23, 1 << 40, -1):     # (times two heads)
            assert f(layer.h, *[C.c_void_p(t.data_ptr())] * 3, n, 32, None) < 0 and "out of range" in layer.last_error()


# ---- attention -----------------------------------------------------------------------------------
def attention(lib, layer, group, batch, window, sinks, seed=0, poison=True, q_stride=None, offset=0.0, in_place=False, rows_checked=None):
    """Runs a step and checks every row; (plan, queries, pool, output)."""
    import torch
    shape, cache = layer.shape, lib.Kv4(group)
    rng = np.random.default_rng([seed, 3])
    hq, dh = shape.n_q_heads, shape.head_dim
    kv = (batch.n_pages, 16, shape.n_kv_heads, dh)
    k, v = (W.f32_to_bf16_bits((rng.standard_normal(kv) + offset * rng.standard_normal(kv[2:])).astype(np.float32)) for _ in range(2))
    if poison:
        used = np.zeros((batch.n_pages, 16), dtype=bool)
        for s in range(batch.n_seq):
            n, rows = int(batch.kv_len[s]), int(batch.row_start[s + 1] - batch.row_start[s])
            p, t = np.arange(n - rows, n)[:, None], np.arange(n)
            seen = np.flatnonzero(((t <= p) & ((t > p - window) | (t < sinks))).any(axis=0))
            used[batch.page_ids[batch.page_start[s] + seen // 16], seen % 16] = True
        k[~used], v[~used] = 0x7FC0, 0xFF80
    pool = layer.kv4_pack(to_gpu(k), to_gpu(v), cache)
    q = _bits(rng, (batch.n_rows, q_stride or hq * dh))
    qt = to_gpu(q)[:, :hq * dh]
    plan = layer.window_plan(batch, window, sinks, cache=cache)
    out = layer.window_attention(plan, qt, pool, out=qt if in_place else None)
    torch.cuda.synchronize()
    got = to_host(out)
    qf = W.bf16_bits_to_f32(q)[:, :hq * dh].astype(np.float64)
    for s in range(batch.n_seq):
        a, b, n = int(batch.row_start[s]), int(batch.row_start[s + 1]), int(batch.kv_len[s])
        if a == b:
            continue
        ids = batch.page_ids[batch.page_start[s]:batch.page_start[s + 1]]
        held = [W.bf16_bits_to_f32(x[np.maximum(ids, 0)]).reshape(-1, kv[2], dh)[:n] for x in (k, v)]
        (K, _), (V, V_size) = (OB.kv4_values(x, group) for x in held)
        rows = qf[a:b].reshape(b - a, hq, dh)
        parts = [(0, b - a)]
        if rows_checked and b - a > rows_checked:
            parts = [(j, j + 1) for j in sorted({0, 1, 31, 32, b - a - 1, *rng.choice(b - a, rows_checked - 5).tolist()}) if j < b - a]
        for j0, j1 in parts:
            m = min(n, max(0, n - (b - a) + j1))     # (tokens that these rows could see)
            ref, _ = OS.window_attention(rows[j0:j1], K[:m], V[:m], n - (b - a) + j0, window, sinks)
            _, size = OS.window_attention(rows[j0:j1], K[:m], V_size[:m], n - (b - a) + j0, window, sinks)
            bound = U * (np.abs(ref) + size) * 1.01 + (1e-5 + 2.0 ** -24 * 55 * (n / 32 + 8)) * size
            err = np.abs(got[a + j0:a + j1].reshape(ref.shape) - ref)
            assert np.all(err <= bound), "sequence %d (rows %d to %d, %d tokens): %.3g over the bound" % (s, j0, j1, n, np.nanmax(err - bound))
            rel = np.linalg.norm(err) / max(1e-30, np.linalg.norm(ref))
            assert rel < 5e-3, "sequence %d: relative error %.3g" % (s, rel)   # (2^-8 / 3^(1/2) twice over, for errors spread evenly)
    return plan, qt, pool, out


@pytest.mark.parametrize("hq,hkv,dh,group", SHAPES)
def test_single_tokens(lib, hq, hkv, dh, group):
    layer = make_layer(lib, hq, hkv, dh)
    batch = make_batch([(1, n) for n in (1, 2, 15, 16, 17, 32, 33, 100, 0, 129, 300)], seed=hq)
    for window, sinks in ((1, 0), (16, 0), (37, 5), (1000, 0), (20, 16)):
        attention(lib, layer, group, batch, window, sinks, seed=window, offset=0.5 if window == 37 else 0.0)


@pytest.mark.parametrize("hq,hkv,dh,group", SHAPES)
def test_rows_of_every_count(lib, hq, hkv, dh, group):
    layer = make_layer(lib, hq, hkv, dh)
    batch = make_batch([(3, 40), (0, 30), (5, 3), (17, 90), (2, 200), (70, 70), (66, 150), (4, 0), (9, 9)], seed=dh)
    for window, sinks in ((33, 3), (1, 0), (50, 70)):
        attention(lib, layer, group, batch, window, sinks, seed=window)


@pytest.mark.parametrize("window,sinks", [(1, 1), (2, 31), (15, 16), (31, 0), (64, 33), (65, 1), (128, 0), (1 << 30, 1 << 30), (100, 1000)])
def test_edges_of_windows_and_sinks(lib, window, sinks):
    layer = make_layer(lib, 8, 2, 128)
    attention(lib, layer, 32 if sinks % 2 else 128, make_batch([(1, 500), (130, 300), (1, 64), (90, 95), (3, 222)], seed=sinks % 97), window, sinks)


@pytest.mark.parametrize("hq,hkv,dh,group", [(8, 2, 128, 64), (4, 4, 64, 64), (8, 1, 128, 32)])
def test_long_contexts_are_split_and_joined(lib, hq, hkv, dh, group):
    layer = make_layer(lib, hq, hkv, dh)
    plan, *_ = attention(lib, layer, group, make_batch([(1, 6000), (2, 5500), (1, 5)]), 5000, 40)
    assert plan.division().split_rows >= 1


@pytest.mark.parametrize("hq,hkv,dh,group", [(8, 2, 128, 128), (12, 2, 64, 32), (6, 2, 128, 32), (16, 1, 64, 64)])
def test_blocks_of_rows(lib, hq, hkv, dh, group):
    layer = make_layer(lib, hq, hkv, dh)
    batch = make_batch([(700 + 13 * i, 900 + 101 * i) for i in range(7)] + [(230, 100), (700, 700), (629, 629)], seed=hq, spare=200)
    for window, sinks in ((150, 20), (10_000, 3)):
        attention(lib, layer, group, batch, window, sinks, seed=window, poison=window < 500)


@pytest.mark.parametrize("hq,hkv,dh,group,n,rows,held,window", [
    (48, 8, 128, 128, 8, 400, 200, 10_000), (48, 8, 128, 64, 4, 400, 500, 10_000), (48, 8, 128, 64, 8, 600, -20, 300), (24, 4, 128, 64, 4, 600, 1000, 10_000),
    (16, 16, 128, 128, 12, 600, 1000, 10_000), (28, 4, 128, 128, 8, 900, 500, 700), (12, 2, 64, 64, 12, 1500, 1000, 10_000), (48, 8, 64, 64, 8, 1000, 500, 300),
    (48, 8, 64, 32, 2, 1000, 1000, 10_000), (48, 16, 64, 64, 12, 400, 500, 10_000)])
def test_rows_that_share_their_pages(lib, hq, hkv, dh, group, n, rows, held, window):
    """Long segments in two blocks of columns to a wavefront, beside single tokens and sequences that are empty or begin in their rows; of each segment the first and
    last rows, those about the end of a unit and some between are checked."""
    layer = make_layer(lib, hq, hkv, dh)
    seqs = [(rows + 13 * (i % 4), rows + 13 * (i % 4) + held + 7 * i) for i in range(n)] + [(1, 300), (0, 20), (1, 1), (1, 0)]
    plan, *_ = attention(lib, layer, group, make_batch(seqs, seed=n), window, 11, seed=rows, poison=window < 1000, rows_checked=12)
    d = plan.division()
    assert d.wide_blocks > n and d.units >= 3


@pytest.mark.parametrize("hq,hkv,dh,group", [(8, 2, 128, 64), (8, 2, 64, 32)])
def test_blocks_and_units_in_one_step(lib, hq, hkv, dh, group):
    layer = make_layer(lib, hq, hkv, dh)
    seqs = [(850 + i, 1700 + 90 * i) for i in range(6)] + [(1, n) for n in (1, 0, 500, 2000, 900, 33, 64)] * 3 + [(3, 1000), (2, 1), (0, 77)]
    for window, sinks in ((400, 4), (1500, 0)):
        plan, *_ = attention(lib, layer, group, make_batch(seqs, seed=hkv), window, sinks, seed=window, poison=window < 500)
        assert plan.division().units >= 20


@pytest.mark.parametrize("hq,hkv,dh,group", [(8, 2, 128, 64), (8, 8, 64, 32)])
def test_streams_shared_by_wavefronts(lib, hq, hkv, dh, group):
    layer, seen = make_layer(lib, hq, hkv, dh), set()
    for n, ctx, window in ((200, 60, 20), (40, 700, 500), (150, 2100, 2000), (90, 2500, 2300), (1, 5000, 4800), (3, 4000, 100_000), (400, 30, 30)):
        plan, *_ = attention(lib, layer, group, make_batch([(1, max(1, ctx - 7 * (i % 9))) for i in range(n)], seed=n), window, 9, poison=n < 50)
        seen.add(plan.division().waves)
    assert len(seen) >= 2


def test_pages_given_up_strided_rows_and_in_place(lib):
    layer = make_layer(lib, 8, 2, 64)
    batch = make_batch([(1, 1000), (40, 900)], given_up={0: range(2, 56), 1: range(2, 46)})
    attention(lib, layer, 32, batch, 100, 20, q_stride=8 * 64 + 2 * 2 * 64, in_place=True)


def test_pages_that_sequences_share(lib):
    layer = make_layer(lib, 8, 2, 128)
    batch = make_batch([(1, 100), (1, 90), (1, 81)])
    table = [batch.page_ids[batch.page_start[i]:batch.page_start[i + 1]] for i in range(3)]
    for t in table[1:]:
        t[:5] = table[0][:5]
    attention(lib, layer, 64, batch, 1000, 0)


def test_a_pool_of_more_than_four_gigabytes(lib):
    # the same pages further back: the same results, and new tokens in the same places of them
    import torch
    layer, cache = make_layer(lib, 32, 8, 128), lib.Kv4(32)
    size, far = layer.page_bytes(cache), 212_000
    assert size * far > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(3)
    for seqs in ([(1, 700), (1, 33), (40, 90), (3, 3)], [(300, 2000), (280, 280)]):
        batch = make_batch(seqs)
        near_pool = torch.randint(0, 256, (batch.n_pages * size,), dtype=torch.uint8, device="cuda", generator=gen)
        k, v = (torch.randn((batch.n_pages, 16, 8, 128), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
        near_pool.copy_(layer.kv4_pack(k, v, cache))
        pool = torch.empty((far + batch.n_pages) * size, dtype=torch.uint8, device="cuda")
        pool[far * size:] = near_pool
        qkv = torch.randn((batch.n_rows, layer.shape.n_qkv), device="cuda", generator=gen).to(torch.bfloat16)
        results = []
        for at, where in ((0, near_pool), (far, pool)):
            moved = make_batch(seqs)
            moved.page_ids[:] = np.where(moved.page_ids >= 0, moved.page_ids + at, moved.page_ids)
            plan = layer.window_plan(moved, 1000, 4, n_pages=where.numel() // size, cache=cache)
            q = layer.rope_append(plan, qkv, where)
            results.append((q, layer.window_attention(plan, q, where), where[at * size:]))
        assert all(torch.equal(a, b) for a, b in zip(*results))


def test_a_step_repeats_itself_and_captured_steps_too(lib):
    import torch
    layer = make_layer(lib, 8, 2, 128)
    batch = make_batch([(1, 3000), (1, 2000), (1, 7), (300, 500)])
    plan, q, pool, out = attention(lib, layer, 64, batch, 100_000, 0)
    again = torch.empty_like(out)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        layer.window_attention(plan, q, pool, out=again, stream=side)
    for _ in range(3):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, out)
        assert torch.equal(layer.window_attention(plan, q, pool), out)
    q2 = torch.randn_like(q)
    want = layer.window_attention(plan, q2, pool)
    q.copy_(q2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, want)


def test_shared_rows_repeat_themselves_in_a_graph_and_in_place(lib):
    import torch
    layer = make_layer(lib, 48, 8, 128)
    batch = make_batch([(400 + i, 900 + 7 * i) for i in range(4)] + [(1, 200)])
    for group in (128, 64):
        plan, q, pool, out = attention(lib, layer, group, batch, 100_000, 0, rows_checked=8)
        assert plan.division().wide_blocks > 0
        again, graph, side = torch.empty_like(out), torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            layer.window_attention(plan, q, pool, out=again, stream=side)
        for _ in range(3):
            again.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(again, out) and torch.equal(layer.window_attention(plan, q, pool), out)
        assert torch.equal(layer.window_attention(plan, q, pool, out=q), out)


def test_plans_of_either_cache_in_turn(lib):
    import torch
    layer, rng = make_layer(lib, 8, 2, 64), np.random.default_rng(5)
    batch, cache = make_batch([(1, 200), (3, 50)]), lib.Kv4(64)
    k, v = (_bits(rng, (batch.n_pages, 16, 2, 64)) for _ in range(2))
    kept = [_kept_bits(W.bf16_bits_to_f32(x), 64) for x in (k, v)]
    q = to_gpu(_bits(rng, (batch.n_rows, 512)))
    four, sixteen = layer.window_plan(batch, 77, 3, cache=cache), layer.window_plan(batch, 77, 3)
    pool4, pool16 = layer.kv4_pack(to_gpu(k), to_gpu(v), cache), layer.pack_pool(*kept)
    a, b = layer.window_attention(four, q, pool4), layer.window_attention(sixteen, q, pool16)
    torch.cuda.synchronize()
    assert np.linalg.norm(to_host(a) - to_host(b)) < 8e-3 * np.linalg.norm(to_host(b))   # (either is below 5e-3 from what it has)
    with pytest.raises(ValueError, match="pool"):
        layer.window_attention(four, q, pool16)
    with pytest.raises(ValueError, match="pool"):
        layer.window_attention(sixteen, q, pool4)
    four.update(make_batch([(2, 30)]), 10)
    assert four.cache == cache and torch.isfinite(layer.window_attention(four, q[:2], pool4)).all()


# ---- append --------------------------------------------------------------------------------------
def append(lib, layer, group, batch, seed=0, positions=None, axis=None, in_place=False, spoil=False):
    """Turns and appends a step's rows; checks queries, the new tokens, and that nothing else moved."""
    import torch
    shape, cache = layer.shape, lib.Kv4(group)
    hq, hkv, dh = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    rng = np.random.default_rng([seed, 9])
    old = [_bits(rng, (batch.n_pages, 16, hkv, dh)) for _ in range(2)]
    pool = layer.kv4_pack(*(to_gpu(x) for x in old), cache)
    before = pool.clone()
    held = [to_host(x) for x in layer.kv4_unpack(pool, cache)]
    width = (hq + 2 * hkv) * dh
    x = _bits(rng, (batch.n_rows, width + 24))
    if spoil:
        x[1, (hq + 1) * dh - 1], x[2, width - 5] = 0x7FC0, 0x7F80
    xt = to_gpu(x)
    plan = layer.window_plan(batch, 5, 0, positions=positions, axis_of_pair=axis, cache=cache)
    q = layer.rope_append(plan, xt[:, :width], pool, q=xt[:, :hq * dh] if in_place else None)
    torch.cuda.synchronize()
    # positions, angles and products as they are defined: angles in 64 bits, rounded to 32; products and sums in 32 bits
    seq = np.repeat(np.arange(batch.n_seq), np.diff(batch.row_start))
    at = batch.kv_len[seq] - batch.row_start[seq + 1] + np.arange(batch.n_rows)
    where = np.maximum(at, 0)[None] if positions is None else np.asarray(positions)
    ax = np.zeros(dh // 2, dtype=np.int64) if axis is None else np.asarray(axis)
    angle = where[ax].T * shape.rope_theta ** (-2.0 * np.arange(dh // 2) / dh)
    cos, sin = np.cos(angle).astype(np.float32)[:, None], np.sin(angle).astype(np.float32)[:, None]
    f = W.bf16_bits_to_f32(x)[:, :width].reshape(batch.n_rows, -1, dh)
    lo, hi = f[:, :hq + hkv, :dh // 2], f[:, :hq + hkv, dh // 2:]
    with np.errstate(invalid="ignore"):
        turned = np.concatenate([lo * cos - hi * sin, hi * cos + lo * sin], axis=-1)
    ref = turned[:, :hq].reshape(batch.n_rows, -1).astype(np.float64)
    assert np.all(np.abs(to_host(q) - ref) <= U * np.abs(ref) + 1e-5)
    new = [turned[:, hq:], f[:, hq + hkv:]]
    touched = np.zeros((batch.n_pages, 16), dtype=bool)
    for r in np.flatnonzero(at >= 0):
        page, slot = int(batch.page_ids[batch.page_start[seq[r]] + at[r] // 16]), int(at[r]) % 16
        touched[page, slot] = True
        for have, fresh in zip(held, new):
            have[page, slot] = OB.kv4_values(fresh[r], group)[0]
    for got, want, kind in zip(layer.kv4_unpack(pool, cache), held, "kv"):
        got = to_host(got)
        near = W.bf16_bits_to_f32(W.f32_to_bf16_bits(want.astype(np.float32)))
        other = ~_equal_or_nan(got, near)
        assert not other[~touched].any(), "%s: a token of no row moved" % kind
        if kind == "v":
            assert not other.any()
        else:
            # an angle that another library rounds the other way moves a key by 2^-24, and a code at a border by one
            assert other.mean() < 1e-4 and np.nanmax(np.abs(got - near)) < 0.7 * np.nanmax(np.abs(near)), (other.sum(), np.nanmax(np.abs(got - near)))
    pages = touched.any(axis=1)
    assert torch.equal(pool.view(batch.n_pages, -1)[torch.from_numpy(~pages)], before.view(batch.n_pages, -1)[torch.from_numpy(~pages)])
    return plan, pool


@pytest.mark.parametrize("hq,hkv,dh,group", SHAPES)
def test_append(lib, hq, hkv, dh, group):
    layer = make_layer(lib, hq, hkv, dh)
    seqs = [(1, 1), (1, 16), (1, 17), (2, 40), (3, 3), (5, 21), (8, 8), (9, 24), (16, 16), (40, 77), (130, 131), (4, 2), (1, 0), (0, 9), (7, 120)]
    append(lib, layer, group, make_batch(seqs, seed=dh), seed=hq)
    append(lib, layer, group, make_batch([(1, 30 + 3 * i) for i in range(21)], seed=1), seed=hq, in_place=True)


@pytest.mark.parametrize("dh,group", [(128, 64), (64, 32)])
def test_append_with_axes_and_what_is_no_number(lib, dh, group):
    layer, rng = make_layer(lib, 8, 2, dh), np.random.default_rng(dh)
    batch = make_batch([(20, 45), (1, 18), (6, 6)])
    positions = rng.integers(0, 9000, (3, batch.n_rows))
    for axis in (np.arange(dh // 2) % 3, np.searchsorted([8, 24, dh // 2], np.arange(dh // 2), side="right")):
        append(lib, layer, group, batch, positions=positions, axis=axis)
    append(lib, layer, group, batch, spoil=True)


def test_append_then_attend_over_many_steps(lib):
    # a stream that grows by one token and by runs, over pages that it fills in turn, against a cache made at once
    import torch
    layer, cache, rng = make_layer(lib, 8, 2, 128), lib.Kv4(64), np.random.default_rng(2)
    width, total = 12 * 128, 90
    x = to_gpu(_bits(rng, (total, width)))
    once = make_batch([(total, total)])
    pool = torch.full((once.n_pages * layer.page_bytes(cache),), 0xFF, dtype=torch.uint8, device="cuda")
    whole = pool.clone()
    q_all = layer.rope_append(layer.window_plan(once, 1, cache=cache), x, whole)
    at, plan = 0, None
    for n in (1, 1, 13, 3, 16, 1, 29, 26):
        batch = make_batch([(n, at + n)])
        batch.page_ids, batch.n_pages = once.page_ids[:-(-(at + n) // 16)], once.n_pages
        plan = layer.window_plan(batch, 1000, 0, cache=cache)
        q = layer.rope_append(plan, x[at:at + n], pool)
        at += n
        assert torch.equal(q, q_all[at - n:at])
        out = layer.window_attention(plan, q, pool)
        assert torch.isfinite(out).all()
    a, b = layer.kv4_unpack(pool, cache), layer.kv4_unpack(whole, cache)
    for s, t in zip(a, b):
        ids = torch.from_numpy(once.page_ids.astype(np.int64)).cuda()
        assert torch.equal(s[ids].flatten(0, 1)[:total], t[ids].flatten(0, 1)[:total])
    last = layer.window_plan(once, 1000, 0, cache=cache)
    full = layer.window_attention(last, q_all, whole)
    assert (full[-26:].float() - out.float()).norm() < 8e-3 * out.float().norm()


# ---- pages ---------------------------------------------------------------------------------------
def test_copies_and_compaction(lib):
    import torch
    layer, cache = make_layer(lib, 8, 2, 64), lib.Kv4(32)
    size = layer.page_bytes(cache)
    pools = torch.randint(0, 256, (3, 20 * size), dtype=torch.uint8, device="cuda")
    want = pools.view(3, 20, size).clone()
    layer.copy_pages(pools, [3, 3, 7], [11, 0, 19], cache=cache)
    want[:, [11, 0, 19]] = want[:, [3, 3, 7]]
    torch.cuda.synchronize()
    assert torch.equal(pools.view(3, 20, size), want)
    tables, live = layer.compact_pages(list(pools), np.array([19, -1, 2, 5, 19, 17]), cache=cache)
    torch.cuda.synchronize()
    assert live == 4 and list(tables) == [3, -1, 2, 0, 3, 1]
    for old, new in zip([19, 2, 5, 17], [tables[0], tables[2], tables[3], tables[5]]):
        assert torch.equal(pools.view(3, 20, size)[:, new], want[:, old])


@pytest.mark.parametrize("hq,hkv,dh,group", SHAPES)
def test_appended_keys_by_their_own_scale(lib, hq, hkv, dh, group):
    """Every key of a step where it belongs.  What is kept is within half a scale of the turned key, and rounded to bf16 when it is read back; the
    reference's angles may be off by the last of 24 bits, which moves the turned key by 2^-23 of its two terms, and what is kept by no more than both halves."""
    import torch
    layer, cache, rng = make_layer(lib, hq, hkv, dh), lib.Kv4(group), np.random.default_rng([hq, dh, group])
    batch = make_batch([(1, 1), (1, 16), (2, 40), (5, 21), (9, 24), (16, 16), (40, 77), (130, 131), (4, 2), (0, 9), (1, 100)], seed=group)
    x = _bits(rng, (batch.n_rows, (hq + 2 * hkv) * dh))
    x[7, (hq + 1) * dh - 1] = 0x7FC0
    pool = torch.zeros(batch.n_pages * layer.page_bytes(cache), dtype=torch.uint8, device="cuda")
    layer.rope_append(layer.window_plan(batch, 5, 0, cache=cache), to_gpu(x), pool)
    got = to_host(layer.kv4_unpack(pool, cache)[0])
    seq = np.repeat(np.arange(batch.n_seq), np.diff(batch.row_start))
    at = batch.kv_len[seq] - batch.row_start[seq + 1] + np.arange(batch.n_rows)
    angle = np.maximum(at, 0)[:, None] * layer.shape.rope_theta ** (-2.0 * np.arange(dh // 2) / dh)
    cos, sin = np.cos(angle).astype(np.float32)[:, None], np.sin(angle).astype(np.float32)[:, None]
    key = W.bf16_bits_to_f32(x).reshape(batch.n_rows, -1, dh)[:, hq:hq + hkv]
    lo, hi = key[..., :dh // 2], key[..., dh // 2:]
    with np.errstate(invalid="ignore"):
        turned = np.concatenate([lo * cos - hi * sin, hi * cos + lo * sin], axis=-1)
        moves = 2.0 ** -23 * np.concatenate([np.abs(lo * cos) + np.abs(hi * sin), np.abs(hi * cos) + np.abs(lo * sin)], axis=-1)
    rows = np.flatnonzero(at >= 0)
    pages = batch.page_ids[batch.page_start[seq[rows]] + at[rows] // 16]
    have, near = got[pages, at[rows] % 16], W.bf16_bits_to_f32(_kept_bits(turned[rows], group)).astype(np.float64)
    assert np.array_equal(np.isnan(have), np.isnan(near)) and np.isnan(near).sum() == min(2 * group, dh)   # (a pair's two channels)
    scale = np.repeat(OB.kv4_numbers(turned[rows], group)[0].astype(np.float64), group, axis=-1)
    bound = scale * (1 + U) + U / 2 * (np.abs(have) + np.abs(near)) + 2 * moves[rows]
    wrong = ~(np.abs(have - near) <= bound) & ~np.isnan(near)
    assert not wrong.any(), "%d of %d" % (wrong.sum(), wrong.size)
    assert (~_equal_or_nan(have, near)).sum() <= max(group, 1e-4 * near.size)
    touched = np.zeros(got.shape[:2], dtype=bool)
    touched[pages, at[rows] % 16] = True
    assert (got[~touched] == 0).all()

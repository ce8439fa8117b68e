"""The stream operators on the GPU against float64 definitions.

Tolerances, from the arithmetic: an output is rounded to bf16 once (8 significant bits: relative 2^-8).  Attention: each probability is
rounded to bf16 before its product with V, which moves an output by at most 2^-8 of the sum of p |v|; scores, exponentials and
sums in 32 bits stay below 1e-5 of it.  Rotary: two products and a sum in 32 bits, angles rounded to 32 bits: 1e-6 of the
pair.  4-bit products: sums of k terms in 32 bits, terms of size |x| (128 + w) scale: 2^-24 of their sum for each of the steps
that a term passes through (at most 128 in its group and one for each group)."""
import numpy as np
import pytest

from oracle import stream as OS
from paper_2411_16102_amd import workloads as W
from stream_cases import make_batch

pytestmark = pytest.mark.gpu
U = 2.0 ** -8   # unit roundoff of bf16: 1 + 2^-8 lies halfway between 1 and its neighbour 1 + 2^-7


def _bits(rng, shape, scale=1.0):
    return W.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


def _tokens(batch, s, pool, n):
    """Tokens 0 .. n - 1 of sequence s of a token-major array [n_pages, 16, ...] (pages that were given up: NaN)."""
    ids = batch.page_ids[batch.page_start[s]:batch.page_start[s] + -(-n // 16)]
    out = pool[np.maximum(ids, 0)].copy()
    out[ids < 0] = np.nan
    return out.reshape((-1,) + pool.shape[2:])[:n]


def _attention(lib, shape, batch, window, sinks, seed=0, poison=True, layer=None, q_stride=None):
    import torch
    rng = np.random.default_rng([seed, 3])
    layer = layer or lib.Layer(shape, device=0)
    width = shape.n_q_heads * shape.head_dim
    kv = (batch.n_pages, 16, shape.n_kv_heads, shape.head_dim)
    k, v = _bits(rng, kv), _bits(rng, kv)
    if poison:
        # what no row sees holds NaN and infinities: slots past the context, pages of nobody, tokens between sinks and windows
        used = np.zeros((batch.n_pages, 16), dtype=bool)
        for s in range(batch.n_seq):
            n, rows = int(batch.kv_len[s]), int(batch.row_start[s + 1] - batch.row_start[s])
            p, t = np.arange(n - rows, n)[:, None], np.arange(n)
            seen = np.flatnonzero(((t <= p) & ((t > p - window) | (t < sinks))).any(axis=0))
            used[batch.page_ids[batch.page_start[s] + seen // 16], seen % 16] = True
        k[~used], v[~used] = 0x7FC0, 0xFF80
    pool = layer.pack_pool(k, v)
    q = _bits(rng, (batch.n_rows, q_stride or width))
    qt = torch.from_numpy(q.view(np.int16)).cuda().view(torch.bfloat16)[:, :width]
    plan = layer.window_plan(batch, window, sinks)
    out = layer.window_attention(plan, qt, pool)
    torch.cuda.synchronize()
    got = out.float().cpu().numpy().astype(np.float64)
    kf, vf, qf = W.bf16_bits_to_f32(k), W.bf16_bits_to_f32(v), W.bf16_bits_to_f32(q)[:, :width]
    for s in range(batch.n_seq):
        a, b, n = int(batch.row_start[s]), int(batch.row_start[s + 1]), int(batch.kv_len[s])
        if a == b:
            continue
        K, V = _tokens(batch, s, kf, n), _tokens(batch, s, vf, n)
        ref, weight = OS.window_attention(qf[a:b].reshape(b - a, shape.n_q_heads, -1), K, V, n - (b - a), window, sinks)
        err = np.abs(got[a:b].reshape(ref.shape) - ref)
        bound = U * (np.abs(ref) + weight) * 1.01 + 1e-5 * weight
        assert np.all(err <= bound), "sequence %d (%d rows, %d tokens): %.3g over the bound" % (s, b - a, n, np.nanmax(err - bound))
        print("sequence %d: %d rows of %d tokens, error over bound %.2f" % (s, b - a, n, float(np.max(err / np.maximum(bound, 1e-30)))))
    return layer, plan, qt, pool, out


HEADS = [(8, 2, 64), (8, 2, 128), (4, 4, 64), (16, 1, 128), (6, 2, 128), (10, 2, 64), (3, 1, 64), (14, 2, 128)]


@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_single_tokens(lib, hq, hkv, dh):
    shape = W.LayerShape(256, hq, hkv, dh, 256)
    batch = make_batch([(1, n) for n in (1, 2, 15, 16, 17, 32, 33, 100, 0, 129, 300)], seed=hq)
    for window, sinks in ((1, 0), (16, 0), (37, 5), (1000, 0), (20, 16)):
        _attention(lib, shape, batch, window, sinks, seed=window)


@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_rows_of_every_count(lib, hq, hkv, dh):
    # padding in front (kv_len below the rows), sequences without rows, a few rows, chunks behind cached tokens
    shape = W.LayerShape(256, hq, hkv, dh, 256)
    batch = make_batch([(3, 40), (0, 30), (5, 3), (17, 90), (2, 200), (70, 70), (66, 150), (4, 0), (9, 9)], seed=dh)
    for window, sinks in ((33, 3), (1, 0), (50, 70)):
        _attention(lib, shape, batch, window, sinks, seed=window)


@pytest.mark.parametrize("window,sinks", [(1, 1), (2, 31), (15, 16), (31, 0), (64, 33), (65, 1), (128, 0), (1 << 30, 1 << 30), (100, 1000)])
def test_edges_of_windows_and_sinks(lib, window, sinks):
    shape = W.LayerShape(256, 8, 2, 128, 256)
    _attention(lib, shape, make_batch([(1, 500), (130, 300), (1, 64), (90, 95), (3, 222)], seed=sinks % 97), window, sinks)


@pytest.mark.parametrize("hq,hkv,dh", [(8, 2, 128), (4, 4, 64)])
def test_long_contexts_are_split_and_joined(lib, hq, hkv, dh):
    shape = W.LayerShape(256, hq, hkv, dh, 256)
    layer, plan, *_ = _attention(lib, shape, make_batch([(1, 3000), (2, 2500), (1, 5)]), 2000, 40)
    assert plan.division().split_rows == 3


WIDE = [(8, 2, 128), (4, 4, 64), (12, 2, 64), (6, 2, 128), (16, 1, 64)]


@pytest.mark.parametrize("hq,hkv,dh", [h for h in WIDE if h[0] != h[1]])
def test_blocks_of_rows(lib, hq, hkv, dh):
    # enough rows that blocks of them are the shorter way: odd lengths, windows that begin in the chunk, before it and
    # before the sequence, rows in front of it
    shape = W.LayerShape(256, hq, hkv, dh, 256)
    batch = make_batch([(700 + 13 * i, 900 + 101 * i) for i in range(7)] + [(230, 100), (700, 700), (629, 629)], seed=hq, spare=200)
    for window, sinks in ((150, 20), (333, 0), (900, 4), (10_000, 3), (17, 100)):
        _, plan, *_ = _attention(lib, shape, batch, window, sinks, seed=window, poison=window < 500)
        assert plan.division().wide_blocks >= 29


@pytest.mark.parametrize("hq,hkv,dh", WIDE)
def test_blocks_of_rows_cut_into_ranges(lib, hq, hkv, dh):
    shape = W.LayerShape(256, hq, hkv, dh, 256)
    for seqs, window, sinks in (([(257, 4500), (260, 4400)], 3001, 1000), ([(600, 6100)], 5000, 50)):
        _, plan, *_ = _attention(lib, shape, make_batch(seqs, seed=dh), window, sinks, seed=window)
        assert plan.division().wide_cut >= 3


@pytest.mark.parametrize("hq,hkv,dh", WIDE)
def test_blocks_and_units_in_one_launch(lib, hq, hkv, dh):
    shape = W.LayerShape(256, hq, hkv, dh, 256)
    seqs = [(850 + i, 1700 + 90 * i) for i in range(6)] + [(1, n) for n in (1, 0, 500, 2000, 900, 33, 64)] * 3 + [(3, 1000), (2, 1), (0, 77)]
    for window, sinks in ((1500, 0),) if hq == hkv else ((400, 4), (1500, 0)):
        _, plan, *_ = _attention(lib, shape, make_batch(seqs, seed=hkv), window, sinks, seed=window, poison=window < 500)
        d = plan.division()
        assert d.wide_blocks >= 24 and d.units >= 20


@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 8, 64)])
def test_streams_shared_by_wavefronts(lib, heads):
    # numbers of streams and windows for which a unit's pages are shared by one, two, four and eight wavefronts, whole and cut
    shape = W.LayerShape(256, *heads, 256)
    for n, ctx, window in ((200, 60, 20), (40, 700, 500), (150, 2100, 2000), (90, 2500, 2300), (1, 5000, 4800), (3, 4000, 100_000)):
        _attention(lib, shape, make_batch([(1, ctx - 7 * (i % 9)) for i in range(n)], seed=n), window, 9, poison=n < 50)


def test_pages_given_up_and_strided_rows(lib):
    shape = W.LayerShape(256, 8, 2, 64, 256)
    batch = make_batch([(1, 1000), (40, 900)], given_up={0: range(2, 56), 1: range(2, 46)})
    _attention(lib, shape, batch, 100, 20, q_stride=8 * 64 + 2 * 2 * 64)


def test_steps_without_rows(lib):
    import torch
    layer, _, _, _, out = _attention(lib, W.LayerShape(256, 3, 1, 64, 256), make_batch([(0, 40), (0, 0)]), 16, 2)
    assert tuple(out.shape) == (0, 192)
    plan = layer.window_plan(make_batch([], spare=0), 16, 2)
    pool = torch.zeros(0, device="cuda", dtype=torch.bfloat16)
    assert layer.rope_append(plan, torch.zeros((0, 5 * 64), device="cuda", dtype=torch.bfloat16), pool).shape == (0, 192)


def test_in_place_and_strided_results_equal(lib):
    import torch
    shape = W.LayerShape(256, 8, 2, 64, 256)
    layer, plan, q, pool, want = _attention(lib, shape, make_batch([(1, 700), (100, 300), (1, 0)]), 90, 4)
    wide = torch.full((q.shape[0], q.shape[1] + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    layer.window_attention(plan, q, pool, out=wide[:, :q.shape[1]])
    assert torch.equal(wide[:, :q.shape[1]], want) and bool((wide[:, q.shape[1]:] == 7.0).all())
    mine = q.clone()
    layer.window_attention(plan, mine, pool, out=mine)
    assert torch.equal(mine, want)


def test_large_scores_and_equal_scores(lib):
    # scores of some hundreds (the running maximum moves in every block), and a query of zeros (all weights equal)
    import torch
    shape = W.LayerShape(256, 8, 2, 128, 256)
    layer = lib.Layer(shape, device=0)
    batch = make_batch([(1, 800), (80, 200)])
    rng = np.random.default_rng(4)
    k, v = _bits(rng, (batch.n_pages, 16, 2, 128), 30.0), _bits(rng, (batch.n_pages, 16, 2, 128))
    pool = layer.pack_pool(k, v)
    plan = layer.window_plan(batch, 150, 3)
    for scale in (3.0, 0.0):
        q = _bits(rng, (batch.n_rows, 8 * 128), scale)
        got = layer.window_attention(plan, torch.from_numpy(q.view(np.int16)).cuda().view(torch.bfloat16), pool).double().cpu().numpy()
        for s, (a, b) in enumerate(((0, 1), (1, 81))):
            n = int(batch.kv_len[s])
            K, V = (_tokens(batch, s, W.bf16_bits_to_f32(x), n) for x in (k, v))
            ref, weight = OS.window_attention(W.bf16_bits_to_f32(q[a:b]).reshape(b - a, 8, 128), K, V, n - (b - a), 150, 3)
            # a score of size s is a sum of 128 products in 32 bits: its exponential is off by 2^-24 * 8 * |s| and the scale's rounding
            smax = np.abs(W.bf16_bits_to_f32(q)).max() * np.abs(W.bf16_bits_to_f32(k)).max() * 128 ** 0.5
            assert np.all(np.abs(got[a:b].reshape(ref.shape) - ref) <= U * (np.abs(ref) + weight) * 1.01 + 2.0 ** -24 * 16 * smax * weight + 1e-5 * weight)


def test_offsets_past_32_bits(lib):
    # pages behind 2^32 bytes of a pool
    import torch
    shape = W.LayerShape(256, 8, 8, 128, 256)
    layer = lib.Layer(shape, device=0)
    size = layer.page_bytes() // 2
    n_pages = 140_000
    assert size * n_pages > 1 << 32
    pool = torch.zeros(n_pages * size, dtype=torch.bfloat16, device="cuda")
    for rows, kv in ((1, 50), (70, 90)):
        batch = make_batch([(rows, kv)])
        n = -(-kv // 16)
        batch.page_ids = (n_pages - 1 - np.arange(n)).astype(np.int32)
        batch.n_pages = n_pages
        rng = np.random.default_rng(rows)
        k, v = _bits(rng, (n, 16, 8, 128)), _bits(rng, (n, 16, 8, 128))
        small = layer.pack_pool(k, v).view(n, size)
        pool.view(n_pages, size)[torch.from_numpy(batch.page_ids.astype(np.int64)).cuda()] = small
        q = _bits(rng, (rows, 1024))
        qt = torch.from_numpy(q.view(np.int16)).cuda().view(torch.bfloat16)
        near = make_batch([(rows, kv)])
        near.page_ids, near.n_pages = np.arange(n, dtype=np.int32), n
        want = layer.window_attention(layer.window_plan(near, 40, 3), qt, small.reshape(-1))
        assert torch.equal(layer.window_attention(layer.window_plan(batch, 40, 3), qt, pool), want)
        # the same for what is appended and copied there
        qkv = torch.randn((rows, 8 * 128 * 3), device="cuda").to(torch.bfloat16)
        p1, p2 = layer.window_plan(near, 40, 3), layer.window_plan(batch, 40, 3)
        assert torch.equal(layer.rope_append(p1, qkv, small.view(-1)), layer.rope_append(p2, qkv, pool))
        assert torch.equal(pool.view(n_pages, size)[torch.from_numpy(batch.page_ids.astype(np.int64)).cuda()], small)
    src, dst = batch.page_ids, np.arange(n, dtype=np.int32)
    layer.copy_pages([pool], src, dst)
    assert torch.equal(pool.view(n_pages, size)[:n], small)


# ---- rotary positions and append ---------------------------------------------------------------
@pytest.mark.parametrize("hq,hkv,dh", [(8, 2, 64), (4, 4, 128), (16, 1, 128), (3, 1, 64), (32, 8, 128)])
@pytest.mark.parametrize("axes,mixed", [(0, False), (1, False), (2, True), (3, False), (3, True), (8, True)])
def test_rope_append(lib, hq, hkv, dh, axes, mixed):
    import torch
    rng = np.random.default_rng([hq, axes])
    shape = W.LayerShape(256, hq, hkv, dh, 256)
    layer = lib.Layer(shape, device=0)
    batch = make_batch([(1, 33), (40, 57), (5, 2), (1, 0), (0, 20), (16, 16), (33, 300), (1, 16)], seed=axes)
    rows, half = batch.n_rows, dh // 2
    pad = 16 if mixed else 0
    x = _bits(rng, (rows, (hq + 2 * hkv) * dh + pad))
    qkv = torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)[:, :(hq + 2 * hkv) * dh]
    at = np.concatenate([np.arange(n - q, n) for q, n in zip(batch.q_len(), batch.kv_len)])
    if axes:
        pos = rng.integers(0, 16384, (axes, rows)).astype(np.int32)
        axis = rng.integers(0, axes, half).astype(np.int32) if mixed else (np.arange(half) * axes // half).astype(np.int32)
    else:
        pos, axis = np.maximum(at, 0)[None], np.zeros(half, dtype=np.int32)
    k0, v0 = _bits(rng, (batch.n_pages, 16, hkv, dh)), _bits(rng, (batch.n_pages, 16, hkv, dh))
    pool = layer.pack_pool(k0, v0)
    plan = layer.window_plan(batch, 8, 0, *((pos, axis) if axes else ()))
    q = layer.rope_append(plan, qkv, pool)
    torch.cuda.synchronize()
    k1, v1 = (t.float().cpu().numpy() for t in layer.unpack_pool(pool, batch.n_pages))
    f = W.bf16_bits_to_f32(x)[:, :(hq + 2 * hkv) * dh].reshape(rows, -1, dh)
    want = OS.rope_axes(f[:, :hq + hkv], pos, axis, shape.rope_theta)
    pair = np.abs(f[:, :hq + hkv, :half]) + np.abs(f[:, :hq + hkv, half:])
    bound = U * np.abs(want) * 1.01 + 1e-6 * np.concatenate([pair, pair], axis=-1)
    got = q.float().cpu().numpy().reshape(rows, hq, dh)
    assert np.all(np.abs(got - want[:, :hq]) <= bound[:, :hq])
    kw, vw = W.bf16_bits_to_f32(k0), W.bf16_bits_to_f32(v0)
    seq = np.repeat(np.arange(batch.n_seq), batch.q_len())
    for r in range(rows):
        if at[r] < 0:
            continue
        page, slot = batch.page_ids[batch.page_start[seq[r]] + at[r] // 16], at[r] % 16
        assert np.all(np.abs(k1[page, slot] - want[r, hq:]) <= bound[r, hq:])
        assert np.array_equal(v1[page, slot], f[r, hq + hkv:])
        kw[page, slot], vw[page, slot] = k1[page, slot], v1[page, slot]
    assert np.array_equal(kw, k1) and np.array_equal(vw, v1), "a slot changed that no row appends to"
    # in place
    layer.rope_append(plan, qkv, pool, q=qkv[:, :hq * dh])
    assert torch.equal(qkv[:, :hq * dh], q)
    left = qkv[:, hq * dh:].float().cpu().numpy().reshape(rows, -1, dh)
    assert np.array_equal(left, f[:, hq:])


# ---- 4-bit products -------------------------------------------------------------------------------
def _w4(lib, m, n, k, group, zeros, seed=0, mean=0.0, layer=None, pad=0):
    import torch
    rng = np.random.default_rng([seed, m, n, k])
    layer = layer or lib.Layer(W.TINY, device=0)
    x = _bits(rng, (m, k + pad))
    if mean:
        x = W.f32_to_bf16_bits((mean + W.bf16_bits_to_f32(x)).astype(np.float32))
    w = rng.integers(0, 16, (n, k)).astype(np.uint8)
    s = W.f32_to_bf16_bits((0.02 * rng.standard_normal((n, k // group))).astype(np.float32))
    z = rng.integers(0, 16, (n, k // group)).astype(np.uint8) if zeros else None
    weight = layer.w4_pack(torch.from_numpy(w[:, 0::2] | (w[:, 1::2] << 4)).cuda(), torch.from_numpy(s.view(np.int16)).cuda().view(torch.bfloat16),
                           torch.from_numpy(z).cuda() if zeros else None)
    xt = torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)[:, :k]
    y = layer.w4_linear(xt, weight)
    xf, sf = W.bf16_bits_to_f32(x)[:, :k].astype(np.float64), W.bf16_bits_to_f32(s).astype(np.float64)
    ref = OS.w4_linear(xf, w, sf, z)
    terms = np.abs(xf) @ (np.repeat(np.abs(sf), group, axis=1) * (128 + 15 + 16 + w)).T
    bound = U * np.abs(ref) * 1.01 + 2.0 ** -24 * (128 + k // group) * terms
    got = y.float().cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - ref) <= bound)
    norm = np.linalg.norm(ref)
    if norm and not mean:
        assert np.linalg.norm(got - ref) <= 1.05 * U * norm
    return layer, weight, xt, y


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("m,n,k", [(1, 16, 128), (1, 1, 128), (2, 17, 256), (5, 100, 384), (16, 64, 1024), (17, 130, 640), (33, 515, 256), (64, 96, 512),
                                   (65, 40, 128), (130, 33, 384), (1, 6144, 4096), (7, 2000, 3840), (40, 1000, 4480)])
def test_w4_linear(lib, m, n, k, group, zeros):
    _w4(lib, m, n, k, group, zeros)


@pytest.mark.parametrize("m,n,k,group,zeros", [(1, 33000, 256, 128, True), (9, 32785, 384, 64, False), (30, 40003, 160, 32, True), (40, 32800, 640, 128, False),
                                               (61, 33001, 384, 64, True), (61, 32900, 1280, 64, False), (130, 16500, 384, 128, True)])
def test_w4_more_tiles_than_cus(lib, m, n, k, group, zeros):
    _w4(lib, m, n, k, group, zeros)


@pytest.mark.parametrize("m,n,k,group,zeros", [(16, 16500, 4992, 128, True), (30, 8210, 4896, 32, False), (40, 6203, 5120, 64, False), (61, 4200, 5120, 64, True)])
def test_w4_tiles_that_share_outputs(lib, m, n, k, group, zeros):
    _w4(lib, m, n, k, group, zeros)


@pytest.mark.parametrize("m,k", [(16, 4736), (16, 4864), (9, 8448), (9, 8576), (1, 76800), (1, 76928)])
def test_w4_rows_that_fill_the_lds(lib, m, k):
    _w4(lib, m, 35, k, 128, True)


@pytest.mark.parametrize("n", [16 * 255 + 1, 16 * 256 + 1, 16 * 512 + 1, 16 * 1024 + 16, 16 * 2048, 16 * 2048 + 1])
@pytest.mark.parametrize("m,k,group", [(1, 384, 128), (9, 544, 32), (16, 256, 64), (17, 320, 64)])
def test_w4_blocks_of_a_cu(lib, n, m, k, group):
    _w4(lib, m, n, k, group, n % 2 == 1)


@pytest.mark.parametrize("m,k", [(8, 8192), (8, 8320), (3, 21888), (1, 65536), (1, 65664)])
def test_w4_inputs_that_just_fit(lib, m, k):
    _w4(lib, m, 70, k, 128, True)


@pytest.mark.parametrize("k,group", [(32, 32), (96, 32), (64, 64), (192, 64), (160, 32), (0, 128)])
def test_w4_inputs_that_end_inside_a_block(lib, k, group):
    _w4(lib, 3, 50, k, group, True)
    _w4(lib, 20, 50, k, group, False, pad=8)


def test_w4_inputs_with_a_mean(lib):
    # sums of x far from zero: what the offset of the operands adds is taken off again
    _w4(lib, 4, 256, 4096, 128, False, mean=3.0)


def test_w4_strided_rows_and_no_rows(lib):
    import torch
    layer, weight, x, y = _w4(lib, 9, 70, 256, 64, True, pad=40)
    wide = torch.full((9, 101), 3.0, dtype=torch.bfloat16, device="cuda")
    layer.w4_linear(x, weight, out=wide[:, 5:75])
    assert torch.equal(wide[:, 5:75], y) and bool((wide[:, :5] == 3.0).all()) and bool((wide[:, 75:] == 3.0).all())
    assert layer.w4_linear(x[:0], weight).shape == (0, 70)


# ---- copies of pages -------------------------------------------------------------------------------
@pytest.mark.parametrize("hkv,dh,layers,n", [(2, 64, 1, 1), (8, 128, 3, 40), (1, 64, 32, 7), (4, 128, 2, 700)])
def test_copy_pages(lib, hkv, dh, layers, n):
    import torch
    layer = lib.Layer(W.LayerShape(256, hkv, hkv, dh, 256), device=0)
    size, n_pages = layer.page_bytes() // 2, 2 * n + 5
    gen = torch.Generator(device="cuda").manual_seed(n)
    pools = torch.randn((layers, n_pages * size), device="cuda", generator=gen).to(torch.bfloat16)
    order = np.random.default_rng(n).permutation(n_pages)
    src, dst = order[:n], order[n:2 * n]
    src[n // 2:] = src[0]                       # several copies of one page
    want = pools.clone().view(layers, n_pages, size)
    want[:, torch.from_numpy(dst).cuda()] = want[:, torch.from_numpy(src).cuda()]
    layer.copy_pages(pools, src, dst)
    assert torch.equal(pools.view(want.shape), want)
    layer.copy_pages([pools[0]], [], [])
    assert torch.equal(pools.view(want.shape), want)


@pytest.mark.parametrize("live", [0.0, 0.1, 0.6, 1.0])
def test_compact_pages(lib, live):
    import torch
    layer = lib.Layer(W.LayerShape(256, 2, 2, 64, 256), device=0)
    size, n_pages = layer.page_bytes() // 2, 300
    rng = np.random.default_rng(int(10 * live))
    named = rng.permutation(n_pages)[:int(live * n_pages)]
    tables = rng.permutation(np.concatenate([named, named[:len(named) // 3], [-1, -1]])).astype(np.int32)
    pools = torch.randn((2, n_pages * size), device="cuda").to(torch.bfloat16)
    before = pools.clone().view(2, n_pages, size)
    new, count = layer.compact_pages(pools, tables)
    assert count == len(named) and np.array_equal(new < 0, tables < 0) and (count == 0 or new.max() == count - 1)
    at = tables >= 0
    assert torch.equal(pools.view(before.shape)[:, torch.from_numpy(new[at].astype(np.int64)).cuda()],
                       before[:, torch.from_numpy(tables[at].astype(np.int64)).cuda()])
    # what stood below the count and is named has not moved
    assert np.array_equal(new[at & (tables < count)], tables[at & (tables < count)])


# ---- refusals, streams, graphs ------------------------------------------------------------------------
def test_refusals_enqueue_nothing(lib):
    import torch
    shape = W.LayerShape(256, 8, 2, 64, 256)
    layer = lib.Layer(shape, device=0)
    batch = make_batch([(1, 40), (3, 20)])
    pool = torch.zeros(batch.n_pages * layer.page_bytes() // 2, dtype=torch.bfloat16, device="cuda")
    plan = layer.window_plan(batch, 8)
    q = torch.zeros((4, 512), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 5.0)
    raw, s = layer.lib, torch.cuda.current_stream().cuda_stream
    for args in ((None, 512, out.data_ptr(), 512, pool.data_ptr()), (q.data_ptr(), 504, out.data_ptr(), 512, pool.data_ptr()),
                 (q.data_ptr(), 516, out.data_ptr(), 512, pool.data_ptr()), (q.data_ptr() + 2, 512, out.data_ptr(), 512, pool.data_ptr()),
                 (q.data_ptr(), 512, q.data_ptr(), 520, pool.data_ptr()), (q.data_ptr(), 512, out.data_ptr(), 512, None)):
        assert raw.bs_window_attention(plan.h, *args, s) == -1
    for args in ((None, 768, out.data_ptr(), 512, pool.data_ptr()), (q.data_ptr(), 760, out.data_ptr(), 512, pool.data_ptr()),
                 (q.data_ptr(), 768, out.data_ptr(), 500, pool.data_ptr()), (q.data_ptr(), 768, q.data_ptr(), 512, pool.data_ptr())):
        assert raw.bs_rope_append(plan.h, *args, s) == -1
    with pytest.raises(ValueError):
        layer.window_attention(plan, q[:3], pool)
    with pytest.raises(ValueError):
        layer.window_attention(plan, q, pool[:100])
    with pytest.raises(ValueError):
        layer.w4_linear(q, lib.W4Weight(pool, 16, 256, 64, False))
    for src, dst, match in (([0], [99], "outside"), ([0, 1], [2, 2], "twice"), ([0, 2], [2, 3], "from and to"), ([-1], [0], "outside")):
        with pytest.raises(lib.BlendStepError, match=match):
            layer.copy_pages([pool], src, dst)
    with pytest.raises(lib.BlendStepError, match="outside the pool"):
        layer.compact_pages([pool], [0, 1, 99])
    # a row beyond the table of angles: attention runs, rotary positions are refused
    far = make_batch([(1, 16390)])
    plan2 = layer.window_plan(far, 8)
    with pytest.raises(lib.BlendStepError, match="max_positions"):
        layer.rope_append(plan2, torch.zeros((1, 768), dtype=torch.bfloat16, device="cuda"),
                          torch.zeros(far.n_pages * layer.page_bytes() // 2, dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    assert bool((out == 5.0).all())


def test_replays_of_a_captured_step(lib):
    import torch
    shape = W.LayerShape(256, 8, 2, 128, 256)
    layer = lib.Layer(shape, device=0)
    batch = make_batch([(1, 1500)] * 5 + [(1, 0), (90, 400), (2, 30)])
    gen = torch.Generator(device="cuda").manual_seed(1)
    pool = torch.randn(batch.n_pages * layer.page_bytes() // 2, device="cuda", generator=gen).to(torch.bfloat16)
    qkv = torch.randn((batch.n_rows, 12 * 128), device="cuda", generator=gen).to(torch.bfloat16)
    packed = torch.randint(0, 256, (1536, 512), dtype=torch.uint8, device="cuda", generator=gen)
    weight = layer.w4_pack(packed, torch.full((1536, 8), 0.01, dtype=torch.bfloat16, device="cuda"))
    x = torch.randn((batch.n_rows, 1024), device="cuda", generator=gen).to(torch.bfloat16)
    plan = layer.window_plan(batch, 1200, 4)
    layer.w4_linear(x, weight, out=qkv)
    want_q = layer.rope_append(plan, qkv, pool)
    want = layer.window_attention(plan, want_q, pool)
    spare = sorted(set(range(batch.n_pages)) - set(batch.page_ids.tolist()))[:1]
    torch.cuda.synchronize()
    q, out, y = torch.zeros_like(want_q), torch.zeros_like(want), torch.zeros_like(qkv)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.w4_linear(x, weight, out=y)
        layer.rope_append(plan, y, pool, q=q)
        layer.window_attention(plan, q, pool, out=out)
        layer.copy_pages([pool], [int(batch.page_ids[0])], spare)
    other = layer.window_plan(make_batch([(1, 900)]), 40)
    for i in range(4):
        for t in (q, out, y):
            t.zero_()
        pool.view(batch.n_pages, -1)[spare] = 0
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, want_q) and torch.equal(out, want) and torch.equal(y, qkv), "replay %d" % i
        assert torch.equal(pool.view(batch.n_pages, -1)[spare[0]], pool.view(batch.n_pages, -1)[int(batch.page_ids[0])])
        layer.window_attention(other, q[:1], pool)
        layer.copy_pages([pool], [int(batch.page_ids[1])], spare)
    with torch.cuda.stream(side):
        with pytest.raises(lib.BlendStepError, match="cannot be captured"):
            with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
                plan.update(batch, 1200, 4)
    torch.cuda.synchronize()


def test_calls_on_another_stream(lib):
    import torch
    shape = W.LayerShape(256, 8, 2, 128, 256)
    layer = lib.Layer(shape, device=0)
    batch = make_batch([(1, 3000), (200, 700)])
    pool = torch.randn(batch.n_pages * layer.page_bytes() // 2, device="cuda").to(torch.bfloat16)
    q = torch.randn((batch.n_rows, 1024), device="cuda").to(torch.bfloat16)
    want = layer.window_attention(layer.window_plan(batch, 2000, 4), q, pool)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(q)
    side.wait_stream(torch.cuda.current_stream())
    plan = layer.window_plan(batch, 2000, 4, stream=side)
    layer.window_attention(plan, q, pool, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)

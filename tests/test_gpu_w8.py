"""Products of 8-bit integers on the GPU against whole-number arithmetic.

Integers and scales of rows are operations in 32 bits, which numpy's float32 does too: equal bit for bit.  Sums of integers are exact; a result is
the sum rounded to 32 bits, two products in 32 bits and one rounding to bf16: relative 2^-8 and three times 2^-24."""
import numpy as np
import pytest

from oracle import bits as OB
from paper_2411_16102_amd import workloads as W

pytestmark = pytest.mark.gpu
BOUND = 2.0 ** -8 + 3 * 2.0 ** -24


@pytest.fixture(scope="module")
def layer(lib):
    return lib.Layer(W.LayerShape(256, 8, 2, 64, 256), device=0)


def to_gpu(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def _bits(rng, shape, scale=1.0):
    return W.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


def _weight(lib, rng, n, k):
    import torch
    w, s = rng.integers(-128, 128, (n, k)).astype(np.int8), (0.001 * (0.5 + rng.random(n))).astype(np.float32)
    return w, s, lib.W8Weight(torch.from_numpy(w).cuda(), torch.from_numpy(s).cuda())


def _reference(q, scale, w, s):
    # (float64 products of integers below 2^53 are exact)
    return (q.astype(np.float64) @ w.astype(np.float64).T) * scale[:, None].astype(np.float64) * s[None].astype(np.float64)


def _check(got, ref):
    got = got.float().cpu().numpy().astype(np.float64)
    same = (np.isnan(got) & np.isnan(ref)) | (np.abs(got - ref) <= BOUND * np.abs(ref) + 1e-37)
    assert same.all(), "%d of %d, worst %.3g" % ((~same).sum(), same.size, np.nanmax(np.abs(got - ref) / np.maximum(np.abs(ref), 1e-30)))


@pytest.mark.parametrize("m,k", [(1, 16), (3, 48), (5, 256), (2, 4096), (7, 8192 + 16), (1, 28672), (300, 688), (40, 1536), (300, 9232)])
def test_rows_as_integers(layer, m, k):
    rng = np.random.default_rng(m + k)
    x = W.f32_to_bf16_bits((rng.standard_normal((m, k + 8)) * np.exp(20 * rng.standard_normal((m, 1)))).astype(np.float32))
    x[0] = W.f32_to_bf16_bits(rng.integers(-64, 65, k + 8).astype(np.float32))   # halves of integers
    x[0, 0] = W.f32_to_bf16_bits(np.float32([63.5]))[0]
    if m > 3:
        x[1], x[2], x[3, k - 1] = 0, W.f32_to_bf16_bits(np.full(k + 8, 1e-37, dtype=np.float32)), 0x7FC0
    if m > 4:
        x[4, 0] = 0xFF80
    rows = layer.w8_quantize(to_gpu(x)[:, :k])
    q, scale = OB.w8_rows(W.bf16_bits_to_f32(x[:, :k]))
    got = rows.scales.cpu().numpy()
    assert np.array_equal(got, scale, equal_nan=True) and np.array_equal(rows.q.cpu().numpy(), q)


# rows up to every kernel's limit and beyond, outputs and inputs of odd numbers of tiles
@pytest.mark.parametrize("m,n,k", [(1, 256, 256), (1, 1, 16), (1, 3, 32), (2, 5000, 4096), (7, 4097, 1024), (15, 514, 8192), (16, 8192, 4096), (17, 4096, 4096),
                                   (31, 771, 2064), (33, 8192, 7168), (47, 130, 28672), (64, 6144, 4096), (65, 257, 4112), (100, 14336, 1024), (128, 4096, 14336),
                                   (129, 4096, 4096), (200, 6145, 4096), (256, 514, 16384), (300, 28672, 512), (511, 6144, 4096), (700, 999, 2000),
                                   (1093, 4096, 4096), (1500, 2050, 1040), (2560, 4096, 1536), (4100, 1030, 528)])
def test_products(lib, layer, m, n, k):
    rng = np.random.default_rng(m * n + k)
    w, s, weight = _weight(lib, rng, n, k)
    x = _bits(rng, (m, k), 3.0)
    if m > 2:
        x[1, k - 1] = 0x7F80
    q, scale = OB.w8_rows(W.bf16_bits_to_f32(x))
    ref = _reference(q, scale, w, s)
    rows = layer.w8_quantize(to_gpu(x))
    y = layer.w8_linear(rows, weight)
    _check(y, ref)
    import torch
    again = layer.w8_linear(to_gpu(x), weight)
    assert torch.equal(y.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("m,n,k,tile", [(9, 2857, 3952, (16, 16)), (1, 5123, 7728, (16, 32)), (51, 412, 4352, (32, 16)), (20, 13329, 2368, (32, 32)),
                                        (53, 15186, 2432, (64, 128)), (678, 1071, 5008, (128, 128)), (1090, 4091, 4080, (192, 128)), (845, 18071, 2880, (128, 256)),
                                        (433, 17789, 10000, (160, 256)), (1123, 9151, 4160, (192, 256)), (2166, 13634, 20416, (256, 256))])
def test_every_tile(lib, layer, m, n, k, tile):
    import torch
    assert layer.w8_division(m, n, k)[:2] == tile
    g = torch.Generator(device="cuda").manual_seed(m)
    q, w = (torch.randint(-128, 128, (i, k), dtype=torch.int8, device="cuda", generator=g) for i in (m, n))
    scales, s = (1e-3 * (0.5 + torch.rand(i, device="cuda", generator=g)) for i in (m, n))
    y = layer.w8_linear(lib.W8Rows(q, scales), lib.W8Weight(w, s)).double()
    # (whole numbers below 2^53: exact in float64 in any order)
    ref = (q.double() @ w.double().t()) * scales.double()[:, None] * s.double()[None]
    wrong = (y - ref).abs() > BOUND * ref.abs() + 1e-37
    assert not wrong.any(), "%d wrong, the first at %s" % (int(wrong.sum()), wrong.nonzero()[0].tolist())


@pytest.mark.parametrize("m", [1, 9, 40, 150, 600])
def test_strides_and_what_lies_between(lib, layer, m):
    # rows of x and y inside wider ones, results at odd addresses; what lies beside them stays
    import torch
    rng = np.random.default_rng(m)
    n, k = 333, 592
    w, s, weight = _weight(lib, rng, n, k)
    x = _bits(rng, (m, k + 24))
    for pad, first in ((7, 3), (11, 4), (1, 0)):
        y = torch.full((m, n + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        out = layer.w8_linear(to_gpu(x)[:, 8:8 + k], weight, out=y[:, first:first + n])
        assert out.data_ptr() == y[:, first:].data_ptr()
        q, scale = OB.w8_rows(W.bf16_bits_to_f32(x[:, 8:8 + k]))
        _check(out, _reference(q, scale, w, s))
        assert (y[:, :first] == 7).all() and (y[:, first + n:] == 7).all()


def test_the_longest_sums(lib, layer):
    # every product the largest: 127 * 128 * 131072 stays in 32 bits
    import torch
    k = 131072
    x = torch.ones((3, k), dtype=torch.bfloat16, device="cuda")
    weight = lib.W8Weight(torch.full((40, k), -128, dtype=torch.int8, device="cuda"), torch.full((40,), 2.0 ** -20, device="cuda"))
    for m in (1, 3):
        _check(layer.w8_linear(x[:m], weight), np.full((m, 40), -128.0 * k * 2.0 ** -20))


def test_more_rows_than_a_launch_has(lib, layer):
    import torch
    m = (1 << 23) + 5
    x = torch.zeros((m, 16), dtype=torch.bfloat16, device="cuda")
    picked = torch.tensor([0, 1, (1 << 23) - 1, 1 << 23, m - 1], device="cuda")
    x[picked, 3] = torch.tensor([127.0, 254.0, -63.5, 1.0, 508.0], dtype=torch.bfloat16, device="cuda")
    rows = layer.w8_quantize(x)
    assert rows.q[picked, 3].tolist() == [127, 127, -127, 127, 127] and int(rows.q.count_nonzero()) == 5
    assert rows.scales[picked].tolist() == [1.0, 2.0, 0.5, float(np.float32(1) / np.float32(127)), 4.0]


@pytest.mark.parametrize("m", [1, 6])
def test_weights_beyond_four_gigabytes(lib, layer, m):
    import torch
    n, k = 150_100, 28_672
    g = torch.Generator(device="cuda").manual_seed(m)
    w = torch.randint(-128, 128, (n, k), dtype=torch.int8, device="cuda", generator=g)
    s = 1e-3 * (0.5 + torch.rand(n, device="cuda", generator=g))
    x = torch.randn((m, k), device="cuda", generator=g).to(torch.bfloat16)
    y = layer.w8_linear(x, lib.W8Weight(w, s))
    q, scale = OB.w8_rows(x.float().cpu().numpy())
    edge = 0xFFFF0000 // k // 256 * 256     # (the first output that offsets of 32 bits do not reach)
    at = torch.tensor([0, 1, edge - 1, edge, edge + 1, n - 1], device="cuda")
    _check(y[:, at], _reference(q, scale, w[at].cpu().numpy(), s[at].cpu().numpy()))
    other = torch.from_numpy(q).cuda().double() @ w[-3000:].double().t()
    assert torch.isfinite(y.float()).all() and ((y[:, -3000:].double() != 0) == (other != 0)).all()


def test_weights_of_rows(lib, layer):
    # a weight that was brought to integers like rows: the product is that of the integers
    rng = np.random.default_rng(1)
    w, x = _bits(rng, (300, 512), 0.02), _bits(rng, (33, 512))
    rows = layer.w8_quantize(to_gpu(w))
    wq, ws = OB.w8_rows(W.bf16_bits_to_f32(w))
    q, scale = OB.w8_rows(W.bf16_bits_to_f32(x))
    y = layer.w8_linear(to_gpu(x), lib.W8Weight(rows.q, rows.scales))
    _check(y, _reference(q, scale, wq, ws))
    full = W.bf16_bits_to_f32(x).astype(np.float64) @ W.bf16_bits_to_f32(w).astype(np.float64).T
    assert np.linalg.norm(y.float().cpu().numpy() - full) < 0.02 * np.linalg.norm(full)   # (two roundings of 1 / 127 / 12^(1/2) of a row's greatest)


def test_no_rows_no_outputs(lib, layer):
    import torch
    weight = lib.W8Weight(torch.zeros((5, 32), dtype=torch.int8, device="cuda"), torch.zeros(5, device="cuda"))
    assert tuple(layer.w8_linear(torch.zeros((0, 32), dtype=torch.bfloat16, device="cuda"), weight).shape) == (0, 5)
    none = lib.W8Weight(torch.zeros((0, 32), dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda"))
    assert tuple(layer.w8_linear(torch.zeros((3, 32), dtype=torch.bfloat16, device="cuda"), none).shape) == (3, 0)


@pytest.mark.parametrize("m,n,k", [(1, 512, 4096), (40, 1024, 8192), (300, 512, 8192)])
def test_captured_products(lib, layer, m, n, k):
    import torch
    rng = np.random.default_rng(m)
    _, _, weight = _weight(lib, rng, n, k)
    x = to_gpu(_bits(rng, (m, k)))
    out = layer.w8_linear(x, weight)
    graph, side, y = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.empty_like(out)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        layer.w8_linear(x, weight, out=y, stream=side)
    for i in range(3):
        x.copy_(to_gpu(_bits(rng, (m, k))))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, layer.w8_linear(x, weight))


def _whole_numbers(layer, lib, m, n, k, seed, chunk=8192):
    """A product of any integers, with every result against whole numbers, some rows and outputs at a time."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, w = (torch.randint(-128, 128, (i, k), dtype=torch.int8, device="cuda", generator=g) for i in (m, n))
    scales, s = (1e-3 * (0.5 + torch.rand(i, device="cuda", generator=g)) for i in (m, n))
    y = layer.w8_linear(lib.W8Rows(q, scales), lib.W8Weight(w, s))
    for m0 in range(0, m, chunk):
        rows = q[m0:m0 + chunk].double()
        for n0 in range(0, n, chunk):
            # (below 2^53: exact in float64 in any order)
            ref = (rows @ w[n0:n0 + chunk].double().t()) * scales[m0:m0 + chunk].double()[:, None] * s[n0:n0 + chunk].double()[None]
            wrong = (y[m0:m0 + chunk, n0:n0 + chunk].double() - ref).abs() > BOUND * ref.abs() + 1e-37
            assert not wrong.any(), "%d wrong, the first at %s of part (%d, %d)" % (int(wrong.sum()), wrong.nonzero()[0].tolist(), m0, n0)


@pytest.mark.parametrize("m,n,k,division", [
    (127, 465, 3616, (64, 128, 6)), (84, 328, 11200, (64, 128, 16)), (340, 1133, 7376, (128, 128, 8)), (69, 7397, 7552, (128, 128, 4)), (133, 5923, 7760, (192, 128, 4)),
    (672, 2081, 8640, (192, 128, 3)), (199, 8826, 5952, (128, 256, 3)), (799, 2509, 7696, (160, 256, 4)), (269, 3145, 13504, (160, 256, 8)), (541, 6409, 11040, (192, 256, 3)),
    (995, 5415, 10832, (256, 256, 2)), (408, 7606, 10288, (256, 256, 4))])
def test_ranges_of_every_tile(lib, layer, m, n, k, division):
    assert layer.w8_division(m, n, k) == division
    _whole_numbers(layer, lib, m, n, k, m)


def test_rows_beyond_four_gigabytes(lib, layer):
    _whole_numbers(layer, lib, 150_100, 40, 28_672, 1)


def test_tiles_of_weights_beyond_four_gigabytes(lib, layer):
    assert layer.w8_division(129, 149_760, 28_672) == (160, 256, 1) and layer.w8_division(129, 340, 28_672)[2] > 1    # (the two parts of it)
    _whole_numbers(layer, lib, 129, 150_100, 28_672, 2)


@pytest.mark.parametrize("m,n", [(1, 40), (1, 2692), (32, 4017), (40, 520), (300, 700), (523, 10848), (700, 1500), (3934, 2579)])
def test_the_greatest_sum_of_all(lib, layer, m, n):
    # 131072 products of -128 and -128 are 2^31, one more than an integer of 32 bits holds; of -127 in a row they stay below, of 127 they are the least of all
    import torch
    k = 131072
    row = torch.tensor([-128, 127, -127, 0], dtype=torch.int8, device="cuda")[torch.arange(m, device="cuda") % 4]
    q = row[:, None].expand(m, k).contiguous()
    weight = lib.W8Weight(torch.full((n, k), -128, dtype=torch.int8, device="cuda"), torch.full((n,), 2.0 ** -20, device="cuda"))
    y = layer.w8_linear(lib.W8Rows(q, torch.ones(m, device="cuda")), weight)
    _check(y, np.broadcast_to((row.cpu().numpy().astype(np.float64) * -128.0 * k * 2.0 ** -20)[:, None], (m, n)))


@pytest.mark.parametrize("m,n,k", [(1, 333, 592), (3, 333, 592), (9, 4099, 1040), (40, 333, 4112), (60, 300, 28672), (300, 700, 7376), (523, 2050, 1040), (1093, 4099, 2064)])
def test_rows_and_scales_of_any_size(lib, layer, m, n, k):
    # a row's scale times its sum may be beyond 32 bits where the result is not, and the other way round a row of the least numbers keeps all of its digits
    rng = np.random.default_rng(m + n)
    w, s, _ = _weight(lib, rng, n, k)
    s = (s * np.where(np.arange(n) % 3 == 0, 1e-20, np.where(np.arange(n) % 3 == 1, 1e-33, 1e-3))).astype(np.float32)
    x = rng.standard_normal((m, k)) * 10.0 ** np.linspace(37.3, -28.0, m)[:, None]
    x = W.f32_to_bf16_bits(x.astype(np.float32))
    import torch
    weight = lib.W8Weight(torch.from_numpy(w).cuda(), torch.from_numpy(s).cuda())
    q, scale = OB.w8_rows(W.bf16_bits_to_f32(x))
    ref = _reference(q, scale, w, s)
    most = 2.0 ** 128 * (1 - 2.0 ** -9)     # (what rounds to more than bf16 holds is an infinity)
    sure = (np.abs(ref) < most * (1 - 2.0 ** -20)) | (np.abs(ref) > most * (1 + 2.0 ** -20))
    for rows in (to_gpu(x), layer.w8_quantize(to_gpu(x))):
        got = layer.w8_linear(rows, weight).float().cpu().numpy().astype(np.float64)
        want = np.where(np.abs(ref) >= most, np.copysign(np.inf, ref), ref)
        same = (got == want) | (np.abs(got - want) <= BOUND * np.abs(want) + 2.0 ** -133) | ~sure
        assert same.all(), "%d of %d, the first at %s" % ((~same).sum(), same.size, np.argwhere(~same)[0])

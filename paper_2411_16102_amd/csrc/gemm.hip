// bf16 "NT" GEMM  C[M,N] = A[M,K] * B[N,K]^T  for gfx950, fp32 accumulation on
// v_mfma_f32_16x16x32_bf16, tiles staged through LDS, fused epilogues.  (The chip lowers its
// clock under matrix load; at that limit the 16x16x32 shape, which moves fewer accumulator
// registers per flop, sustains 1.87 PFLOP/s on random operands where 32x32x16 sustains
// 1.7, and this kernel gained 10 to 24 % from the change.)
//
// Operand roles are swapped with respect to the usual picture: the weight rows
// feed the MFMA "A" operand and the activation rows the "B" operand, so an
// accumulator block holds C^T: a lane owns ONE activation row (m = lane % 16) and
// a run of four consecutive output features (n = 4 * (lane / 16) ..).  Every fused epilogue is then
// lane-local: the RMSNorm factor of a row is one scalar per lane, a RoPE pair
// (i, i + dh/2) and a SwiGLU (gate, up) pair sit in two accumulator blocks of the
// same lane; all but gate/up then turn round in LDS on their way out.
//
// Tiles travel global -> LDS directly (global_load_lds_dwordx4), so no VGPRs are spent
// on staging.  A k-tile is BK = 64 wide: a tile row is then one whole 128-byte cache
// line, which the memory pipeline delivers about 1.5 times faster than the two 64-byte
// halves fetched separately (measured: 41 against 26 B/clk/CU into LDS).  LDS holds two
// rings of panels, three weight panels and two activation panels of one k-tile each for a 256x256
// tile: while tile kt is multiplied, tile kt+1 has landed or is landing and the weight panel of
// tile kt+2 is in flight; 160x256 and 128x256 tiles have room for a third activation panel.
// (Of at most 256 rows, what the few-row kernel leaves, gate/up and plain products and the
// k-ranges of the others, uses a second pipeline where it pays, DEEP in the kernel below: one row
// of tiles, a few slots for the activation panel and all other LDS for the weight
// panel, the two kinds of panel requested by different wavefronts.)  Rows are 128 B whose eight 16-byte chunks are XOR-swizzled with
// ((row >> 1) & 7): two consecutive rows fill the 256-byte bank row, so the swizzle
// must change every two rows for the ds_read_b128 of a fragment (16 rows by four chunk
// columns) to be conflict-free.  Waits on the LDS-DMA loads are placed by hand
// (s_waitcnt vmcnt + s_barrier); the compiler does not track them.
#include <algorithm>
#include <numeric>
#include <utility>
#include "gemm.hpp"
#include "attn_device.hpp"
#include "k_order.hpp"
#include "common.hpp"

namespace bs {

// sixteen bytes of zeros: the source of tile chunks that lie beyond K
__device__ __align__(16) uint16_t g_gemm_zero_chunk[8];

}  // namespace bs

#include "gemm_device.hpp"

namespace bs {

namespace {

template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DH, int DEEP = 0>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64, 2) void gemm_kernel(const GemmArgs a) {
  gemm_tile<BM, BN, WAVES_M, WAVES_N, EPI, DH, DEEP>(a, (int)blockIdx.x);
}

// (All 256 registers are in use: 36 to 66 spill, around the loop over k-tiles and never in it, as do 4 to 7 of the whole
// 256x256 tiles of the QKV projection.)
template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DH>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64) void gemm_sk_kernel(const GemmArgs a, const SkPlan p) {
  const int w = (int)blockIdx.x, G = (int)gridDim.x;
  int pid = w;
  int i = 0, i1 = 0, j0 = 0;
  if (w < p.g_sk) {
    i = sk_bound(p, w);
    i1 = sk_bound(p, w + 1);
    j0 = i / p.nk;
  }
  bool again = false;
  for (;;) {
    SkSeg s;
    if (pid < p.n_dp) {
      s = SkSeg{pid, 0, p.nk, 0, 1, 0, 0};
      pid += G;
    } else if (i < i1) {
      const int j = i / p.nk, kt0 = i - j * p.nk;
      const int kt1 = (i1 - j * p.nk) < p.nk ? (i1 - j * p.nk) : p.nk;
      s = SkSeg{p.n_dp + j, kt0, kt1, j, 1, 0, 0};
      if (kt0 > 0 || kt1 < p.nk) {
        sk_tile_span(p, j, &s.w_first, &s.parts);
        s.my_slot = 2 * w + (j == j0 ? 0 : 1);
      }
      i = j * p.nk + kt1;
    } else {
      break;
    }
    if (again) __syncthreads();  // the panel ring and the flag word change hands
    again = true;
    gemm_tile<BM, BN, WAVES_M, WAVES_N, EPI, DH, 0, true>(a, 0, &p, s);
  }
}

// A GEMM launch that carries decode attention (Section 3.3: a step whose compute-bound and
// memory-bound operators overlap costs the larger of their times; Section 2.2, operator-level
// overlapping).  Grid: `head` attention workgroups, the GEMM tiles, `tail` attention
// workgroups.  A workgroup of either kind takes a whole CU (the tile all of its LDS, either
// kind half of every SIMD's registers per wavefront), so the two kinds never share one: the
// head workgroups hold their CUs for as long as the GEMM runs and stream KV pages beside it,
// the tail workgroups start on the CUs that the last, partly filled round of tiles leaves
// idle.  The attention wavefronts draw 16-row units from the step's queue; the tile that
// brings the count of finished tiles to `close_at` closes the queue for this launch and
// hands its position to the next one, so nobody starts a unit that would outlast the GEMM
// by more than its own length.  No workgroup ever waits for another.
template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DH, int ADH>
__global__ __launch_bounds__(WAVES_M *WAVES_N * 64) void gemm_attn_kernel(const GemmArgs a, const GemmRide r, const int n_tiles,
                                                                              const unsigned close_at) {
  static_assert(WAVES_M * WAVES_N == 8, "attention workgroups are written for eight wavefronts");
  const int b = (int)blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint64_t *rec = r.q.trace ? r.q.trace + (size_t)TRACE_WORDS * (8 * b + wave) : nullptr;
  if (b < r.head || b >= r.head + n_tiles) {
    attn_dev::decode_queue_worker<ADH>(r.q, wave, threadIdx.x & 63, rec);
    return;
  }
  const uint64_t t0 = rec ? wall_clock64() : 0;
  gemm_tile<BM, BN, WAVES_M, WAVES_N, EPI, DH>(a, b - r.head);
  if (threadIdx.x == 0) {
    const unsigned before = atomicAdd(r.done, 1u);
    if (before + 1 == close_at) {
      const unsigned pos = atomicAdd(r.q.ticket, DECODE_QUEUE_CLOSED);
      const unsigned capped = pos < (unsigned)r.q.n_units ? pos : (unsigned)r.q.n_units;
      atomicExch(r.ticket_next, capped);
      if (r.closed_at) *r.closed_at = capped;
    }
    if (rec) attn_dev::trace_record(rec, t0, TRACE_TILE, before + 1 == close_at ? 1u : 0u, 0u);
  }
}

constexpr int MAX_SPLITS = 8;

// four consecutive columns of one row, summed over the k-ranges in a fixed order; the loads are
// independent of one another and go out together
__device__ __forceinline__ f32x4_t splitk_sum(const float *p, size_t plane, int k_splits) {
  f32x4_t part[MAX_SPLITS];
#pragma unroll
  for (int s = 0; s < MAX_SPLITS; ++s)
    part[s] = s < k_splits ? *reinterpret_cast<const f32x4_t *>(p + s * plane) : f32x4_t{0.f, 0.f, 0.f, 0.f};
  f32x4_t v = part[0];
#pragma unroll
  for (int s = 1; s < MAX_SPLITS; ++s) v += part[s];
  return v;
}

// Second half of a split-K product: adds the k_splits partial rows and applies the epilogue.
// RESID: y = resid + sum, one thread per four columns.
__global__ __launch_bounds__(256) void splitk_reduce_resid_kernel(const GemmArgs a) {
  const int m = blockIdx.x, n = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (n >= a.N) return;
  f32x4_t v = splitk_sum(a.sk_ws + (size_t)m * a.N + n, (size_t)a.M * a.N, a.k_splits);
  if (a.resid32) {
    v += *reinterpret_cast<const f32x4_t *>(a.resid32 + (size_t)m * a.ldr + n);
  } else {
    const u32x2_t rr = *reinterpret_cast<const u32x2_t *>(a.resid + (size_t)m * a.ldr + n);
    v[0] += __uint_as_float(rr.x << 16);
    v[1] += __uint_as_float(rr.x & 0xFFFF0000u);
    v[2] += __uint_as_float(rr.y << 16);
    v[3] += __uint_as_float(rr.y & 0xFFFF0000u);
  }
  store_bf16x4(a.C + (size_t)m * a.ldc + n, v[0], v[1], v[2], v[3]);
}

// RESID_NORM: x1 = resid + sum in fp32, bf16(x1 * gain), and the row's sum of squares, complete,
// in ss_out slot 0; one workgroup per row, of as many threads as the row has groups of four columns
// (up to 1024), so that a row is one round trip to memory.
__global__ __launch_bounds__(1024) void splitk_reduce_resid_norm_kernel(const GemmArgs a) {
  const int m = blockIdx.x;
  float ss = 0.f;
  for (int n = threadIdx.x * 4; n < a.N; n += (int)blockDim.x * 4) {
    f32x4_t v = splitk_sum(a.sk_ws + (size_t)m * a.N + n, (size_t)a.M * a.N, a.k_splits);
    const u32x2_t rr = *reinterpret_cast<const u32x2_t *>(a.resid + (size_t)m * a.ldr + n);
    v[0] += __uint_as_float(rr.x << 16);
    v[1] += __uint_as_float(rr.x & 0xFFFF0000u);
    v[2] += __uint_as_float(rr.y << 16);
    v[3] += __uint_as_float(rr.y & 0xFFFF0000u);
    const u32x2_t gg = *reinterpret_cast<const u32x2_t *>(a.gain + n);
    const float g0 = __uint_as_float(gg.x << 16), g1 = __uint_as_float(gg.x & 0xFFFF0000u);
    const float g2 = __uint_as_float(gg.y << 16), g3 = __uint_as_float(gg.y & 0xFFFF0000u);
    ss += v[0] * v[0] + v[1] * v[1] + v[2] * v[2] + v[3] * v[3];
    *reinterpret_cast<f32x4_t *>(a.C32 + (size_t)m * a.ldc + n) = v;
    store_bf16x4(a.C_gain + (size_t)m * a.ldc + n, v[0] * g0, v[1] * g1, v[2] * g2, v[3] * g3);
  }
  __shared__ float part[16];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
  __syncthreads();
  if (threadIdx.x == 0) {
    float row = 0.f;
    for (int w = 0; w < ((int)blockDim.x + 63) / 64; ++w) row += part[w];
    a.ss_out[m] = row;
    if (a.rstd_out) a.rstd_out[m] = rsqrtf(row / (float)a.N + a.rstd_eps);
  }
}

// QKV: scale by the row's RMSNorm factor, rotate the q and k heads (pairs i, i + dh/2), store q
// to its buffer, k and v into the row's page slot (v transposed).  One thread per four
// consecutive pairs (q and k heads) or four consecutive v elements.
__global__ __launch_bounds__(256) void splitk_reduce_qkv_kernel(const GemmArgs a, int dh) {
  const int m = blockIdx.x;
  const int item = blockIdx.y * 256 + threadIdx.x;
  const size_t plane = (size_t)a.M * a.N;
  const float *ws = a.sk_ws + (size_t)m * a.N;
  const float rs = a.rstd[m];
  const int half = dh / 2, q4 = half / 4;
  const size_t page = a.row_page[m];
  const int slot = a.row_slot[m];
  const size_t tile_elems = (size_t)16 * dh;
  const int n_rot = (a.n_q_heads + a.n_kv_heads) * q4;
  if (item < n_rot) {
    const int head = item / q4, i = (item % q4) * 4, pos = a.row_pos[m];
    const f32x4_t l = splitk_sum(ws + head * dh + i, plane, a.k_splits) * rs;
    const f32x4_t h = splitk_sum(ws + head * dh + half + i, plane, a.k_splits) * rs;
    const f32x4_t c = *reinterpret_cast<const f32x4_t *>(a.rope_cos + (size_t)pos * half + i);
    const f32x4_t sn = *reinterpret_cast<const f32x4_t *>(a.rope_sin + (size_t)pos * half + i);
    uint16_t *dst = head < a.n_q_heads
                        ? a.q_out + (size_t)m * (a.n_q_heads * dh) + head * dh
                        : a.kv_pool + ((page * 2 + 0) * a.n_kv_heads + (head - a.n_q_heads)) * tile_elems + (size_t)slot * dh;
    const f32x4_t lo = l * c - h * sn, hi = h * c + l * sn;
    store_bf16x4(dst + i, lo[0], lo[1], lo[2], lo[3]);
    store_bf16x4(dst + half + i, hi[0], hi[1], hi[2], hi[3]);
  } else if (item < n_rot + a.n_kv_heads * (dh / 4)) {
    const int w = (item - n_rot) * 4, head = w / dh, e = w % dh;
    const f32x4_t v = splitk_sum(ws + (a.n_q_heads + a.n_kv_heads) * dh + w, plane, a.k_splits) * rs;
    uint16_t *dst = a.kv_pool + ((page * 2 + 1) * a.n_kv_heads + head) * tile_elems + slot;
#pragma unroll
    for (int j = 0; j < 4; ++j) dst[(e + j) * 16] = f32_to_bf16(v[j]);
  }
}

template <int MI, int NI>
hipError_t launch_rows_one(const GemmArgs &a, int epi, int dh, hipStream_t stream) {
  typedef RowsKernel<MI, NI> R;
  const int n_cu = a.n_cu > 0 ? a.n_cu : 256, tiles_m = (a.M + 16 * MI - 1) / (16 * MI);
  if (tiles_m * 16 * MI > ROWS_MAX_M || a.N % 8) return hipErrorInvalidValue;
  const long items = (long)tiles_m * ((rows_blocks(a.N, epi) + NI - 1) / NI), rounds = (items + n_cu - 1) / n_cu;
  if (items <= 0 || items >= (1L << 30)) return hipErrorInvalidValue;
  auto kern = gemm_rows_kernel<MI, NI>;
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(kern), R::LDS)) return e;
  // as many workgroups as give each the same number of items
  hipLaunchKernelGGL(kern, dim3((unsigned)((items + rounds - 1) / rounds)), dim3(512), R::LDS, stream, a, epi, dh, tiles_m, (int)items);
  return hipGetLastError();
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DH, int DEEP = 0>
hipError_t launch_one(const GemmArgs &a, hipStream_t stream) {
  constexpr int OUT_BN = (EPI == EPI_SWIGLU) ? BN / 2 : BN;
  constexpr int LDS = DEEP ? LDS_CU : ring_bytes(WAVES_M * WAVES_N);
  auto kern = gemm_kernel<BM, BN, WAVES_M, WAVES_N, EPI, DH, DEEP>;
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(kern), LDS)) return e;
  const int n_cols = a.n_count ? a.n_count : a.N;
  const int tiles = ((a.M + BM - 1) / BM) * ((n_cols + OUT_BN - 1) / OUT_BN) * (EPI == EPI_PARTIAL ? a.k_splits : 1);
  if (tiles <= 0) return hipSuccess;
  hipLaunchKernelGGL(kern, dim3(tiles), dim3(WAVES_M * WAVES_N * 64), LDS, stream, a);
  return hipGetLastError();
}

constexpr int SK_MAX_G = 256;  // workgroups of a shared-tile launch at most: one per CU

template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DH>
hipError_t launch_sk(const GemmArgs &a, hipStream_t stream) {
  constexpr int OUT_BN = (EPI == EPI_SWIGLU) ? BN / 2 : BN;
  constexpr int LDS = ring_bytes(WAVES_M * WAVES_N);
  static_assert(BM == 256 && BN == 256, "the workspace slots are sized for 256x256 tiles");
  if (!a.sk_ws || !a.sk_cnt || a.n_count || a.k_splits > 1) return hipErrorInvalidValue;
  auto kern = gemm_sk_kernel<BM, BN, WAVES_M, WAVES_N, EPI, DH>;
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(kern), LDS)) return e;
  const long tiles = (long)((a.M + BM - 1) / BM) * ((a.N + OUT_BN - 1) / OUT_BN);
  if (tiles <= 0) return hipSuccess;
  const int G = a.n_cu > 0 && a.n_cu < SK_MAX_G ? a.n_cu : SK_MAX_G;
  SkPlan p{};
  p.nk = (a.K + BK - 1) / BK;
  p.ws = a.sk_ws;
  p.cnt = a.sk_cnt;
  if (tiles % G == 0) {
    p.n_dp = (int)tiles;
  } else {
    // (with more than one round the last whole round is shared too: every workgroup then has more
    // than a tile's worth of iterations and at most two cuts)
    p.n_sk = tiles > G ? (int)(tiles % G) + G : (int)tiles;
    p.n_dp = (int)tiles - p.n_sk;
    const long total = (long)p.n_sk * p.nk;
    p.g_sk = (int)std::min<long>(G, std::max<long>(1, total / SK_MIN_ITERS));
    if (total * p.g_sk >= (1L << 31)) return hipErrorInvalidValue;
  }
  const int grid = (int)std::min<long>(G, std::max<long>(p.g_sk, p.n_dp));
  hipLaunchKernelGGL(kern, dim3(grid), dim3(WAVES_M * WAVES_N * 64), LDS, stream, a, p);
  return hipGetLastError();
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int ADH>
hipError_t launch_ride(const GemmArgs &a, const GemmRide &r, hipStream_t stream) {
  constexpr int OUT_BN = (EPI == EPI_SWIGLU) ? BN / 2 : BN;
  constexpr int LDS = ring_bytes(WAVES_M * WAVES_N);
  static_assert(LDS == LDS_CU, "a workgroup of either kind must take the whole LDS of its CU");
  auto kern = gemm_attn_kernel<BM, BN, WAVES_M, WAVES_N, EPI, 64, ADH>;
  static OncePerDevice once;
  if (const hipError_t e = allow_lds(once, reinterpret_cast<const void *>(kern), LDS)) return e;
  const int tiles = ((a.M + BM - 1) / BM) * ((a.N + OUT_BN - 1) / OUT_BN);
  if (tiles <= 0) return hipErrorInvalidValue;
  // (a negative margin: no tile closes the queue, the launch drains it)
  const int close_at = r.close_margin < 0 ? tiles + 1 : (tiles - r.close_margin > 1 ? tiles - r.close_margin : 1);
  hipLaunchKernelGGL(kern, dim3(r.head + tiles + r.tail), dim3(WAVES_M * WAVES_N * 64), LDS, stream, a, r, tiles,
                     (unsigned)close_at);
  return hipGetLastError();
}

// Tile shapes.  BIG: 256x256, 8 wavefronts.  TALL: 160x256, 8 wavefronts of 80x64: 2560 (and
// 5120) rows by 4096 (8192) columns then make exactly one (four) full rounds of 256
// workgroups where 256x256 tiles leave 38 % (17 %) of the CUs idle.  SMALL: 128x128.
// S128 / S256: 128x256 and 256x128 tiles on the deep weight ring, for at most 128 / 256 rows; D64 / D128: 64x128 and
// 128x128 tiles on it, for whole products of at most 64 / 128 rows.  MID: 192x256, 8 wavefronts of 96x64; WIDE: 128x256, 8 of 64x64.
// activation slots of the short-row pipeline, minus one: three slots leave four weight slots of 16 KB
// (256x128) or three of 32 KB (128x256); measured against two slots (six / four weight slots) on the
// 256-row gate/up GEMM of the 8B layer: 0.075 against 0.078 ms, the other GEMMs the same
constexpr int DEEP_X = 2;
enum { V_AUTO = 0, V_BIG = 1, V_TALL = 2, V_SMALL = 3, V_S128 = 4, V_S256 = 5, V_SHARED = 6, V_ROWS = 7, V_D64 = 8, V_D128 = 9, V_MID = 10, V_WIDE = 11 };
constexpr int N_CU = 256;

thread_local int g_forced_variant = V_AUTO;  // set by the calling entry point from its context, for the launches of that call

long n_tiles(int m, int n, int bm, int bn) { return (long)((m + bm - 1) / bm) * ((n + bn - 1) / bn); }

// few rows: one tile row on the deep weight ring (0 where the rows do not fit one tile, or a shape is forced)
int short_variant(int m) {
  if (g_forced_variant != V_AUTO || m > 256) return 0;
  return m <= 128 ? V_S128 : V_S256;
}

// The few-row kernel's item, as 10 MI + NI (0: the tiles are the better choice, or a shape is forced).  Up to 16 rows it is
// ahead everywhere (70B down projection at 16 rows 88 against 86 us, the one exception).  Beyond, the activation rows of an
// item outweigh its weights: it needs one round of items (gate/up two, which saves nothing else) over a short K, or its
// eight wavefronts hold too little of K in flight.  Measured at 32 rows against the tiles, both with cold
// weights: N = 3072, K = 2048 QKV 7.2 against 12.2 us, N = K = 4096 output projection 11.3 against 15.9, N = 2048,
// K = 8192 down 16.3 against 17.7; N = 4096, K = 14336 31 against 28.5; gate/up of 2 x 8192 columns, K = 2048 17 against 24.8,
// of 2 x 14336, K = 4096 51.5 against 54 for shallow tiles.  Above 64 rows only where a wavefront has one k-tile or two:
// 136 rows, N = 512, K = 256 5 against 10.5 us; N = 256, K = 688 5 against 12.
int rows_item(int m, int n, int k, int epilogue, int n_cu) {
  if (g_forced_variant != V_AUTO || m > ROWS_MAX_M || n % 8) return 0;
  const long nk = (k + BK - 1) / BK, blocks = rows_blocks(n, epilogue);
  if (m <= 16) return 11;
  const long tiles_m = (m + 31) / 32, longest = m <= 64 ? 128 : 12;
  if (nk > longest) return 0;
  if (tiles_m * blocks <= n_cu) return 21;
  const long rounds = epilogue == EPI_SWIGLU && m <= 32 ? 2 : 1;
  return tiles_m * ((blocks + 1) / 2) <= rounds * n_cu ? 22 : 0;
}

// Estimated time of a product in microseconds.  A k-tile costs between `lo` (few workgroups on the chip) and `hi` (all of
// them: the clock falls under matrix load); 128x128 tiles, two to a CU, cost `lo` up to one per CU.  A round of whole tiles
// has its start and its epilogue (`round`), a cut product the second kernel and the partial products once out and once back
// in (most of it the last-level cache); the output projection whole needs the pass that closes the second norm.
// Fitted on MI355X to the products of eight layers (QKV, output, gate/up and down projections, 1024 to 57344 columns, K 1024
// to 28672) at 26 row counts each, those above 512, weights cold, every shape and cut timed: 2.7 % from the times that matter.
struct Shape {
  int v, bm, bn, per_cu;
  double hi, lo, round[4];  // QKV, output projection, down projection, gate/up
};
constexpr Shape SHAPES[5] = {{V_BIG, 256, 256, 1, 1.44, 0.81, {11.6, 19.7, 18.5, 9.5}},
                             {V_TALL, 160, 256, 1, 0.97, 0.65, {8.6, 11.7, 7.7, 6.6}},
                             {V_SMALL, 128, 128, 2, 0.95, 0.51, {6.5, 8.4, 5.0, 4.0}},
                             {V_MID, 192, 256, 1, 1.13, 0.72, {9.2, 13.7, 11.3, 7.6}},
                             {V_WIDE, 128, 256, 1, 0.85, 0.58, {7.6, 10.1, 5.9, 5.9}}};
constexpr double TWO_PER_CU = 0.65, CLOSING_US = 4.5, SECOND_US[3] = {10.4, 10.3, 7.3}, PARTIAL_BYTES_US = 7.0e6;
constexpr int FIT_MIN_K = 1024;

// k-tiles of one workgroup after the other over `tiles` workgroups of the shape, in microseconds
double rounds_us(const Shape &c, long tiles, double hi, double lo, double two, int n_cu) {
  const long slots = (long)n_cu * c.per_cu, full = tiles / slots, rem = tiles % slots;
  double part = 0.0;
  if (rem && c.per_cu == 1) part = lo + (hi - lo) * (double)rem / (double)slots;
  else if (rem) part = rem <= n_cu ? lo : lo + (hi - lo) * (two + (1.0 - two) * (double)(rem - n_cu) / (double)n_cu);
  return (double)full * hi + part;
}
int epi_column(int epilogue) { return epilogue == EPI_QKV ? 0 : epilogue == EPI_RESID_NORM ? 1 : epilogue == EPI_SWIGLU ? 3 : 2; }
double whole_us(const Shape &c, int m, int n, int k, int n_cu, int epilogue) {
  const long tiles = n_tiles(m, n, c.bm, c.bn), slots = (long)n_cu * c.per_cu;
  return (double)((k + BK - 1) / BK) * rounds_us(c, tiles, c.hi, c.lo, TWO_PER_CU, n_cu) +
         c.round[epi_column(epilogue)] * (double)((tiles + slots - 1) / slots) + (epilogue == EPI_RESID_NORM ? CLOSING_US : 0.0);
}
double cut_us(const Shape &c, int m, int n, int k, int s, int n_cu, int epilogue) {
  const long nk = (k + BK - 1) / BK;
  return (double)((nk + s - 1) / s) * rounds_us(c, n_tiles(m, n, c.bm, c.bn) * s, c.hi, c.lo, TWO_PER_CU, n_cu) +
         SECOND_US[epi_column(epilogue)] + 8.0 * s * m * n / PARTIAL_BYTES_US;
}

// Columns of 256x256 tiles that fill whole rounds where the last round leaves more than a quarter of the chip idle, else 0.
long round_split_columns(long tm, long tn, int n_cu) {
  const long tiles = tm * tn, full = tiles / n_cu, idle = (full + 1) * n_cu - tiles, cols = full * n_cu / tm;
  return full < 1 || tiles % n_cu == 0 || idle * 4 <= n_cu || cols < 1 || cols >= tn ? 0 : cols;
}

// What the second launch of a product in two costs beside its rounds.  Of 386 gate/up products of eight layers, timed in steps whole and
// in two launches, the choice is 0.3 % off the best on average and 4 % at most with 2 to 3; with none, products of 45 to 80 us
// went out as two launches for an expected 2 us and took 3 to 6 more (K = 1024, 2 x 4096 columns, 2056 rows: 48.0 us, whole 42.3).
constexpr double SECOND_LAUNCH_US = 2.0;

// Gate/up of more than 512 rows: the shape with the smallest estimate, and that estimate.  *cols: 0, or the columns of 256x256 tiles
// that go out in whole rounds of their own, the rest behind them on 128x128 tiles, where that is expected to be shorter than whole
// (timed both ways, 8B layer: 1160 rows 254 us whole, 237 in two launches; 3300 rows 553 and 570).  Of 182 products of seven layers timed
// with cold weights it is 0.6 % off the best on average.  1580 rows of the 8B layer: 192x256 tiles 330 us, 160x256 tiles, faster
// since they have three activation panels, 316.  (Below K = 1024, where nothing was fitted, the relation of rounds in choose_variant.)
double gate_up_us(int m, int n_b_rows, int k, int n_cu, int *v, int *cols) {
  double best_t = 1e300;
  auto offer = [&](double t, int variant, int columns) {
    if (t < best_t) { best_t = t; *v = variant; *cols = columns; }
  };
  for (const Shape &c : SHAPES) offer(whole_us(c, m, n_b_rows, k, n_cu, EPI_SWIGLU), c.v, 0);
  const int split = (int)round_split_columns((m + 255) / 256, (n_b_rows + 255) / 256, n_cu);
  if (split)
    offer(whole_us(SHAPES[0], m, split * 256, k, n_cu, EPI_SWIGLU) + whole_us(SHAPES[2], m, n_b_rows - split * 256, k, n_cu, EPI_SWIGLU) +
              SECOND_LAUNCH_US, V_BIG, split);
  return best_t;
}

// Two shapes for one product: whole rounds of one of the 256-wide shapes over the first `cols` tile columns, another shape, whose
// rounds the rest happens to fill, over the others.  Taken where the estimate of the two launches is 3 % below the best single
// choice, about its own error.  Measured in steps, 8B layer: 776 rows 192 us on one shape, 170 as one round of 160x256 tiles and
// 256x256 ones for the rest; 1288 rows 269 -> 251.
bool gate_up_pair(int m, int n_b_rows, int k, int n_cu, int *head, int *tail, int *cols) {
  int single, single_cols;
  double best_t = 0.97 * gate_up_us(m, n_b_rows, k, n_cu, &single, &single_cols);
  bool found = false;
  for (const Shape &c : SHAPES) {
    if (c.bn != 256) continue;
    const long tm = (m + c.bm - 1) / c.bm, tn = (n_b_rows + 255) / 256, full = tm * tn / n_cu;
    for (long f = std::max(1L, full - 2); f <= full; ++f) {
      const long n = f * n_cu / tm;
      if (n < 1 || n >= tn) continue;
      const double t = whole_us(c, m, (int)n * 256, k, n_cu, EPI_SWIGLU) + SECOND_LAUNCH_US;
      for (const Shape &c2 : SHAPES) {
        const double t2 = t + whole_us(c2, m, n_b_rows - (int)n * 256, k, n_cu, EPI_SWIGLU);
        if (t2 >= best_t) continue;
        best_t = t2;
        *head = c.v;
        *tail = c2.v;
        *cols = (int)n;
        found = true;
      }
    }
  }
  return found;
}

// Tile shape of a gate/up or plain product, or of any with a forced shape (QKV, output and down projection:
// gemm_plan).
// Gate/up of more than 512 rows goes by the estimate in microseconds (gate_up_us), the others by that of a launch in
// units of one full round of 256x256 tiles: full rounds of
// workgroups (the 128x128 tile runs two per CU) cost T each; a last, partly filled round costs
// T (a + (1 - a) fill): workgroups that share the chip with fewer others run faster, but not in
// proportion.  T and a were fitted on MI355X to the four GEMM shapes of the 8B layer at 384 to
// 2560 rows (the 160x256 tile: 0.072 ms per full round at K = 4096 where the 256x256 tile takes
// 0.100 and 512 tiles of 128x128 take 0.075).
// share_k: the contraction length if the launch may share tiles between workgroups (it has the
// workspace for it and covers all columns), else 0
int choose_variant(int m, int n_b_rows, int k, int epilogue, int dh, int n_cu, int share_k = 0) {
  if (n_cu <= 0) n_cu = N_CU;
  if (g_forced_variant != V_AUTO && !(g_forced_variant == V_TALL && epilogue == EPI_QKV)) return g_forced_variant;
  (void)dh;
  // Few rows that the few-row kernel leaves: measured, cold weights, against 128x128 tiles on the shallow ring, 64 (90, 128)
  // rows: 2 x 14336 columns, K = 4096 54.9 -> 44.1 (55.9 -> 48.9, 57.2 -> 52.4) us; 2 x 8192, K = 3072 34.9 -> 31.0
  // (35.9 -> 35.0, 37.8 -> 37.5); 2 x 13824, K = 5120 60.9 -> 55.7 (62.5 -> 61.5, 66.3 -> 66.1); 2 x 4096, K = 1024
  // 13.7 -> 11.8 (14.0 -> 13.5, 14.4 -> 14.3); of more than one round only at 64 rows: 2 x 28672, K = 8192 165 -> 162
  // (128x128 tiles 179 against 162 of 128x256).
  if (g_forced_variant == V_AUTO && m <= 128 && (epilogue == EPI_SWIGLU || epilogue == EPI_PLAIN)) {
    if (m <= 64) return V_D64;
    if (n_tiles(m, n_b_rows, 128, 128) <= n_cu) return V_D128;
  }
  if (const int sv = short_variant(m); sv && (epilogue == EPI_SWIGLU || epilogue == EPI_PLAIN)) {
    // worth it once the single row of tiles fills at least half the chip
    if (2 * n_tiles(m, n_b_rows, sv == V_S128 ? 128 : 256, sv == V_S128 ? 256 : 128) >= n_cu) return sv;
  }
  const bool estimated = epilogue == EPI_SWIGLU && g_forced_variant == V_AUTO && k >= FIT_MIN_K;
  if (estimated && m > 512) {
    int best, cols;
    gate_up_us(m, n_b_rows, k, n_cu, &best, &cols);
    return best;
  }
  struct Cand { int v, bm, bn, per_cu; double T, a; };
  // 192x256 tiles (gate/up) fetch a tenth less per flop than 160x256 ones, and waste fewer rows than 256x256 where the
  // rows end early in a tile.  T and a from the gate/up products of three layers at 44 row counts from 257 to 4096,
  // every shape timed with cold weights, before 160x256 tiles had a third activation panel.  2 x 14336 columns, K = 4096:
  // 359 rows 97 -> 91 us (256x256); 2 x 8192, K = 2048: 359 rows 43 against 36 of 128x128.
  const Cand cands[4] = {{V_BIG, 256, 256, 1, 1.00, 0.72}, {V_TALL, 160, 256, 1, 0.76, 0.65}, {V_SMALL, 128, 128, 2, 0.75, 0.60},
                         {V_MID, 192, 256, 1, 0.85, 0.75}};
  int best = V_SMALL;
  double best_t = 1e300;
  for (const Cand &c : cands) {
    if (c.v == V_TALL && epilogue == EPI_QKV) continue;  // (QKV comes here for forced shapes alone, which do not force it to 160x256)
    if (c.v == V_MID && epilogue != EPI_SWIGLU) continue;
    const long tiles = n_tiles(m, n_b_rows, c.bm, c.bn);
    const long slots = (long)n_cu * c.per_cu;
    const long full = tiles / slots, rem = tiles % slots;
    const double t = (double)full * c.T + (rem ? c.T * (c.a + (1.0 - c.a) * (double)rem / (double)slots) : 0.0);
    if (t < best_t) { best_t = t; best = c.v; }
  }
  // Up to 512 rows 128x256 tiles where the estimate puts them ahead of that choice: 2 x 8192 columns, K = 2048 at 359 rows
  // 37.1 us on 128x128 tiles, 33.5 on these; 5 % on average over 51 products of 257 to 512 rows, and none slower than that
  // choice, though 128x128 tiles would be ahead of both where N and K are small (2 x 4096, K = 1024 at 308 rows 13.1 us
  // against 17.9, and 20.7 on 160x256 ones).
  if (estimated && m > 256) {
    for (const Shape &c : SHAPES)
      if (c.v == best && whole_us(SHAPES[4], m, n_b_rows, k, n_cu, EPI_SWIGLU) < whole_us(c, m, n_b_rows, k, n_cu, EPI_SWIGLU)) return V_WIDE;
  }
  // Shared 256x256 tiles: the chip's worth of k-tile iterations with nothing idle, 3 % for the
  // persistent loop, and what the cuts cost: a workgroup passes up to two partial tiles through
  // memory, about 0.08 ms per launch whatever its size (measured on the GEMMs of the 8B and 70B
  // layers), i.e. 53 k-tiles' worth of a round.  It pays only where K is long.
  if (share_k >= 4096 && m > 256) {
    const long tiles = n_tiles(m, n_b_rows, 256, 256);
    const long g = std::min<long>(n_cu, N_CU);
    if (tiles % g) {
      const double t = (double)tiles / (double)g * 1.03 + 53.0 / (double)((share_k + BK - 1) / BK);
      if (t < best_t) { best_t = t; best = V_SHARED; }
    }
  }
  return best;
}

template <int EPI>
hipError_t launch_variant(const GemmArgs &a, int v, hipStream_t stream) {
  if (v == V_BIG) return launch_one<256, 256, 2, 4, EPI, 64>(a, stream);
  if (v == V_SHARED) return launch_sk<256, 256, 2, 4, EPI, 64>(a, stream);
  if (v == V_TALL) return launch_one<160, 256, 2, 4, EPI, 64>(a, stream);
  if constexpr (EPI == EPI_SWIGLU || EPI == EPI_PLAIN) {
    if (v == V_D64) return launch_one<64, 128, 4, 2, EPI, 64, DEEP_X>(a, stream);
    if (v == V_D128) return launch_one<128, 128, 4, 2, EPI, 64, DEEP_X>(a, stream);
    if (v == V_S128) return launch_one<128, 256, 2, 4, EPI, 64, DEEP_X>(a, stream);
    if (v == V_S256) return launch_one<256, 128, 4, 2, EPI, 64, DEEP_X>(a, stream);
  }
  if constexpr (EPI != EPI_PLAIN) {  // (no plain product is given these)
    if (v == V_MID) return launch_one<192, 256, 2, 4, EPI, 64>(a, stream);
    if (v == V_WIDE) return launch_one<128, 256, 2, 4, EPI, 64>(a, stream);
  }
  return launch_one<128, 128, 2, 2, EPI, 64>(a, stream);
}

template <int DH>
hipError_t launch_qkv(const GemmArgs &a, int v, hipStream_t stream) {
  if (v == V_SHARED) return launch_sk<256, 256, 2, 4, EPI_QKV, DH>(a, stream);
  if (v == V_BIG) return launch_one<256, 256, 2, 4, EPI_QKV, DH>(a, stream);
  if (v == V_TALL) return launch_one<160, 256, 2, 4, EPI_QKV, DH>(a, stream);
  if (v == V_MID) return launch_one<192, 256, 2, 4, EPI_QKV, DH>(a, stream);
  if (v == V_WIDE) return launch_one<128, 256, 2, 4, EPI_QKV, DH>(a, stream);
  return launch_one<128, 128, 2, 2, EPI_QKV, DH>(a, stream);
}

}  // namespace

void gemm_force_variant(int v) { g_forced_variant = v; }
size_t gemm_sk_workspace_floats() { return (size_t)2 * SK_MAX_G * 256 * 256; }
int gemm_sk_counters() { return 2 * SK_MAX_G; }

bool gemm_streams_weights(const GemmArgs &a, int epilogue) {
  return !a.n_count && a.k_splits <= 1 && rows_item(a.M, a.N, a.K, epilogue, a.n_cu > 0 ? a.n_cu : N_CU) != 0;
}

bool gemm_round_split(const GemmArgs &a, int epilogue, int dh, GemmArgs *head, GemmArgs *tail) {
  if (epilogue != EPI_SWIGLU || g_forced_variant != V_AUTO || a.k_splits > 1) return false;
  const int n_cols = a.n_count ? a.n_count : a.N;
  if (gemm_streams_weights(a, epilogue)) return false;
  const int n_cu = a.n_cu > 0 ? a.n_cu : N_CU;
  int first, rest, cols;
  const bool estimated = a.M > 512 && a.K >= FIT_MIN_K;
  if (!estimated || !gate_up_pair(a.M, 2 * n_cols, a.K, n_cu, &first, &rest, &cols)) {
    if (estimated) {
      gate_up_us(a.M, 2 * n_cols, a.K, n_cu, &first, &cols);
    } else {
      if (choose_variant(a.M, 2 * n_cols, a.K, epilogue, dh, a.n_cu) != V_BIG) return false;
      cols = (int)round_split_columns((a.M + 255) / 256, (n_cols + 127) / 128, n_cu);  // a 256x256 tile yields 128 output columns
    }
    if (!cols) return false;
    first = V_BIG;
    rest = V_SMALL;  // two workgroups per CU fill the chip best with what is left of a round
  }
  *head = a;
  *tail = a;
  head->n_count = cols * 128;
  tail->n_begin = a.n_begin + head->n_count;
  tail->n_count = n_cols - head->n_count;
  head->tile_variant = first;
  tail->tile_variant = rest;
  return true;
}

void gemm_plan(GemmArgs &a, int epilogue) {
  a.k_splits = 1;
  const int n_cu = std::min(a.n_cu > 0 ? a.n_cu : N_CU, N_CU);
  if (gemm_streams_weights(a, epilogue)) {
    a.tile_variant = V_ROWS;
    return;
  }
  const long nk = (a.K + BK - 1) / BK;
  const size_t room = a.sk_ws && a.N % 4 == 0 ? gemm_sk_workspace_floats() : 0;
  // k-ranges of at least eight k-tiles, one round of workgroups, partial products that fit the workspace
  auto max_splits = [&](long tiles, long slots) {
    long s = std::min<long>(std::min<long>(MAX_SPLITS, nk / 8), slots / tiles);
    while (s > 1 && (size_t)s * a.M * a.N > room) --s;
    return std::max<long>(s, 1);
  };
  const bool may_share = a.sk_ws && a.sk_cnt && !a.n_count;
  if (g_forced_variant != V_AUTO) {
    a.tile_variant = choose_variant(a.M, a.N, a.K, epilogue, 0, a.n_cu, may_share ? a.K : 0);
    if (a.tile_variant == V_SMALL) a.k_splits = (int)max_splits(n_tiles(a.M, a.N, 128, 128), 2L * n_cu);
    return;
  }
  // At most 256 rows: the weights stream from HBM, so what counts is how many workgroups ask for them.
  // One row of tiles on the deep weight ring, cut along K until there is one workgroup per CU; of 128
  // rows and less, 128x128 tiles where MAX_SPLITS ranges of the 256-wide ones would leave a quarter of
  // the CUs without one (measured with cold weights, 64 rows, reduction included: K = 14336, N = 4096,
  // 128 workgroups of 128x256 35 us, 256 of 128x128 30; K = N = 8192, 192 of 128x256 34, 128x128 37).
  if (a.M <= 256) {
    const bool s128 = a.M <= 128;
    const long tiles = s128 ? n_tiles(a.M, a.N, 128, 256) : n_tiles(a.M, a.N, 256, 128);
    const long s = max_splits(tiles, n_cu);
    if (s >= 2 && (!s128 || 4 * s * tiles > 3 * n_cu)) {
      a.tile_variant = s128 ? V_S128 : V_S256;
      a.k_splits = (int)s;
      return;
    }
    const long small = n_tiles(a.M, a.N, 128, 128), ss = max_splits(small, n_cu);
    if (s128 && ss >= 2) {
      a.tile_variant = V_SMALL;
      a.k_splits = (int)ss;
      return;
    }
  }
  // Above, up to 1024 rows: the estimate of an earlier fit (the same terms, 256x256, 160x256 and 128x128 tiles, the products
  // of twelve layers of 256 to 12288 columns and K 256 to 28672, before the requests of the main loop were dealt out).  With the
  // present kernels its choices are 3.5 % off the best of all shapes and cuts on average over 293 products, 74 of them by more than
  // 5 % and the worst by 33 (down projection, N = 3072, K = 8192 at 667 rows: 256x256 tiles in seven ranges 60.8 us, 45.7 on 160x256
  // tiles in four).  The present fit over these three shapes gives no more; 192x256 and 128x256 tiles, cut, are not offered here.
  struct Earlier { double round, second, closing; };
  const Earlier ep = epilogue == EPI_QKV ? Earlier{7.1, 5.2, 0.0} : epilogue == EPI_RESID_NORM ? Earlier{6.7, 7.4, 4.0} : Earlier{5.7, 4.0, 0.0};
  constexpr double PARTIAL_ROUND = 5.0, PARTIAL_BYTES_PER_US = 6.4e6, HI[3] = {1.35, 1.05, 1.03}, LO[3] = {1.09, 1.06, 0.63};
  double best = 1e300;
  auto offer = [&](double t, int v, long s) {
    if (t < best) { best = t; a.tile_variant = v; a.k_splits = (int)s; }
  };
  const bool few = a.M <= 1024;
  for (int i = 0; few && i < 3; ++i) {
    const Shape &c = SHAPES[i];
    const long tiles = n_tiles(a.M, a.N, c.bm, c.bn), slots = (long)n_cu * c.per_cu;
    for (long s = 1; s <= max_splits(tiles, slots); ++s) {
      if (s == 1 && c.v == V_TALL && epilogue == EPI_QKV) continue;
      double t = (double)((nk + s - 1) / s) * rounds_us(c, tiles * s, HI[i], LO[i], 0.59, n_cu) +
                 (s > 1 ? PARTIAL_ROUND : ep.round) * (double)((tiles * s + slots - 1) / slots);
      t += s > 1 ? ep.second + 8.0 * (double)s * a.M * a.N / PARTIAL_BYTES_PER_US : ep.closing;
      offer(t, c.v, s);
    }
  }
  // QKV of 513 to 1024 rows: whole 160x256, 192x256 and 128x256 tiles against that choice by the present fit (8B layer,
  // 1024 rows: 256x256 tiles in two ranges 64.8 us, 128x256 whole 55.4; 3.4 % on average over 49 products, 2.8 % slower at worst).
  // Above 1024 rows every shape, whole and cut: against the earlier fit's choices QKV is 6.2 % faster on average over 136 products (5.3 %
  // slower at worst, 41.4 -> 43.6 us), output projection 3.5 % over 135 (9 %, 19.6 -> 21.4), down projection 4.9 % over 134 (2 %), and
  // 1.3, 0.3 and 0.2 % off the best (8B layer, 1580 rows: QKV 80 us on 256x256 tiles, 68 on 160x256; output projection 69.5 on
  // 256x256 tiles in two ranges, 61 on 128x256 whole.  70B layer, 5120 rows: QKV 721 on shared tiles, 636 on 160x256).  Of more
  // than one round QKV stays off 192x256 and 128x256 tiles, which would be ahead in 13 of the 136 by more than 5 % (70B layer,
  // 2207 rows 332 us against 309; 8B layer, 3644 rows 183 against 159; N = 3072, K = 2048 at 7000 rows 103 against 86): a
  // test holds the division of 2200 rows of the 70B layer to whole 256x256 tiles.
  if (!few || (epilogue == EPI_QKV && a.M > 512)) {
    if (few) {
      const Shape &c = SHAPES[a.tile_variant - V_BIG];  // one of the first three, numbered alike
      best = a.k_splits > 1 ? cut_us(c, a.M, a.N, a.K, a.k_splits, n_cu, epilogue) : whole_us(c, a.M, a.N, a.K, n_cu, epilogue);
    }
    for (const Shape &c : SHAPES) {
      const long tiles = n_tiles(a.M, a.N, c.bm, c.bn), slots = (long)n_cu * c.per_cu;
      const bool added = c.v == V_MID || c.v == V_WIDE;
      if (epilogue == EPI_QKV && added && tiles > slots) continue;
      if (few && !added && c.v != V_TALL) continue;
      offer(whole_us(c, a.M, a.N, a.K, n_cu, epilogue), c.v, 1);
      for (long s = 2; !few && s <= max_splits(tiles, slots); ++s) offer(cut_us(c, a.M, a.N, a.K, (int)s, n_cu, epilogue), c.v, s);
    }
  }
  // Shared 256x256 tiles: the chip's worth of k-tile iterations with nothing idle, and 22 us for the cuts (a
  // workgroup passes up to two partial tiles through memory).  Only where K is long, more than one round of tiles cannot be
  // cut evenly, and the tiles beyond whole rounds are a multiple of a quarter round: else the workgroups walk K in
  // eight and more phases and share few panels in L2 (QKV of 12288 columns, K = 4096, 5600 rows: 522 us, 461 on whole
  // 256x256 tiles; down projection of the 70B layer, 6695 rows: 2847 against 2581; of 124 such products two are
  // ahead of the best other choice, by 1 %, and all are 31 % behind it on average).  Four phases cost 4 % more per k-tile than one
  // or two.  Fitted to the 67 products of up to four phases in steps of six layers; it takes the eleven on which these tiles
  // are ahead: 70B down projection of 5120 rows 1760 us (1828 on the best other tiles), of 7012 rows 2454 (2608), N = 5120,
  // K = 13824 at 4029 rows 452 (484).
  if (may_share && a.K >= 4096 && a.M > 256) {
    const long tiles = n_tiles(a.M, a.N, 256, 256), rem = tiles % n_cu, phases = rem ? n_cu / std::gcd((long)n_cu, rem) : 1;
    const double t = (double)nk * (phases <= 2 ? 1.49 : 1.545) * (double)tiles / (double)n_cu + 22.0 +
                     SHAPES[0].round[epi_column(epilogue)] * (double)((tiles + n_cu - 1) / n_cu);
    if (rem && tiles > n_cu && phases <= 4 && t < best) { a.tile_variant = V_SHARED; a.k_splits = 1; }
  }
}

int gemm_shape(const GemmArgs &a, int epilogue, int dh) {
  if (a.tile_variant) return a.tile_variant;
  if ((epilogue == EPI_SWIGLU || epilogue == EPI_PLAIN) && gemm_streams_weights(a, epilogue)) return V_ROWS;
  const int n_cols = a.n_count ? a.n_count : a.N;
  return choose_variant(a.M, epilogue == EPI_SWIGLU ? 2 * n_cols : n_cols, a.K, epilogue, dh, a.n_cu, a.sk_ws && a.sk_cnt && !a.n_count ? a.K : 0);
}

int gemm_ss_parts(const GemmArgs &a, int epilogue, int dh) {
  if (a.k_splits > 1) return 1;  // the split-K reduction leaves whole row sums
  const int v = a.tile_variant ? a.tile_variant
                               : choose_variant(a.M, a.N, a.K, epilogue, dh, a.n_cu, a.sk_ws && a.sk_cnt && !a.n_count ? a.K : 0);
  if (v == V_ROWS) return (a.N + 15) / 16;  // one per block of 16 columns
  // partial row sums: one per (column tile, wavefront column)
  return v == V_SMALL ? ((a.N + 127) / 128) * 2 : ((a.N + 255) / 256) * 4;
}

int gemm_ride_variant(int m, int n_b_rows, int n_cu) {
  // the eight-wavefront tiles only: 256x256 or 160x256, by the same cost model of rounds
  struct Cand { int v, bm; double T, a; };
  const Cand cands[2] = {{V_BIG, 256, 1.00, 0.72}, {V_TALL, 160, 0.76, 0.65}};
  if (n_cu <= 0) n_cu = N_CU;
  int best = V_BIG;
  double best_t = 1e300;
  for (const Cand &c : cands) {
    const long tiles = n_tiles(m, n_b_rows, c.bm, 256);
    const long full = tiles / n_cu, rem = tiles % n_cu;
    const double t = (double)full * c.T + (rem ? c.T * (c.a + (1.0 - c.a) * (double)rem / (double)n_cu) : 0.0);
    if (t < best_t) { best_t = t; best = c.v; }
  }
  return best;
}

int gemm_ride_tiles(const GemmArgs &a, int epilogue) {
  const int bm = a.tile_variant == V_TALL ? 160 : 256, out_bn = epilogue == EPI_SWIGLU ? 128 : 256;
  return ((a.M + bm - 1) / bm) * ((a.N + out_bn - 1) / out_bn);
}

hipError_t launch_gemm_with_attention(const GemmArgs &a, int epilogue, int dh, const GemmRide &r, hipStream_t stream) {
  (void)dh;
  if (a.k_splits > 1 || a.n_count || r.head < 0 || r.head % XCDS || r.tail < 0 || !r.done || !r.ticket_next || !r.q.ticket)
    return hipErrorInvalidValue;
  const int b_rows = (epilogue == EPI_SWIGLU) ? 2 * a.N : a.N;
  if ((size_t)a.M * a.lda * 2 >= ((size_t)1 << 32) || (size_t)b_rows * a.ldb * 2 >= ((size_t)1 << 32))
    return hipErrorInvalidValue;
  const int v = a.tile_variant ? a.tile_variant : gemm_ride_variant(a.M, b_rows, N_CU - r.head);
  if (v != V_BIG && v != V_TALL) return hipErrorInvalidValue;
  const int adh = r.q.d.s.head_dim;
  if (adh != 64 && adh != 128) return hipErrorInvalidValue;
#define BS_RIDE(EPI)                                                                                  \
  return v == V_BIG ? (adh == 128 ? launch_ride<256, 256, 2, 4, EPI, 128>(a, r, stream)               \
                                  : launch_ride<256, 256, 2, 4, EPI, 64>(a, r, stream))               \
                    : (adh == 128 ? launch_ride<160, 256, 2, 4, EPI, 128>(a, r, stream)               \
                                  : launch_ride<160, 256, 2, 4, EPI, 64>(a, r, stream))
  switch (epilogue) {
    case EPI_RESID_NORM: BS_RIDE(EPI_RESID_NORM);
    case EPI_SWIGLU: BS_RIDE(EPI_SWIGLU);
    case EPI_RESID: BS_RIDE(EPI_RESID);
    default: return hipErrorInvalidValue;
  }
#undef BS_RIDE
}

hipError_t launch_gemm(const GemmArgs &a, int epilogue, int dh, hipStream_t stream) {
  // the kernels address operand rows with 32-bit byte offsets from the matrix base
  if ((size_t)a.M * a.lda * 2 >= ((size_t)1 << 32) ||
      (size_t)((epilogue == EPI_SWIGLU) ? 2 * a.N : a.N) * a.ldb * 2 >= ((size_t)1 << 32))
    return hipErrorInvalidValue;
  if (a.k_splits > 1) {
    if ((epilogue != EPI_RESID && epilogue != EPI_RESID_NORM && epilogue != EPI_QKV) || !a.sk_ws || a.N % 4)
      return hipErrorInvalidValue;
    if (a.k_splits > MAX_SPLITS || (size_t)a.k_splits * a.M * a.N > gemm_sk_workspace_floats() ||
        ((a.tile_variant == V_S128 || a.tile_variant == V_S256) && a.M > (a.tile_variant == V_S128 ? 128 : 256)))
      return hipErrorInvalidValue;
    hipError_t e;
    switch (a.tile_variant) {
      case V_S128: e = launch_one<128, 256, 2, 4, EPI_PARTIAL, 64, DEEP_X>(a, stream); break;
      case V_S256: e = launch_one<256, 128, 4, 2, EPI_PARTIAL, 64, DEEP_X>(a, stream); break;
      case V_BIG: e = launch_one<256, 256, 2, 4, EPI_PARTIAL, 64>(a, stream); break;
      case V_TALL: e = launch_one<160, 256, 2, 4, EPI_PARTIAL, 64>(a, stream); break;
      case V_SMALL: e = launch_one<128, 128, 2, 2, EPI_PARTIAL, 64>(a, stream); break;
      case V_MID: e = launch_one<192, 256, 2, 4, EPI_PARTIAL, 64>(a, stream); break;
      case V_WIDE: e = launch_one<128, 256, 2, 4, EPI_PARTIAL, 64>(a, stream); break;
      default: return hipErrorInvalidValue;
    }
    if (e != hipSuccess) return e;
    if (epilogue == EPI_QKV) {
      const int items = ((a.n_q_heads + a.n_kv_heads) * (dh / 2) + a.n_kv_heads * dh) / 4;
      hipLaunchKernelGGL(splitk_reduce_qkv_kernel, dim3(a.M, (items + 255) / 256), dim3(256), 0, stream, a, dh);
    } else if (epilogue == EPI_RESID) {
      hipLaunchKernelGGL(splitk_reduce_resid_kernel, dim3(a.M, (a.N / 4 + 255) / 256), dim3(256), 0, stream, a);
    } else {
      const int threads = std::min(1024, (a.N / 4 + 63) / 64 * 64);
      hipLaunchKernelGGL(splitk_reduce_resid_norm_kernel, dim3(a.M), dim3(threads), 0, stream, a);
    }
    return hipGetLastError();
  }
  if (a.n_count && epilogue != EPI_SWIGLU && epilogue != EPI_PLAIN) return hipErrorInvalidValue;
  const int v = gemm_shape(a, epilogue, dh);
  if (v == V_ROWS) {
    switch (rows_item(a.M, a.N, a.K, epilogue, a.n_cu > 0 ? a.n_cu : N_CU)) {
      case 11: return launch_rows_one<1, 1>(a, epilogue, dh, stream);
      case 21: return launch_rows_one<2, 1>(a, epilogue, dh, stream);
      case 22: return launch_rows_one<2, 2>(a, epilogue, dh, stream);
      default: return hipErrorInvalidValue;
    }
  }
  switch (epilogue) {
    case EPI_PLAIN: return launch_variant<EPI_PLAIN>(a, v, stream);
    case EPI_RESID: return launch_variant<EPI_RESID>(a, v, stream);
    case EPI_RESID_NORM: return launch_variant<EPI_RESID_NORM>(a, v, stream);
    case EPI_SWIGLU: return launch_variant<EPI_SWIGLU>(a, v, stream);
    case EPI_QKV:
      if (dh == 128) return launch_qkv<128>(a, v, stream);
      if (dh == 64) return launch_qkv<64>(a, v, stream);
      return hipErrorInvalidValue;
    default:
      return hipErrorInvalidValue;
  }
}

}  // namespace bs

// Device code of the products: tiles through LDS rings (gemm_tile) and the stream of weights past few rows (gemm_rows), see gemm.hip.
// The file that includes this defines g_gemm_zero_chunk, sixteen bytes of zeros on the device: the source of tile chunks that lie beyond K.
// Products of 8-bit integers (w8.hip) take both with rows of K / 2 bf16 numbers' bytes: where things lie, and travel, is a matter of bytes.
#pragma once
#include <type_traits>
#include <utility>

#include "attn_device.hpp"
#include "common.hpp"
#include "gemm.hpp"
#include "k_order.hpp"

namespace bs {
namespace {

constexpr int BK = K_TILE;  // k-extent of one k-tile: rows of 128 bytes
constexpr int LDS_CU = 160 * 1024;
// the panel ring of a workgroup: all of a CU's LDS, or half where two workgroups of four wavefronts share a CU; three
// weight panels, as many activation panels as fit beside them (three are enough), and what is left to weights again
constexpr int ring_bytes(int waves) { return waves > 4 ? LDS_CU : LDS_CU / 2; }
constexpr int ring_x_slots(int bm, int bn, int waves) {
  const int n = (ring_bytes(waves) - 3 * bn * BK * 2) / (bm * BK * 2);
  return n < 3 ? n : 3;
}
constexpr int ring_w_slots(int bm, int bn, int waves) { return (ring_bytes(waves) - ring_x_slots(bm, bn, waves) * bm * BK * 2) / (bn * BK * 2); }
constexpr int XCDS = 8;

struct TileCoord { int tm, tn; };
struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// Workgroup ids are dealt round-robin to the 8 XCDs; give each XCD a contiguous
// range of tiles and walk that range in groups of GM tile rows, so the tiles in
// flight on one XCD share activation and weight panels in that XCD's L2.
__device__ __forceinline__ TileCoord map_tile(int pid, int n_tiles, int tiles_m, int tiles_n) {
  const int per = n_tiles / XCDS, rem = n_tiles % XCDS;
  const int xcd = pid % XCDS, idx = pid / XCDS;
  const int lin = xcd * per + (xcd < rem ? xcd : rem) + idx;
  constexpr int GM = 4;
  const int group = GM * tiles_n;
  const int g = lin / group;
  const int first_m = g * GM;
  const int gm = (tiles_m - first_m) < GM ? (tiles_m - first_m) : GM;
  const int in = lin - g * group;
  TileCoord t;
  t.tm = first_m + in % gm;
  t.tn = in / gm;
  return t;
}

__device__ __forceinline__ void store_bf16x4(uint16_t *p, float a, float b, float c, float d) {
  u32x2_t v;
  v.x = pack_bf16x2(a, b);
  v.y = pack_bf16x2(c, d);
  *reinterpret_cast<u32x2_t *>(p) = v;
}

// Columns of the fused projection enter the tiles in groups of 64: 32 features of a head and those dh/2 behind them, so
// that rotation pairs meet in a lane.  Groups of value heads are dealt evenly between the others: the rows of
// decode sequences store them two bytes at a time, one lane per clock, 28 us for a 256x256 tile of nothing else
// (QKV of 1093 prefill and 487 decode rows 111 -> 106 us against the columns in their own order).
struct QkvGroup { int head, i0; };  // features i0 .. i0 + 31 and i0 + dh/2 .. of the head; head >= all of them: beyond the last
__device__ __forceinline__ QkvGroup qkv_group(int p, const GemmArgs &a, int dh) {
  const int per_head = dh / 64, n_v = a.n_kv_heads * per_head, n_rot = (a.n_q_heads + a.n_kv_heads) * per_head, n = n_rot + n_v;
  const int v = (int)((unsigned)(p * n_v) / (unsigned)n);
  const int g = p >= n ? n : (int)((unsigned)((p + 1) * n_v) / (unsigned)n) > v ? n_rot + v : p - v;
  return QkvGroup{g / per_head, g % per_head * 32};
}

// s_waitcnt immediate (gfx9 encoding): wait until at most `vm` vector-memory
// operations are outstanding and, if lgkm0, until all LDS reads have returned
constexpr int waitcnt_imm(int vm, bool lgkm0) {
  return (vm & 0xF) | ((vm >> 4) << 14) | 0x70 | (lgkm0 ? 0 : 0xF00);
}

// Shared tiles.  A launch of G persistent workgroups takes the tiles [0, n_dp) of the launch's
// tile order whole, workgroup w the tiles w, w + G, ...; the k-tiles of the other n_sk tiles
// form one line of n_sk * nk iterations that the first g_sk workgroups cut into equal
// consecutive ranges, so a tile at a cut is computed by two or more workgroups, each over a
// part of K.  Every such workgroup leaves its partial tile in the workspace and counts itself
// in; the one that arrives last adds the parts up (always in the order of their k-ranges,
// its own part re-read like the others, so the sum does not depend on who was last) and runs
// the epilogue.  Nobody waits for anybody.
struct SkPlan {
  int n_dp, n_sk, g_sk, nk;
  float *ws;      // [2 * G][BM * BN]: slot 2 w of workgroup w for its first segment, 2 w + 1 for its last
  unsigned *cnt;  // [n_sk] arrivals at each shared tile; zero between launches
};
struct SkSeg {
  int pid, kt0, kt1;  // tile, k-tiles [kt0, kt1)
  int j;              // index of the tile among the shared ones
  int parts;          // workgroups that hold a part of the tile (1: this one has all of it)
  int w_first;        // the first of them; they are consecutive
  int my_slot;
};
constexpr int SK_SNAP = 4;      // a cut this close to a tile boundary moves onto it
constexpr int SK_MIN_ITERS = 16;  // shortest range worth a workgroup of its own

// first iteration of workgroup w's range (w = g_sk: the end of the line)
__device__ __forceinline__ int sk_bound(const SkPlan &p, int w) {
  const int total = p.n_sk * p.nk;
  int b = (int)((long)total * w / p.g_sk);
  const int r = b % p.nk;
  if (r < SK_SNAP) b -= r;
  else if (p.nk - r < SK_SNAP) b += p.nk - r;
  return b;
}
// the workgroups whose ranges meet shared tile j
__device__ __forceinline__ void sk_tile_span(const SkPlan &p, int j, int *w_first, int *parts) {
  const int lo = j * p.nk, hi = lo + p.nk;
  int w = (int)((long)lo * p.g_sk / (p.n_sk * p.nk));
  while (w + 1 < p.g_sk && sk_bound(p, w + 1) <= lo) ++w;
  while (w > 0 && sk_bound(p, w) > lo) --w;
  int n = 1;
  while (w + n < p.g_sk && sk_bound(p, w + n) < hi) ++n;
  *w_first = w;
  *parts = n;
}

// The accumulators of a product and the matrix instruction behind them: bf16 into 32-bit numbers, or 8-bit into 32-bit integers.
template <bool I8>
using GemmAcc = std::conditional_t<I8, i32x4_t, f32x4_t>;
__device__ __forceinline__ void gemm_mfma(f32x4_t &c, bf16x8_t w, bf16x8_t x) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }
__device__ __forceinline__ void gemm_mfma(i32x4_t &c, bf16x8_t w, bf16x8_t x) {
  c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, w), __builtin_bit_cast(i32x4_t, x), c, 0, 0, 0);
}
constexpr bool gemm_in_integers(int epi) { return epi == EPI_W8 || epi == EPI_W8_PARTIAL; }

// Sums of products of 8-bit integers as 32-bit numbers.  131072 products of -128 and -128 are 2^31, which 32 bits hold as -2^31; every other sum
// is more than that by 2^24 at least (127 * 128 * 131072), and so is what it is rounded to.
constexpr int W8_LONG = 131072 / 2;  // GemmArgs::K of such sums
__device__ __forceinline__ f32x4_t w8_sums(i32x4_t s) {
  f32x4_t v = __builtin_convertvector(s, f32x4_t);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = v[e] == -0x1p31f ? 0x1p31f : v[e];
  return v;
}

// A row's scale as its sums are multiplied by it, and what a result is multiplied by last: a sum is up to 2^31, so that times a scale of 2^96 and more
// leaves the range of 32 bits where the result, with an output's scale, need not.
struct W8RowScale {
  float scale, back;
  __device__ __forceinline__ explicit W8RowScale(float s) {
    const bool far = fabsf(s) >= 0x1p96f;
    scale = far ? s * 0x1p-32f : s;
    back = far ? 0x1p32f : 1.f;
  }
};

// four neighbouring results of a row, of which those below n_lim exist
__device__ __forceinline__ void store_scaled4(uint16_t *p, f32x4_t v, int n, int n_lim, bool aligned) {
  if (aligned && n + 4 <= n_lim) {
    store_bf16x4(p, v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < n_lim) p[e] = f32_to_bf16(v[e]);
  }
}

// One workgroup's tile; `bid` is the workgroup's number among the GEMM workgroups of the launch
// (SK: the tile and the k-range come from `seg` instead).
template <int BM, int BN, int WAVES_M, int WAVES_N, int EPI, int DH, int DEEP = 0, bool SK = false>
__device__ __forceinline__ void gemm_tile(const GemmArgs &a, const int bid, const SkPlan *sp = nullptr, const SkSeg seg = SkSeg{}) {
  constexpr bool I8 = gemm_in_integers(EPI), PART = EPI == EPI_PARTIAL || EPI == EPI_W8_PARTIAL;
  typedef GemmAcc<I8> Acc;
  static_assert(!SK || (!DEEP && !PART && !I8), "shared tiles use the two rings of whole tiles and a real epilogue");
  constexpr int NW = WAVES_M * WAVES_N;
  // DEEP: the pipeline for one round of tiles over few rows, where every CU streams a weight
  // panel of its own from HBM; the first half of the wavefronts requests the activation
  // panels, the second half the weight panels (see the pipeline below)
  constexpr int XW = DEEP ? NW / 2 : NW, WW = DEEP ? NW / 2 : NW;  // wavefronts that share the loads of a panel
  constexpr int WTM = BM / WAVES_M, WTN = BN / WAVES_N;
  constexpr int MI = WTM / 16, NI = WTN / 16;  // 16x16 accumulator blocks of a wavefront's tile
  constexpr int OUT_BN = (EPI == EPI_SWIGLU) ? BN / 2 : BN;
  constexpr int ROWB = BK * 2;                       // bytes of one tile row
  constexpr int LDS_BYTES = DEEP ? LDS_CU : ring_bytes(NW);
  constexpr int GA = BM / 8, GB = BN / 8;            // 8-row groups = one 1 KB wavefront load each
  constexpr int LA = (GA + XW - 1) / XW, LB = (GB + WW - 1) / WW;  // loads per thread per panel
  static_assert(!DEEP || NW % 2 == 0, "two halves of the workgroup share the loads");
  static_assert(BK == 64, "swizzle and fragment addressing assume 128-byte tile rows");
  static_assert(WTM % 16 == 0 && WTN % 16 == 0, "tiles are made of 16x16 MFMA blocks");
  static_assert(EPI != EPI_SWIGLU || WTN % 64 == 0, "32 gate rows and their 32 up rows pair up inside a wave");
  static_assert(EPI != EPI_QKV || (WTN % 64 == 0 && BN % DH == 0), "32 pairs of a head's features meet inside a wave");
  static_assert(2 * LA + 2 * LB < 64, "outstanding loads must fit the vmcnt field");

  extern __shared__ __align__(16) unsigned char smem[];

  const int n_lim = a.n_count ? a.n_begin + a.n_count : a.N;  // end of the output columns of this launch
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (n_lim - a.n_begin + OUT_BN - 1) / OUT_BN;
  // split-K: consecutive workgroups are the k-ranges of one tile
  const int split = PART ? bid % a.k_splits : 0;
  const int tile_id = SK ? seg.pid : PART ? bid / a.k_splits : bid;
  const TileCoord tc = map_tile(tile_id, tiles_m * tiles_n, tiles_m, tiles_n);
  const int m0 = tc.tm * BM, n0 = a.n_begin + tc.tn * OUT_BN;

  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm0 = (wave / WAVES_N) * WTM, wn0 = (wave % WAVES_N) * WTN;
  const int lr = lane & 15, lg = lane >> 4;  // row of a 16-row block; k-chunk of a fragment, feature group of an accumulator

  // ---- global -> LDS, without passing through registers ---------------------------
  // One wavefront load moves 8 tile rows (1 KB): lane i lands at LDS byte 16 i of the
  // group, i.e. row i/8, 16-byte slot i%8, and fetches the chunk that the XOR swizzle
  // assigns to that slot, so the eight lanes of a row cover one whole cache line.  Rows
  // past the matrix edge are clamped to the last row (their accumulators are never
  // stored); chunks past K read a block of zeros instead.
  const int g_row = lane >> 3, g_slot = lane & 7;
  // byte offsets from the matrix base (the host checks that they fit 32 bits): the address
  // of a load is then a uniform 64-bit base, advanced per k-tile by scalar code, plus a
  // per-lane offset that never changes
  uint32_t off_a[LA], off_b[LB];
  int ka[LA], kb[LB];        // element offset of this lane's chunk inside a k-tile
  int dst_a[LA], dst_b[LB];  // LDS byte offset of the group inside a unit
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    // when the groups do not divide over the wavefronts the surplus loads repeat the last
    // group (same bytes to the same place), so every wavefront issues LA loads per panel
    const int grp = (wave % XW + i * XW) < GA ? (wave % XW + i * XW) : GA - 1;
    const int row = grp * 8 + g_row;
    const int chunk = g_slot ^ ((row >> 1) & 7);
    ka[i] = chunk * 8;
    dst_a[i] = grp * 1024;
    int gm = m0 + row;
    gm = gm < a.M ? gm : a.M - 1;
    off_a[i] = (uint32_t)(((size_t)gm * a.lda + chunk * 8) * 2);
  }
#pragma unroll
  for (int i = 0; i < LB; ++i) {
    const int grp = (wave % WW + i * WW) < GB ? (wave % WW + i * WW) : GB - 1;
    const int wr = grp * 8 + g_row;
    const int chunk = g_slot ^ ((wr >> 1) & 7);
    kb[i] = chunk * 8;
    dst_b[i] = grp * 1024;
    int gn;
    if (EPI == EPI_SWIGLU) {
      const int blk = wr >> 5;
      int col = n0 + (blk >> 1) * 32 + (wr & 31);
      col = col < a.N ? col : a.N - 1;
      gn = col + ((blk & 1) ? a.N : 0);
    } else if (EPI == EPI_QKV) {
      const QkvGroup q = qkv_group((n0 + wr) >> 6, a, DH);
      gn = q.head * DH + q.i0 + (wr & 31) + ((wr & 32) ? DH / 2 : 0);
      gn = gn < a.N ? gn : a.N - 1;
    } else {
      gn = n0 + wr;
      gn = gn < a.N ? gn : a.N - 1;
    }
    off_b[i] = (uint32_t)(((size_t)gn * a.ldb + chunk * 8) * 2);
  }
  constexpr bool TURNED = DEEP && !PART && BM <= 128;
  const int nk_whole = (a.K + BK - 1) / BK;
  const int first_kt = TURNED ? first_k_tile(tile_id, a.K, a.ldb) : 0;
  auto turned_kt = [&](int kt) {
    if (!TURNED || kt >= nk_whole) return kt;
    return kt + first_kt >= nk_whole ? kt + first_kt - nk_whole : kt + first_kt;
  };
  // load number i of panel X(kt) / W(kt) to LDS byte offset `lds_off`; `checked` handles chunks past K.  Buffer loads take the
  // k-tile as a scalar offset: no address arithmetic per load, and 16 registers less than 64-bit addresses.
#ifdef __HIP_DEVICE_COMPILE__
  const __amdgpu_buffer_rsrc_t rsrc_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(a.A), 0, 0xffffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t rsrc_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t *>(a.B), 0, 0xffffffff, 0x00020000);
#else
  const int rsrc_a = 0, rsrc_b = 0;
#endif
  auto dma = [&](const uint16_t *mat, auto rsrc, int kt, uint32_t off, int ke, int lds_off, auto checked) {
    kt = turned_kt(kt);
#ifdef __HIP_DEVICE_COMPILE__
    auto *dst = (__attribute__((address_space(3))) void *)(smem + lds_off);
    if constexpr (decltype(checked)::value) {
      const void *p = reinterpret_cast<const unsigned char *>(mat) + (size_t)kt * ROWB + off;
      if (kt * BK + ke >= a.K) p = g_gemm_zero_chunk;
      __builtin_amdgcn_global_load_lds(p, dst, 16, 0, 0);
    } else {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, dst, 16, off, kt * ROWB, 0, 0);
    }
#endif
  };
  auto dma_a = [&](int kt, int lds_off, int i, auto checked) { dma(a.A, rsrc_a, kt, off_a[i], ka[i], lds_off + dst_a[i], checked); };
  auto dma_b = [&](int kt, int lds_off, int i, auto checked) { dma(a.B, rsrc_b, kt, off_b[i], kb[i], lds_off + dst_b[i], checked); };

  Acc acc[NI][MI];
#pragma unroll
  for (int ni = 0; ni < NI; ++ni)
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) acc[ni][mi] = Acc{0, 0, 0, 0};

  // fragment addresses: tile row of the lane, chunk 4*ks + lg swizzled by ((row >> 1) & 7)
  const int sw = (lr >> 1) & 7;
  const int xfrag = (wm0 + lr) * ROWB;
  const int wfrag = (wn0 + lr) * ROWB;

  const int nk_all = (a.K + BK - 1) / BK;
  // this workgroup's k-tiles [kt0, kt1): all of them, or one of k_splits nearly equal ranges
  const int kt0 = SK ? seg.kt0 : PART ? (int)((long)nk_all * split / a.k_splits) : 0;
  const int kt1 = SK ? seg.kt1 : PART ? (int)((long)nk_all * (split + 1) / a.k_splits) : nk_all;
  constexpr int NF = MI + NI;   // fragment reads per 32-wide k-step
  constexpr int NMF = MI * NI;  // MFMAs per 32-wide k-step
  // read number o of k-step ks (32 wide, two per tile) of the panels in ring slots sa, sb
  // (xo, wo: LDS byte offsets of the two panels)
  auto frag = [&](int xo, int wo, int ks, int o, bf16x8_t (&xf)[MI], bf16x8_t (&wf)[NI]) {
    const int ch = ((ks * 4 + lg) ^ sw) << 4;
    if (o < MI)
      xf[o] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(smem + xo + xfrag + o * 16 * ROWB + ch));
    else
      wf[o - MI] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(smem + wo + wfrag + (o - MI) * 16 * ROWB + ch));
  };
  // One k-step: its NMF MFMAs in program order, with `n_ops` side operations (LDS reads of the next k-step, DMA
  // requests) dealt out between them, operation o behind MFMA at(o), so that the matrix pipe is never left idle
  // behind a run of memory instructions.
  auto step = [&](const bf16x8_t (&xf)[MI], const bf16x8_t (&wf)[NI], int n_ops, auto &&at, auto &&op) {
#pragma unroll
    for (int j = 0; j < NMF; ++j) {
      const int ni = j / MI, mi = j % MI;
      gemm_mfma(acc[ni][mi], wf[ni], xf[mi]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int o = 0; o < n_ops; ++o)
        if (at(o) == j) op(o);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Where the operations of a k-step go: NF reads, then `n_dma` requests.  A request keeps the CU's address unit busy for
  // 16 to 24 clocks, and eight wavefronts that ask for eight KB each without a pause stand still behind one another, MFMAs
  // and all: a request every third MFMA (every second where a step is short), reads in between.
  // (The deep ring, bound by its weight stream, asks as early as it can: 256 rows, N = 4096, K = 14336 43.4 against 44.8 us.)
  constexpr auto place = [](int o, int n_dma) {
    if (DEEP) return o * NMF / (NF + n_dma > NMF ? NF + n_dma : NMF);
    const int pitch = 3 * n_dma - 1 <= NMF ? 3 : 2;
    const int j = o >= NF ? pitch - 1 + pitch * (o - NF) : pitch == 3 ? o + o / 2 : o;
    return j < NMF ? j : NMF - 1;
  };
  // LDS -> registers: the fragments of the next 32-wide k-step are requested while the MFMAs of the current one are
  // issued, across tile boundaries too, so the matrix pipe never waits for a whole LDS read phase.
  // The compiler counts an LDS-DMA load as a pending LDS operation of unknown order, so
  // every wait it places before an MFMA is lgkmcnt(0); waiting explicitly at the start of
  // a k-step, for reads issued during the first MFMAs of the previous one, keeps those
  // waits from covering reads that were only just issued.
  constexpr int LGKM0 = waitcnt_imm(63, true);
  constexpr int UX = BM * ROWB, UW = BN * ROWB;  // bytes of a panel
  bf16x8_t xa[MI], wa[NI], xb[MI], wb[NI];
  if constexpr (!DEEP) {
    // Panel X(kt) lives in activation slot kt % NXS, W(kt) in weight slot kt % NWS.  Once the last fragments of tile kt
    // are in registers, at the one barrier of the iteration, X(kt+NXS) and W(kt+NWS) are requested into the two slots
    // that tile kt frees: the weight panel, which in a layer streams from HBM, has two k-tiles of look-ahead, and the
    // activation panel, which the previous kernel has just left in the caches, one, or two where three slots fit.
    constexpr int NXS = ring_x_slots(BM, BN, NW), NWS = ring_w_slots(BM, BN, NW), W_BASE = NXS * UX;
    constexpr int AHEAD = NXS > NWS ? NXS : NWS;
    // loads requested after both panels of the next tile, and so still in flight when these have landed
    constexpr int YOUNG = NXS < NWS ? (NXS - 2) * (LA + LB) + LB : (NWS - 2) * (LA + LB);
    static_assert(NXS >= 2 && NWS >= 2 && W_BASE + NWS * UW <= LDS_BYTES && NXS * LA + NWS * LB < 64, "slots and the vmcnt field");
#pragma unroll
    for (int r = -AHEAD; r < 0; ++r) {
      if (r + NXS >= 0)
#pragma unroll
        for (int i = 0; i < LA; ++i) dma_a(kt0 + r + NXS, (r + NXS) * UX, i, Yes{});
      if (r + NWS >= 0)
#pragma unroll
        for (int i = 0; i < LB; ++i) dma_b(kt0 + r + NWS, W_BASE + (r + NWS) * UW, i, Yes{});
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_imm(YOUNG + LA + LB, true));  // tile 0 has landed
    __builtin_amdgcn_s_barrier();
    int xo = 0, wo = W_BASE;  // slots of the tile being multiplied
#pragma unroll
    for (int o = 0; o < NF; ++o) frag(xo, wo, 0, o, xa, wa);
    auto tile = [&](int kt, auto checked) {
      __builtin_amdgcn_s_waitcnt(LGKM0);
      step(xa, wa, NF, [&](int o) { return place(o, 0); }, [&](int o) { frag(xo, wo, 1, o, xb, wb); });
      // Every fragment of tile kt is in registers once the LDS reads have returned, and
      // tile kt+1 has landed once this wavefront's loads other than the YOUNG last ones
      // are done; after the barrier both hold for every wavefront, so the two
      // slots of tile kt can be refilled and tile kt+1 can be read.
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(YOUNG, true));
      __builtin_amdgcn_s_barrier();
      const int nx = xo == (NXS - 1) * UX ? 0 : xo + UX, nw = wo == W_BASE + (NWS - 1) * UW ? W_BASE : wo + UW;
      step(xb, wb, NF + LA + LB, [&](int o) { return place(o, LA + LB); }, [&](int o) {
        if (o < NF)
          frag(nx, nw, 0, o, xa, wa);
        else if (o < NF + LA)
          dma_a(kt + NXS, xo, o - NF, checked);
        else
          dma_b(kt + NWS, wo, o - NF - LA, checked);
      });
      xo = nx;
      wo = nw;
    };
    int kt = kt0;
    const int n_plain = a.K / BK - AHEAD;  // tiles kt for which X(kt+NXS) and W(kt+NWS) lie wholly inside K
    for (; kt < n_plain && kt < kt1; ++kt) tile(kt, No{});
    for (; kt < kt1; ++kt) tile(kt, Yes{});
  } else {
    // One round of tiles over few rows: every CU streams a weight panel of its own from HBM,
    // and the rings above give it two k-tiles of look-ahead at most.  Here LDS
    // holds NXS = DEEP + 1 slots for the activation panel (shared by all tiles, served by the
    // L2: NXS - 1 k-tiles of look-ahead) and all the rest, NWS slots, for the weight panel:
    // NWS - 1 k-tiles of look-ahead.  The memory counter of a wavefront retires its loads in
    // order, so a wait for an activation panel would also wait for every weight panel
    // requested before it; the two kinds of request therefore come from different wavefronts:
    // the first half of the workgroup loads activations and waits until its NXS - 2 youngest
    // panels remain, the second half loads weights and waits until its NWS - 2 youngest remain.
    constexpr int NXS = DEEP + 1;  // activation slots
    constexpr int W_BASE = NXS * UX;
    constexpr int NWS = (LDS_BYTES - W_BASE) / UW;
    static_assert(NWS >= 3 && (NWS - 1) * LB < 64 && (NXS - 1) * LA < 64, "slots and the vmcnt field");
    const bool loads_x = wave < XW;  // uniform
    if (loads_x) {
#pragma unroll
      for (int sl = 0; sl < NXS; ++sl)
#pragma unroll
        for (int i = 0; i < LA; ++i) dma_a(kt0 + sl, sl * UX, i, Yes{});
      __builtin_amdgcn_s_waitcnt(waitcnt_imm((NXS - 1) * LA, true));
    } else {
#pragma unroll
      for (int sl = 0; sl < NWS; ++sl)
#pragma unroll
        for (int i = 0; i < LB; ++i) dma_b(kt0 + sl, W_BASE + sl * UW, i, Yes{});
      __builtin_amdgcn_s_waitcnt(waitcnt_imm((NWS - 1) * LB, true));
    }
    __builtin_amdgcn_s_barrier();  // tile 0 has landed
    int xs = 0, ws = 0;            // activation and weight slot numbers of the tile being multiplied
#pragma unroll
    for (int o = 0; o < NF; ++o) frag(xs * UX, W_BASE + ws * UW, 0, o, xa, wa);
    auto tile = [&](int kt, auto checked) {
      const int wo = W_BASE + ws * UW, xo = xs * UX;
      __builtin_amdgcn_s_waitcnt(LGKM0);
      step(xa, wa, NF, [&](int o) { return place(o, 0); }, [&](int o) { frag(xo, wo, 1, o, xb, wb); });
      // after the barrier: every wavefront holds all fragments of tile kt, X(kt+1) has landed
      // (the activation half waited until only X(kt+2) .. X(kt+NXS-1) were outstanding) and so
      // has W(kt+1) (the weight half: only W(kt+2) .. W(kt+NWS-1))
      if (loads_x)
        __builtin_amdgcn_s_waitcnt(waitcnt_imm((NXS - 2) * LA, true));
      else
        __builtin_amdgcn_s_waitcnt(waitcnt_imm((NWS - 2) * LB, true));
      __builtin_amdgcn_s_barrier();
      const int nxs = xs + 1 == NXS ? 0 : xs + 1, nws = ws + 1 == NWS ? 0 : ws + 1;
      const int nxo = nxs * UX;
      const int nwo = W_BASE + nws * UW;
      if (loads_x)
        step(xb, wb, NF + LA, [&](int o) { return place(o, LA); }, [&](int o) {
          if (o < NF)
            frag(nxo, nwo, 0, o, xa, wa);
          else
            dma_a(kt + NXS, xo, o - NF, checked);
        });
      else
        step(xb, wb, NF + LB, [&](int o) { return place(o, LB); }, [&](int o) {
          if (o < NF)
            frag(nxo, nwo, 0, o, xa, wa);
          else
            dma_b(kt + NWS, wo, o - NF, checked);
        });
      xs = nxs;
      ws = nws;
    };
    int kt = kt0;
    const int n_plain = a.K / BK - (NWS > NXS ? NWS : NXS);  // tiles kt for which X(kt+NXS) and W(kt+NWS) lie wholly inside K
    for (; kt < n_plain && kt < kt1; ++kt) tile(kt, No{});
    for (; kt < kt1; ++kt) tile(kt, Yes{});
  }
  // drain the look-ahead loads (zeros or clamped rows) before the LDS is released
  __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, true));
  if (EPI != EPI_SWIGLU) __syncthreads();  // results pass through LDS on their way out: nobody may still be reading panels there

  if constexpr (SK) {
    if (seg.parts > 1) {
      constexpr int NT = NW * 64;
      constexpr size_t TILE = (size_t)BM * BN;
      // The register image of the accumulators, 16 bytes per thread and block (whoever adds the
      // parts up has the same layout).  The eight XCDs keep L2 caches of their own, so parts
      // written and read with ordinary accesses would need the whole-cache write-back and
      // invalidation of a device-wide fence at every cut (measured: a quarter of a millisecond
      // per launch); the parts travel with the device-scope cache policy instead (sc1: to and
      // from the point where all XCDs agree), which touches nothing else.
      typedef unsigned int u4_t __attribute__((ext_vector_type(4)));
      constexpr int SC1 = 16;
      const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(sp->ws, 0, 0x7fffffff, 0x00020000);
      const unsigned voff = (unsigned)t * 16u;
      {
        const unsigned soff = (unsigned)seg.my_slot * (unsigned)(TILE * 4);
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
          for (int mi = 0; mi < MI; ++mi) {
            const f32x4_t c = acc[ni][mi];
            const u4_t v = {__float_as_uint(c[0]), __float_as_uint(c[1]), __float_as_uint(c[2]), __float_as_uint(c[3])};
            __builtin_amdgcn_raw_buffer_store_b128(v, rs, voff + (unsigned)((ni * MI + mi) * NT * 16), soff, SC1);
          }
      }
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(0, true));  // the part has arrived there before the workgroup counts itself in
      __syncthreads();
      volatile unsigned *flag = reinterpret_cast<volatile unsigned *>(smem + LDS_BYTES - 16);
      if (t == 0) *flag = atomicAdd(sp->cnt + seg.j, 1u);
      __syncthreads();
      if (*flag + 1u != (unsigned)seg.parts) return;
      if (t == 0) atomicExch(sp->cnt + seg.j, 0u);  // as the next launch expects it
      for (int q = 0; q < seg.parts; ++q) {
        const int w2 = seg.w_first + q;
        const int slot = 2 * w2 + (sk_bound(*sp, w2) / sp->nk == seg.j ? 0 : 1);
        const unsigned soff = (unsigned)slot * (unsigned)(TILE * 4);
        // sixteen blocks at a time: the loads of a batch are all in flight before the first is
        // used (each is a round trip past the L2; the registers of the fragments are free now)
        constexpr int NB = NI * MI, BATCH = NB < 16 ? NB : 16;
        static_assert(NB % BATCH == 0, "whole batches");
#pragma unroll
        for (int b0 = 0; b0 < NB; b0 += BATCH) {
          u4_t v[BATCH];
#pragma unroll
          for (int b = 0; b < BATCH; ++b)
            v[b] = __builtin_amdgcn_raw_buffer_load_b128(rs, voff + (unsigned)((b0 + b) * NT * 16), soff, SC1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < BATCH; ++b) {
            const int ni = (b0 + b) / MI, mi = (b0 + b) % MI;
            const f32x4_t c = {__uint_as_float(v[b].x), __uint_as_float(v[b].y), __uint_as_float(v[b].z), __uint_as_float(v[b].w)};
            acc[ni][mi] = q == 0 ? c : acc[ni][mi] + c;
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }

  // ---- epilogues ---------------------------------------------------------------
  // accumulator element e of block (ni, mi): m = m0 + wm0 + mi*16 + lr, n = n_tile + wn0 + ni*16 + 4*lg + e.
  // Neighbouring lanes hold neighbouring ROWS, and a CU serves loads and stores of such lanes at about one lane per
  // clock.  The wavefront therefore turns its 64 columns round in LDS, CM blocks of 16 rows at a time, and comes back with
  // sixteen lanes along a row: 16 tiles of 256x256 with K = 64, launch included, output projection 28 -> 17 us, down
  // projection 15.8 -> 12.5, QKV 15.8 -> 12.7; 8192 rows of the 8B layer 287 -> 248, 756 -> 737, 353 -> 333.
  static_assert(WTN == 64, "an epilogue hands 64 columns to 16 lanes");
  constexpr int CM = MI <= 4 ? MI : (MI + 1) / 2;
  constexpr int RS = 64 * 4 + 16;  // bytes of a row of 64 floats: rows four banks apart
  static_assert(NW * CM * 16 * RS <= LDS_BYTES, "the turned blocks fit the panel ring");
  unsigned char *turned = smem + wave * (CM * 16 * RS);
  float row_scale[MI];
  if constexpr (EPI == EPI_W8) {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) row_scale[mi] = a.row_scale[min(m0 + wm0 + mi * 16 + lr, a.M - 1)];
  }
  constexpr int BACK = 64 * 4;  // where W8RowScale::back of a turned row stands, behind its numbers
  // blocks [c, c + CM) of rows into LDS (read and written by this wavefront alone, whose LDS operations complete in order);
  // whole_range: sums and scales of integers of any size
  auto turn = [&](int c, auto whole_range) {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < CM; ++j)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
        if (c + j < MI) {
          unsigned char *row = turned + (j * 16 + lr) * RS, *to = row + (ni * 16 + 4 * lg) * 4;
          if constexpr (EPI == EPI_W8 && decltype(whole_range)::value) {
            const W8RowScale by(row_scale[c + j]);
            *reinterpret_cast<f32x4_t *>(to) = w8_sums(__builtin_bit_cast(i32x4_t, acc[ni][c + j])) * by.scale;
            if (ni == 0 && lg == 0) *reinterpret_cast<float *>(row + BACK) = by.back;
          } else if constexpr (EPI == EPI_W8) {
            *reinterpret_cast<f32x4_t *>(to) = __builtin_convertvector(acc[ni][c + j], f32x4_t) * row_scale[c + j];
          } else {
            *reinterpret_cast<Acc *>(to) = acc[ni][c + j];
          }
        }
    __builtin_amdgcn_wave_barrier();
  };
  constexpr auto rows_in = [](int c) { return (MI - c < CM ? MI - c : CM) * 16; };
  const int r16 = lane >> 4, c16 = 4 * (lane & 15);  // four rows of 64 columns per step

  if constexpr (EPI == EPI_PARTIAL || EPI == EPI_PLAIN || EPI == EPI_RESID || EPI == EPI_RESID_NORM) {
    const int n = n0 + wn0 + c16;
    const bool n_ok = n < n_lim;
    const int nc = min(n, a.N - 4);  // loads beyond an edge repeat the last column or row
    constexpr int U = 4;             // steps of four rows whose residuals are in flight
    float *ws = a.sk_ws + (size_t)split * a.M * a.N;
    f32x4_t gain = {0.f, 0.f, 0.f, 0.f};
    auto bf16x4 = [](u32x2_t v) {
      return f32x4_t{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u)};
    };
    if constexpr (EPI == EPI_RESID_NORM) gain = bf16x4(*reinterpret_cast<const u32x2_t *>(a.gain + nc));
    auto resid = [&](int row) -> f32x4_t {
      const size_t at = (size_t)min(m0 + wm0 + row, a.M - 1) * a.ldr + nc;
      if (EPI == EPI_RESID && a.resid32) return *reinterpret_cast<const f32x4_t *>(a.resid32 + at);
      return bf16x4(*reinterpret_cast<const u32x2_t *>(a.resid + at));
    };
    constexpr bool ADDS = EPI == EPI_RESID || EPI == EPI_RESID_NORM;
    f32x4_t r[U];
    if constexpr (ADDS) {
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = resid(4 * u + r16);
    }
#pragma unroll
    for (int c = 0; c < MI; c += CM) {
      turn(c, No{});
#pragma unroll 1
      for (int g = 0; g < rows_in(c); g += 4 * U) {
        f32x4_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          v[u] = *reinterpret_cast<const f32x4_t *>(turned + (g + 4 * u + r16) * RS + c16 * 4);
          if constexpr (ADDS) v[u] += r[u];
        }
        if constexpr (ADDS) {  // the next rows, ahead of the stores: a load does not pass a store that may write what it reads
#pragma unroll
          for (int u = 0; u < U; ++u) r[u] = resid(c * 16 + g + 4 * U + 4 * u + r16);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int m = m0 + wm0 + c * 16 + g + 4 * u + r16;
          const bool ok = n_ok && m < a.M;
          if constexpr (EPI == EPI_PARTIAL) {
            if (ok) *reinterpret_cast<f32x4_t *>(ws + (size_t)m * a.N + n) = v[u];
          } else if constexpr (EPI == EPI_RESID_NORM) {
            float ss = ok ? v[u][0] * v[u][0] + v[u][1] * v[u][1] + v[u][2] * v[u][2] + v[u][3] * v[u][3] : 0.f;
            if (ok) {
              // x1 stays in fp32 for the second residual add; the next GEMM reads bf16(x1 * gain)
              *reinterpret_cast<f32x4_t *>(a.C32 + (size_t)m * a.ldc + n) = v[u];
              store_bf16x4(a.C_gain + (size_t)m * a.ldc + n, v[u][0] * gain[0], v[u][1] * gain[1], v[u][2] * gain[2], v[u][3] * gain[3]);
            }
            // the sixteen lanes of the row add up: one partial sum per wavefront column
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) ss += __shfl_xor(ss, o, 64);
            if (c16 == 0 && m < a.M) a.ss_out[(size_t)(tc.tn * WAVES_N + (wave % WAVES_N)) * a.ss_stride + m] = ss;
          } else {
            if (ok) store_bf16x4(a.C + (size_t)m * a.ldc + n, v[u][0], v[u][1], v[u][2], v[u][3]);
          }
        }
      }
    }
  }

  if constexpr (I8) {
    const int n = n0 + wn0 + c16;
    const bool aligned = ((reinterpret_cast<uintptr_t>(a.C) | (uintptr_t)a.ldc * 2) & 7) == 0;
    const int stride = w8_part_stride(a.N);
    int32_t *ws = reinterpret_cast<int32_t *>(a.sk_ws) + (size_t)split * a.M * stride;
    f32x4_t scale = {0.f, 0.f, 0.f, 0.f};
    if constexpr (EPI == EPI_W8) {
#pragma unroll
      for (int e = 0; e < 4; ++e) scale[e] = a.col_scale[min(n + e, a.N - 1)];
    }
    const auto store = [&](auto whole_range) {
#pragma unroll
      for (int c = 0; c < MI; c += CM) {
        turn(c, whole_range);
#pragma unroll 4
        for (int g = 0; g < rows_in(c); g += 4) {
          const int m = m0 + wm0 + c * 16 + g + r16;
          const unsigned char *row = turned + (g + r16) * RS, *from = row + c16 * 4;
          if (m >= a.M || n >= n_lim) continue;
          if constexpr (EPI == EPI_W8) {
            f32x4_t v = *reinterpret_cast<const f32x4_t *>(from) * scale;
            if constexpr (decltype(whole_range)::value) v *= *reinterpret_cast<const float *>(row + BACK);
            store_scaled4(a.C + (size_t)m * a.ldc + n, v, n, n_lim, aligned);
          } else {
            *reinterpret_cast<i32x4_t *>(ws + (size_t)m * stride + n) = *reinterpret_cast<const i32x4_t *>(from);
          }
        }
      }
    };
    // (what few products need takes 2 % of the time of large ones, so it is a path of its own: 2560 x 28672 x 4096 271 against 265 us)
    bool far = a.K >= W8_LONG;
    if constexpr (EPI == EPI_W8) {
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) far |= W8RowScale(row_scale[mi]).back != 1.f;
    }
    if (EPI == EPI_W8 && __builtin_amdgcn_ballot_w64(far) != 0) store(Yes{});
    else store(No{});
  }

  float rstd[MI];
  if constexpr (EPI == EPI_QKV || EPI == EPI_SWIGLU) {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) rstd[mi] = a.rstd[min(m0 + wm0 + mi * 16 + lr, a.M - 1)];
  }

  if constexpr (EPI == EPI_SWIGLU) {
    // the weight tile interleaves 32 gate rows with the matching 32 up rows: blocks 0, 1 are gate
    // features, blocks 2, 3 their up features.  A quarter of the output projection's bytes, straight from the
    // registers (turned round in LDS as well: 1580 rows of the 8B layer 351 -> 357 us)
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) {
      const int m = m0 + wm0 + mi * 16 + lr;
      const float s = rstd[mi];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = n0 + (wn0 >> 1) + h * 16 + 4 * lg;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float g = acc[h][mi][e] * s;
          const float u = acc[2 + h][mi][e] * s;
          v[e] = g / (1.f + __expf(-g)) * u;
        }
        if (m < a.M && n < n_lim) store_bf16x4(a.C + (size_t)m * a.ldc + n, v[0], v[1], v[2], v[3]);
      }
    }
  }

  if constexpr (EPI == EPI_QKV) {
    // the 64 tile columns of a wavefront: features i0 .. i0 + 31 of a head (blocks 0, 1) and i0 + dh/2 .. (blocks 2, 3)
    constexpr int HALF = DH / 2;
    const size_t tile_elems = (size_t)16 * DH;  // one K or V tile of a (page, head)
    const QkvGroup group = qkv_group((n0 + wn0) >> 6, a, DH);
    const int head = group.head, i0 = group.i0;
    const bool is_q = head < a.n_q_heads;
    const bool is_k = !is_q && head < a.n_q_heads + a.n_kv_heads;
    if (head >= a.n_q_heads + 2 * a.n_kv_heads) {
      // a wavefront beyond the last head
    } else if (is_q || is_k) {
      // eight rows per step, eight lanes with four rotation pairs each along a row
      const int r8 = lane >> 3, p8 = 4 * (lane & 7), i = i0 + p8;
      constexpr int U = 2;  // steps at a time; the angles of the next ones and the positions of those behind are under way
      int pos[U], page[U], slot[U], page_n[U] = {}, slot_n[U] = {};
      float s[U], s_n[U];
      f32x4_t cs[U], sn[U];
      auto ask_rows = [&](int row) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int m = min(m0 + wm0 + row + 8 * u + r8, a.M - 1);
          pos[u] = a.row_pos[m];
          s_n[u] = a.rstd[m];
          if (is_k) {
            page_n[u] = a.row_page[m];
            slot_n[u] = a.row_slot[m];
          }
        }
      };
      auto ask_angles = [&]() {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          cs[u] = *reinterpret_cast<const f32x4_t *>(a.rope_cos + (size_t)pos[u] * HALF + i);
          sn[u] = *reinterpret_cast<const f32x4_t *>(a.rope_sin + (size_t)pos[u] * HALF + i);
          s[u] = s_n[u];
          page[u] = page_n[u];
          slot[u] = slot_n[u];
        }
      };
      ask_rows(0);
      ask_angles();
      ask_rows(8 * U);
#pragma unroll
      for (int c = 0; c < MI; c += CM) {
        turn(c, No{});
#pragma unroll 1
        for (int g = 0; g < rows_in(c); g += 8 * U) {
          f32x4_t lo[U], hi[U];
          uint16_t *dst[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const unsigned char *row = turned + (g + 8 * u + r8) * RS;
            const f32x4_t l = *reinterpret_cast<const f32x4_t *>(row + p8 * 4) * s[u];
            const f32x4_t h = *reinterpret_cast<const f32x4_t *>(row + (32 + p8) * 4) * s[u];
            lo[u] = l * cs[u] - h * sn[u];
            hi[u] = h * cs[u] + l * sn[u];
            const int m = m0 + wm0 + c * 16 + g + 8 * u + r8;
            dst[u] = is_q ? a.q_out + (size_t)m * (a.n_q_heads * DH) + head * DH + i
                          : a.kv_pool + (((size_t)page[u] * 2 + 0) * a.n_kv_heads + (head - a.n_q_heads)) * tile_elems +
                                (size_t)slot[u] * DH + i;
          }
          ask_angles();
          ask_rows(c * 16 + g + 16 * U);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (m0 + wm0 + c * 16 + g + 8 * u + r8 >= a.M) continue;
            store_bf16x4(dst[u], lo[u][0], lo[u][1], lo[u][2], lo[u][3]);
            store_bf16x4(dst[u] + HALF, hi[u][0], hi[u][1], hi[u][2], hi[u][3]);
          }
        }
      }
    } else {
      // V^T tiles hold, per feature, the 16 slots of a page side by side, while a lane
      // holds four features of one row: the wavefront turns its block round in LDS
      // (feature-major, FS bytes per feature: the row count padded so that neither the
      // 2-byte writes nor the 8-byte reads below collide on banks)
      constexpr int FS = (WTM + 4) * 2;
      static_assert(64 * FS <= CM * 16 * RS, "the features of a wavefront fit its part of the ring");
#pragma unroll
      for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint16_t *>(turned + (b * 16 + 4 * lg + e) * FS + (mi * 16 + lr) * 2) = f32_to_bf16(acc[b][mi][e] * rstd[mi]);
      // Back out of LDS: lane = 4 * feature + quad reads rows 4 quad .. 4 quad + 3 of a 16-row block for one
      // feature.  Inside a prefill segment these are four adjacent slots of one page, and the 64 lanes then
      // cover 512 contiguous bytes of the page's V^T tile; they go out as one 8-byte store (or two
      // 4-byte ones) where the address allows.  Rows of different sequences, or on either
      // side of a page boundary, take a 2-byte store each.
      __builtin_amdgcn_wave_barrier();
      const int vh = head - a.n_q_heads - a.n_kv_heads;
      const int fl = lane >> 2, rq = lane & 3;
      int pg[4], sl[4], pn[4], ln[4];
      auto ask = [&](int mi, int (&p)[4], int (&l)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = min(m0 + wm0 + mi * 16 + rq * 4 + e, a.M - 1);
          p[e] = a.row_page[m];
          l[e] = a.row_slot[m];
        }
      };
      ask(0, pg, sl);
#pragma unroll 1
      for (int mi = 0; mi < MI; ++mi) {
        const int ml = mi * 16 + rq * 4, mb = m0 + wm0 + ml;
        ask(mi + 1, pn, ln);
        bool run = mb + 3 < a.M;
#pragma unroll
        for (int e = 1; e < 4; ++e) run = run && pg[e] == pg[0] && sl[e] == sl[0] + e;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int ei = (b >> 1) * HALF + i0 + (b & 1) * 16 + fl;
          const u32x2_t v = *reinterpret_cast<const u32x2_t *>(turned + (b * 16 + fl) * FS + ml * 2);
          uint16_t *d0 = a.kv_pool + (((size_t)pg[0] * 2 + 1) * a.n_kv_heads + vh) * tile_elems + ei * 16 + sl[0];
          if (run && (reinterpret_cast<uintptr_t>(d0) & 7) == 0) {
            *reinterpret_cast<u32x2_t *>(d0) = v;
          } else if (run && (reinterpret_cast<uintptr_t>(d0) & 3) == 0) {
            reinterpret_cast<uint32_t *>(d0)[0] = v.x;
            reinterpret_cast<uint32_t *>(d0)[1] = v.y;
          } else {
            const uint16_t ve[4] = {(uint16_t)(v.x & 0xFFFFu), (uint16_t)(v.x >> 16), (uint16_t)(v.y & 0xFFFFu), (uint16_t)(v.y >> 16)};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (mb + e < a.M) a.kv_pool[(((size_t)pg[e] * 2 + 1) * a.n_kv_heads + vh) * tile_elems + ei * 16 + sl[e]] = ve[e];
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          pg[e] = pn[e];
          sl[e] = ln[e];
        }
      }
    }
  }
}

// Few rows: a product is the stream of its weights.  One workgroup of eight wavefronts per CU takes items, 16 NI weight
// rows by 16 MI activation rows, in turn and cuts K among its wavefronts, k-tiles of 64 dealt round (together they walk
// 1 KB of every weight row at a time).  A wavefront has a ring of S k-tiles of its own in LDS, both panels, filled by its
// own requests and read by nobody else: no barrier while it streams, and the ring runs on across items.  At the end of
// an item the eight partial sums of a value meet in LDS, one wavefront adds them in the order of the wavefronts and runs
// the epilogue while the others stream on: no partial products in memory, no second kernel.
// The 16 rows of a weight block are two units of eight where the epilogue pairs rows: gate and up rows, or the lower and
// upper half of a head's rotation pairs.
// Measured, cold weights, second kernels included, 8B layer at 8 rows: QKV 17.1 -> 12.9 us, output projection
// 14.9 -> 9.1, gate/up 53.8 -> 39.5 (5.9 TB/s), down 27.9 -> 22.9; K = N = 256 7.7 -> 3.4.  Not depth but the order of
// the requests makes the difference: 128x128 tiles with as many bytes in flight take 54 us for gate/up, every workgroup
// at the same column of 128 rows 8 KB apart.  Loads straight into registers (a lane's operand: 16 bytes of a row
// 8 KB from its neighbour's) reach 16 bytes per clock and CU: 56 us.
constexpr int ROWS_MAX_M = 256;
// blocks of 16 weight rows of a product (of pairs of eight where the epilogue pairs rows)
constexpr long rows_blocks(int n, int epi) { return epi == EPI_QKV ? n / 16 : epi == EPI_SWIGLU ? n / 8 : (n + 15) / 16; }
template <int MI, int NI>  // blocks of 16 activation rows, blocks of 16 weight rows
struct RowsKernel {
  static constexpr int L = 2 * (MI + NI), STAGE = L * 1024;  // loads and bytes of a k-tile
  static constexpr int RED = 8 * MI * 1024, META = ROWS_MAX_M * 16;
  static constexpr int S = (160 * 1024 - RED - META) / 8 / STAGE;
  static constexpr int LDS = 8 * S * STAGE + RED + META;
};

// waits until at most J * L vector-memory operations are outstanding, for the J that equals `left`
template <int L, int... J>
__device__ __forceinline__ void wait_for_all_but(int left, std::integer_sequence<int, J...>) {
  ((left == J ? __builtin_amdgcn_s_waitcnt(waitcnt_imm(J * L, false)) : (void)0), ...);
}

template <int MI, int NI, bool I8 = false>
__global__ __launch_bounds__(512) void gemm_rows_kernel(const GemmArgs a, const int epi, const int dh, const int tiles_m, const int n_items) {
  typedef RowsKernel<MI, NI> R;
  typedef GemmAcc<I8> Acc;
  constexpr int S = R::S, L = R::L;
  static_assert(S >= 2 && (S - 1) * L < 64, "look-ahead, and the vmcnt field");
  extern __shared__ __align__(16) unsigned char smem[];
  Acc *red = reinterpret_cast<Acc *>(smem + 8 * S * R::STAGE);  // [8][MI][64]
  float *meta_rs = reinterpret_cast<float *>(smem + 8 * S * R::STAGE + R::RED);  // [ROWS_MAX_M] per row: norm factor, position, page, slot
  int *meta_pos = reinterpret_cast<int *>(meta_rs + ROWS_MAX_M), *meta_page = meta_pos + ROWS_MAX_M, *meta_slot = meta_page + ROWS_MAX_M;
  const bool paired = !I8 && (epi == EPI_QKV || epi == EPI_SWIGLU);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int lr = lane & 15, lg = lane >> 4;
  unsigned char *ring = smem + wave * S * R::STAGE;

  // requests: 8 lanes per row of 128 bytes, chunks swizzled as in gemm_tile
  const int g_row = lane >> 3, g_slot = lane & 7;
  const int chunk[2] = {g_slot ^ (g_row >> 1), g_slot ^ ((g_row + 8) >> 1)};  // rows g_row and g_row + 8 of a block
  uint32_t off_x[2 * MI], off_w[2 * NI];
  const int per_head = dh / 16;
  auto first_row = [&](int blk) { return epi == EPI_QKV ? blk / per_head * dh + blk % per_head * 8 : paired ? blk * 8 : blk * 16; };
  const int second = epi == EPI_QKV ? dh / 2 : a.N;  // from a paired unit's first eight rows to its second
  // items: the row tiles of a weight block one after the other
  auto set_item = [&](int item) {
    const int blk = item / tiles_m, m0 = item % tiles_m * 16 * MI;
#pragma unroll
    for (int i = 0; i < 2 * MI; ++i) off_x[i] = (uint32_t)(((size_t)min(m0 + i * 8 + g_row, a.M - 1) * a.lda + chunk[i & 1] * 8) * 2);
#pragma unroll
    for (int i = 0; i < 2 * NI; ++i) {
      // rows beyond the last repeat it (a unit of eight is whole or beyond it altogether)
      const int row = min(first_row(blk * NI + i / 2) + (paired ? 0 : 8 * (i & 1)) + g_row, a.N - 1 - (epi == EPI_QKV ? second : 0)) +
                      (paired ? (i & 1) * second : 0);
      off_w[i] = (uint32_t)(((size_t)row * a.ldb + chunk[i & 1] * 8) * 2);
    }
  };
  const int nk = (a.K + BK - 1) / BK;
  const int n = nk > wave ? (nk - wave + 7) / 8 : 0;  // k-tiles of this wavefront per item
  const int mine = (n_items - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
  const int total = n * mine;                       // k-tiles it will see
  int i_item = (int)blockIdx.x, i_k = 0, i_slot = 0, issued = 0;
  auto dma = [](const void *p, unsigned char *lds) {
    __builtin_amdgcn_global_load_lds(p, (__attribute__((address_space(3))) void *)lds, 16, 0, 0);
  };
  auto issue = [&]() __attribute__((always_inline)) {
    const int kt = wave + 8 * i_k;
    const unsigned char *bw = reinterpret_cast<const unsigned char *>(a.B) + (size_t)kt * 128;
    const unsigned char *bx = reinterpret_cast<const unsigned char *>(a.A) + (size_t)kt * 128;
    unsigned char *dst = ring + i_slot * R::STAGE;
    const int beyond = (kt + 1) * BK > a.K ? a.K - kt * BK : BK;  // first element of the k-tile that lies beyond K
    if (beyond == BK) {
#pragma unroll
      for (int i = 0; i < 2 * NI; ++i) dma(bw + off_w[i], dst + i * 1024);
#pragma unroll
      for (int i = 0; i < 2 * MI; ++i) dma(bx + off_x[i], dst + (2 * NI + i) * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < 2 * NI; ++i) dma(chunk[i & 1] * 8 >= beyond ? (const void *)g_gemm_zero_chunk : bw + off_w[i], dst + i * 1024);
#pragma unroll
      for (int i = 0; i < 2 * MI; ++i) dma(chunk[i & 1] * 8 >= beyond ? (const void *)g_gemm_zero_chunk : bx + off_x[i], dst + (2 * NI + i) * 1024);
    }
    ++issued;
    i_slot = i_slot + 1 == S ? 0 : i_slot + 1;
    if (++i_k == n) {
      i_k = 0;
      i_item += (int)gridDim.x;
      if (i_item < n_items) set_item(i_item);
    }
  };
  if (total > 0) set_item(i_item);
  for (int s = 0; s < S && issued < total; ++s) issue();

  // what the epilogue asks per row
  const int rows = tiles_m * 16 * MI;  // at most ROWS_MAX_M
  if (t < rows) {
    const int m = min(t, a.M - 1);
    if (epi == EPI_QKV) {
      meta_pos[t] = a.row_pos[m];
      meta_page[t] = a.row_page[m];
      meta_slot[t] = a.row_slot[m];
    }
    if (paired && !a.ss_in_parts) meta_rs[t] = a.rstd[m];
  }
  if (paired && a.ss_in_parts) {
    // the second norm's factor from the output projection's partial row sums: 512 / rows threads per row
    const int per_row = 512 / rows, r = t % rows, q = t / rows;
    float s = 0.f;
    if (q < per_row) {
#pragma unroll 8
      for (int p = q; p < a.ss_in_parts; p += per_row) s += a.ss_in[(size_t)p * a.ss_stride + min(r, a.M - 1)];
    }
    float *part = reinterpret_cast<float *>(red);
    part[t] = s;
    __syncthreads();
    if (t < rows) {
      s = 0.f;
      for (int i = 0; i < per_row; ++i) s += part[t + rows * i];
      meta_rs[t] = rsqrtf(s / (float)a.K + a.rstd_eps);
    }
    __syncthreads();
  }

  const int sw = (lr >> 1) & 7;
  int slot = 0, left = total, turn = 0;
  for (int item = (int)blockIdx.x; item < n_items; item += (int)gridDim.x, ++turn) {
    const int blk = item / tiles_m, m0 = item % tiles_m * 16 * MI;
    Acc acc[NI][MI];
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) acc[ni][mi] = Acc{0, 0, 0, 0};
    for (int k = 0; k < n; ++k) {
      --left;  // k-tiles behind this one
      if (left >= S - 1) {
        __builtin_amdgcn_s_waitcnt(waitcnt_imm((S - 1) * L, false));
      } else {
        wait_for_all_but<L>(left, std::make_integer_sequence<int, S - 1>{});
      }
      const unsigned char *st = ring + slot * R::STAGE;
      bf16x8_t w[2][NI], x[2][MI];
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int ch = ((ks * 4 + lg) ^ sw) << 4;
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) w[ks][ni] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(st + ni * 2048 + lr * 128 + ch));
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) x[ks][mi] = as_bf16x8(*reinterpret_cast<const u32x4_t *>(st + (NI + mi) * 2048 + lr * 128 + ch));
      }
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));  // the slot may be filled again
#pragma unroll
      for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
#pragma unroll
          for (int mi = 0; mi < MI; ++mi) gemm_mfma(acc[ni][mi], w[ks][ni], x[ks][mi]);
      if (left >= S) issue();
      slot = slot + 1 == S ? 0 : slot + 1;
    }
    // the partial sums of 16 weight rows at a time meet; the requests in flight are left alone
#pragma unroll
    for (int ni = 0; ni < NI; ++ni) {
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));
      __builtin_amdgcn_s_barrier();  // nobody reads the sums before these any more
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) red[(wave * MI + mi) * 64 + lane] = acc[ni][mi];
      __builtin_amdgcn_s_waitcnt(waitcnt_imm(63, true));
      __builtin_amdgcn_s_barrier();
#pragma unroll
      for (int mi = 0; mi < MI; ++mi) {
        if (wave != ((turn * NI + ni) * MI + mi) % 8) continue;
        auto total_of = [&](int l) {
          Acc s = red[mi * 64 + l];
#pragma unroll
          for (int v = 1; v < 8; ++v) s += red[(v * MI + mi) * 64 + l];
          return s;
        };
        const int ml = m0 + 16 * mi + lr;  // (at most ROWS_MAX_M - 1)
        const bool ok = ml < a.M;
        if constexpr (I8) {
          const int n0 = (blk * NI + ni) * 16 + 4 * lg;
          if (!ok || n0 >= a.N) continue;
          const W8RowScale by(a.row_scale[ml]);
          f32x4_t v = w8_sums(total_of(lane)) * by.scale;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] *= a.col_scale[min(n0 + e, a.N - 1)];
          store_scaled4(a.C + (size_t)ml * a.ldc + n0, v * by.back, n0, a.N, ((reinterpret_cast<uintptr_t>(a.C) | (uintptr_t)a.ldc * 2) & 7) == 0);
        } else if (paired) {
          const int u = first_row(blk * NI + ni) + 4 * (lg & 1);  // first of this lane's four rows of the lower unit
          const f32x4_t lo = total_of(lane & 31) * meta_rs[ml], hi = total_of((lane & 31) + 32) * meta_rs[ml];
          if (!ok || lg > 1 || u >= a.N) continue;
          if (epi == EPI_SWIGLU) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = lo[e] / (1.f + __expf(-lo[e])) * hi[e];
            store_bf16x4(a.C + (size_t)ml * a.ldc + u, v[0], v[1], v[2], v[3]);
          } else {
            const int head = u / dh, i0 = u % dh, half = dh / 2;
            const size_t tile_elems = (size_t)16 * dh, page = meta_page[ml];
            const int slot_in = meta_slot[ml];
            if (head < a.n_q_heads + a.n_kv_heads) {
              const size_t at = (size_t)meta_pos[ml] * half + i0;
              const f32x4_t cs = *reinterpret_cast<const f32x4_t *>(a.rope_cos + at), sn = *reinterpret_cast<const f32x4_t *>(a.rope_sin + at);
              const f32x4_t l = lo * cs - hi * sn, h = hi * cs + lo * sn;
              uint16_t *dst = head < a.n_q_heads
                                  ? a.q_out + (size_t)ml * (a.n_q_heads * dh) + head * dh
                                  : a.kv_pool + ((page * 2 + 0) * a.n_kv_heads + (head - a.n_q_heads)) * tile_elems + (size_t)slot_in * dh;
              store_bf16x4(dst + i0, l[0], l[1], l[2], l[3]);
              store_bf16x4(dst + half + i0, h[0], h[1], h[2], h[3]);
            } else {
              uint16_t *dst = a.kv_pool + ((page * 2 + 1) * a.n_kv_heads + (head - a.n_q_heads - a.n_kv_heads)) * tile_elems + slot_in;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                dst[(i0 + e) * 16] = f32_to_bf16(lo[e]);
                dst[(i0 + half + e) * 16] = f32_to_bf16(hi[e]);
              }
            }
          }
        } else {
          f32x4_t v = total_of(lane);
          const int n0 = (blk * NI + ni) * 16 + 4 * lg;
          const bool in = ok && n0 < a.N;
          const size_t at = (size_t)ml * a.ldr + n0;
          if (in && epi == EPI_RESID && a.resid32) {
            v += *reinterpret_cast<const f32x4_t *>(a.resid32 + at);
          } else if (in && epi != EPI_PLAIN) {
            const u32x2_t rr = *reinterpret_cast<const u32x2_t *>(a.resid + at);
            v += f32x4_t{__uint_as_float(rr.x << 16), __uint_as_float(rr.x & 0xFFFF0000u), __uint_as_float(rr.y << 16), __uint_as_float(rr.y & 0xFFFF0000u)};
          }
          if (epi == EPI_RESID_NORM) {
            float ss = 0.f;
            if (in) {
              const u32x2_t gg = *reinterpret_cast<const u32x2_t *>(a.gain + n0);
              ss = v[0] * v[0] + v[1] * v[1] + v[2] * v[2] + v[3] * v[3];
              *reinterpret_cast<f32x4_t *>(a.C32 + (size_t)ml * a.ldc + n0) = v;
              store_bf16x4(a.C_gain + (size_t)ml * a.ldc + n0, v[0] * __uint_as_float(gg.x << 16), v[1] * __uint_as_float(gg.x & 0xFFFF0000u),
                           v[2] * __uint_as_float(gg.y << 16), v[3] * __uint_as_float(gg.y & 0xFFFF0000u));
            }
            ss += __shfl_xor(ss, 16, 64);
            ss += __shfl_xor(ss, 32, 64);
            if (lg == 0 && in) a.ss_out[(size_t)(blk * NI + ni) * a.ss_stride + ml] = ss;
          } else if (in) {
            store_bf16x4(a.C + (size_t)ml * a.ldc + n0, v[0], v[1], v[2], v[3]);
          }
        }
    }
    }
  }
}

}  // namespace
}  // namespace bs

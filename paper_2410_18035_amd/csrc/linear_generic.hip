// Any-shape, any-dtype routed LoRA linear (paper Eq. 1 with the layer-level gate of Sec. 3.3): fp32 tensors, and bf16 ones
// of widths or alignments that the bf16 matrix-core kernels do not take.  All arithmetic is fp32, on the fp32 matrix
// instructions (157 TFLOP/s on the chip, twice the rate of vector FMA, each product and sum rounded as there).
//
// Operands are taken four consecutive k per lane (any element alignment; the row's last k one by one): instruction e of
// four multiplies element e of both sides, so the k of a block of 8 or 16 are taken in another order than memory's, the
// same one on both sides.  All sums run in a fixed order.
#include "common.h"

namespace milora {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4_a2 __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4_a4*>(p); }
__device__ __forceinline__ f32x4 load4(const bf16_t* p) {
  const u16x4_a2 v = *reinterpret_cast<const u16x4_a2*>(p);
  return f32x4{bf16_to_f32(v[0]), bf16_to_f32(v[1]), bf16_to_f32(v[2]), bf16_to_f32(v[3])};
}
// Elements k .. k + 3 of a row of K, zero past its end.
template <typename T>
__device__ __forceinline__ f32x4 load4_end(const T* row, int k, int K) {
  f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
  if (k + 4 <= K) v = load4(row + k);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k + e < K) v[e] = Elem<T>::load(row, k + e);
  return v;
}
// Columns of one launch: a grid has to stay below 2^32 threads (512 for 16 columns in the few-row kernel).
constexpr int kLaunchCols = 1 << 26;

__device__ __forceinline__ int pow2_above(int r) {
  int p = 1;
  while (p < r) p <<= 1;
  return p;
}

// ---- LoRA shrink: t[m][c] = sum_k X[m][k] * A[k][c], c < r, one workgroup per (row, site) -------------------------
// Threads are laid out with the rank index fastest (coalesced reads of A's rows), eight rows of A per thread on their
// way; the k-lanes are summed through LDS in a fixed order.  Bound by the latency of those loads: 512 threads instead of
// 256 and eight loads in flight instead of one.
constexpr int kShrinkT = 512;
template <typename T>
__global__ void __launch_bounds__(kShrinkT) shrink_rows_kernel(const T* __restrict__ X, int64_t ldx, int64_t M, int d1,
                                                               const int32_t* __restrict__ row_to_req, AdapterView ad,
                                                               int site0, const int32_t* __restrict__ tenant_id,
                                                               const uint8_t* __restrict__ route, int B,
                                                               float* __restrict__ t) {
  __shared__ float red[kShrinkT];
  const int64_t m = blockIdx.x;
  const int site = site0 + blockIdx.y;
  const int64_t req = row_to_req ? (int64_t)row_to_req[m] : m;
  int tenant = 0;
  const int r = (req >= 0 && req < B) ? routed_rank(ad, tenant_id, route, (int)req, B, site, &tenant) : 0;
  if (r == 0) return;
  const T* A = (const T*)ad.A[tenant * MILORA_NUM_SITES + site];
  const int rpad = pow2_above(r);
  const int c = threadIdx.x & (rpad - 1), krow = threadIdx.x / rpad, rpp = kShrinkT / rpad;
  const T* x = X + (size_t)m * ldx;
  float acc = 0.f;
  if (c < r) {
    int k = krow;
    for (; k + 7 * rpp < d1; k += 8 * rpp) {
      float xv[8], av[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        xv[u] = Elem<T>::load(x, k + u * rpp);
        av[u] = Elem<T>::load(A, (size_t)(k + u * rpp) * r + c);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) acc += xv[u] * av[u];
    }
    for (; k < d1; k += rpp) acc += Elem<T>::load(x, k) * Elem<T>::load(A, (size_t)k * r + c);
  }
  red[threadIdx.x] = acc;
  __syncthreads();
  if (krow == 0 && c < r) {
    float s = 0.f;
    for (int j = 0; j < rpp; ++j) s += red[j * rpad + c];
    t[((size_t)blockIdx.y * M + m) * ad.r_max + c] = s;
  }
}

// ---- few rows: up to 16 --------------------------------------------------------------------------------------------
// A workgroup takes 16 columns of one linear (gate and up: of both) and the whole reduction, dealt to its waves in
// blocks of 16 k that go straight from global memory into matrix operands; the waves' sums meet in LDS.  Where rows, ranks
// and widths are small the shrinks are formed here too (FUSED, fuse_shrink), each wave over its share of k and one row after
// the other, again in every workgroup; else they come from shrink_rows_kernel.
// The layer's glue is part of the store: a decode step of a layer is four launches instead of eighteen.
// Bound: launches (about 2.4 us each with nothing in them), and the code a launch runs through, whose time goes with its
// bytes (4.6 KB 4.8 us, 7.7 KB 8.0 us): what a call does not need is compiled out, the shrinks of two sites are one loop, and
// four waves run through it where that is enough (few_waves: d = 256 22.3 -> 19.6 us).  A decode step of 4 rows through the 256 x 688 fp32 layer, rank 8: 284 us with eighteen launches,
// 22.3 us with four of eight waves and both expands in them, 19.6 us so.  Tried: base and adapter pointers asked for ahead of the
// look-ups (fewer dependent loads, more code: 26.9 against 24.3 us), 32-bit offsets with a path for whole trips (41.1 against 35.6 us at
// 16 rows, d = 504).
constexpr int kFewBlocks = 4;  // blocks of 16 k per wave on their way
constexpr int kFewNarrow = 256;  // no reduction longer than this on four waves

template <typename T>
__device__ __forceinline__ float round_to(float v) {
  T q;
  Elem<T>::store(&q, 0, v);
  return Elem<T>::load(&q, 0);
}

template <typename T, int MODE, int kFewW, bool FUSED>
__global__ void __launch_bounds__(kFewW * 64, 4) few_rows_kernel(const FewArgs g) {
  constexpr bool kPair = MODE == kFewGateUp || MODE == kFewGated;
  constexpr int NW = kPair ? 2 : 1;
  __shared__ float red[NW][kFewW][16][17];
  __shared__ float tpart[FUSED ? NW : 1][FUSED ? kFewW : 1][16][kFuseRank];
  __shared__ float ts[FUSED ? NW : 1][16][kFuseRank];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s0 = kPair ? 0 : blockIdx.y, n0 = g.col0 + blockIdx.x * 16;
  const int d1 = g.d1;

  // rank and tenant of row li at the workgroup's site, of its two sites in lanes 0 .. 15 and 16 .. 31 (route byte and tenant id are
  // asked for together)
  int rank = 0, ten = 0;
  {
    const int64_t req = li < g.M ? (g.row_to_req ? (int64_t)g.row_to_req[li] : li) : -1;
    const bool in = req >= 0 && req < g.B;
    const uint8_t rt = in ? g.route[req] : (uint8_t)MILORA_ROUTE_NONE;
    const int tn = in ? g.tenant_id[req] : -1;
    const bool known = tn >= 0 && tn < g.ad.n_tenants;
    const int r = known ? g.ad.rank[tn] : 0;
    if (known && lq < NW && route_has(rt, g.site[s0] + lq) && r >= 1 && r <= g.ad.r_max) {  // (sites of a workgroup are consecutive)
      rank = r;
      ten = tn;
    }
  }

  // ---- base linear ----
  const T* const xr = (const T*)g.X + (size_t)(li < g.M ? li : g.M - 1) * g.ldx;  // (rows past the end: results dropped)
  const int col = n0 + li < g.d2 ? n0 + li : g.d2 - 1;
  const T* wr[NW];
  f32x4 acc[NW];
#pragma unroll
  for (int j = 0; j < NW; ++j) {
    wr[j] = (const T*)g.W[s0 + j] + (size_t)col * d1;
    acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int full = d1 >> 4;
  for (int b0 = w; b0 < full; b0 += kFewW * kFewBlocks) {
    f32x4 xv[kFewBlocks], wv[NW][kFewBlocks];
#pragma unroll
    for (int u = 0; u < kFewBlocks; ++u) {
      const int b = b0 + u * kFewW < full ? b0 + u * kFewW : full - 1;
      xv[u] = load4(xr + b * 16 + lq * 4);
#pragma unroll
      for (int j = 0; j < NW; ++j) wv[j][u] = load4(wr[j] + b * 16 + lq * 4);
    }
#pragma unroll
    for (int u = 0; u < kFewBlocks; ++u)
      if (b0 + u * kFewW < full)
#pragma unroll
        for (int j = 0; j < NW; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[j][u][e], xv[u][e], acc[j], 0, 0, 0);
  }
  if (__builtin_expect(full * 16 < d1 && w == full % kFewW, 0)) {
    const f32x4 x = load4_end(xr, full * 16 + lq * 4, d1);
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const f32x4 v = load4_end(wr[j], full * 16 + lq * 4, d1);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e], x[e], acc[j], 0, 0, 0);
    }
  }
  // (lane: row li, columns 4 lq .. + 3 of the 16)
#pragma unroll
  for (int j = 0; j < NW; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[j][w][li][lq * 4 + e] = acc[j][e];

  // ---- shrinks of the routed rows over this wave's share of k ----
  if constexpr (FUSED) {
    const int share = (d1 + kFewW - 1) / kFewW, k0 = w * share, k1 = k0 + share < d1 ? k0 + share : d1;
    for (unsigned long long left = __ballot(rank > 0); left; left &= left - 1) {
      const int at = __builtin_ctzll(left), m = at & 15, j = NW > 1 ? at >> 4 : 0;
      const int r = __builtin_amdgcn_readlane(rank, at), tn = __builtin_amdgcn_readlane(ten, at);
      const T* const A = (const T*)g.ad.A[tn * MILORA_NUM_SITES + g.site[s0] + j];
      const T* const x = (const T*)g.X + (size_t)m * g.ldx;
      const int rpad = pow2_above(r), c = lane & (rpad - 1), kpl = 64 / rpad;
      float sum = 0.f;
      for (int k = k0 + lane / rpad; __any(k < k1); k += 8 * kpl) {
        float xv[8], av[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int kk = k + u * kpl < k1 ? k + u * kpl : d1 - 1;
          xv[u] = Elem<T>::load(x, kk);
          av[u] = Elem<T>::load(A, (size_t)kk * r + (c < r ? c : 0));
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += k + u * kpl < k1 ? xv[u] * av[u] : 0.f;
      }
      for (int off = rpad; off < 64; off <<= 1) sum += __shfl_xor(sum, off, 64);
      if (lane < r) tpart[j][w][m][lane] = sum;
    }
  }
  __syncthreads();
  const int m = tid >> 4, n = n0 + (tid & 15);  // threads 0 .. 255: one output each; their lanes' rows are 4 (tid / 64) ..
  int rm[NW], tm[NW];
#pragma unroll
  for (int j = 0; j < NW; ++j) {
    rm[j] = __shfl(rank, (m & 15) + 16 * j, 64);
    tm[j] = __shfl(ten, (m & 15) + 16 * j, 64);
  }
  if (FUSED && tid < 256) {
    const int c = tid & 15;
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      float s = 0.f;
      if (c < rm[j])
        for (int k = 0; k < kFewW; ++k) s += tpart[j][k][m][c];
      ts[j][m][c] = s;  // (read by the same sixteen lanes)
    }
  }
  __syncthreads();
  if (tid >= 256 || m >= g.M || n >= g.d2) return;

  // ---- bias, LoRA expand, glue, one rounding ----
  float val[NW];
#pragma unroll
  for (int j = 0; j < NW; ++j) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kFewW; ++k) v += red[j][k][m][tid & 15];
    if (g.bias) v += Elem<T>::load((const T*)g.bias, n);
    if (rm[j] > 0) {
      const T* const Bm = (const T*)g.ad.B[tm[j] * MILORA_NUM_SITES + g.site[s0 + j]] + n;
      const float* const tg = FUSED ? nullptr : g.t + ((size_t)(s0 + j) * g.M + m) * g.ad.r_max;
      float delta = 0.f;
      for (int c0 = 0; c0 < rm[j]; c0 += 8) {
        float bv[8], tv[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int c = c0 + u < rm[j] ? c0 + u : rm[j] - 1;
          bv[u] = Elem<T>::load(Bm, (size_t)c * g.d2);
          tv[u] = FUSED ? ts[j][m][c & (kFuseRank - 1)] : tg[c];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) delta += c0 + u < rm[j] ? tv[u] * bv[u] : 0.f;
      }
      v += delta;
    }
    val[j] = v;
  }
  if constexpr (MODE == kFewPlain) {
    Elem<T>::store((T*)g.Y[s0], (size_t)m * g.ldy + n, val[0]);
  } else if constexpr (MODE == kFewResid) {
    const size_t i = (size_t)m * g.d2 + n;
    const float h = Elem<T>::load((const T*)g.x_res, i) + round_to<T>(val[0]);
    g.h[i] = h;
    if (g.Y[0]) Elem<T>::store((T*)g.Y[0], i, h);
  } else if constexpr (MODE == kFewGateUp) {
    Elem<T>::store((T*)g.Y[0], (size_t)m * g.ldy + n, silu(round_to<T>(val[0])) * round_to<T>(val[1]));
  } else if constexpr (MODE == kFewGated) {
    const size_t i = (size_t)m * g.d2 + n;
    if (g.gate_out) g.gate_out[i] = val[0];
    if (g.up_out) g.up_out[i] = val[1];
    Elem<T>::store((T*)g.Y[0], (size_t)m * g.ldy + n, silu(val[0]) * val[1]);
  } else {
    const size_t i = (size_t)m * g.d2 + n;
    Elem<T>::store((T*)g.Y[0], i, g.h[i] + round_to<T>(val[0]));
  }
}

// ---- more rows ------------------------------------------------------------------------------------------------------
// A workgroup of eight waves computes a BM x BN tile: KQ groups of waves share a stage's k, the waves of a group the tile,
// 32 x 32 each (v_mfma_f32_32x32x2_f32).  Stages go through registers (four on their way) into one of two LDS buffers.
// WIDE (d1 >= 4): every load is four elements without a branch, a row's end read from its last four and shifted when it
// is stored (a branch around the loads makes the compiler wait for all of them at each store: 28.9 us a call of 300 rows on
// 1000 x 2730 without LoRA rows against 27.5 us).
// Bound: the matrix instructions (13.7 us of that call) and the chain of look-ups, t and W^B behind them (10 us where rows
// carry a LoRA term).  Seven fp32 linears of 300 rows, 1000 x 2730: 1757 us with vector FMA out of single-buffered tiles,
// 190 us here.  64 x 64 tiles where they are at least half the compute units, 32 x 32 with the reduction over eight waves
// below (300 rows on 1000 x 1000: 17.6 us).
template <int BM_, int BN_, int KW_>
struct GenCfg {
  static constexpr int BM = BM_, BN = BN_, KW = KW_;                 // KW: k of a stage per wave
  static constexpr int WM = BM / 32, WN = BN / 32, KQ = 8 / (WM * WN);
  static constexpr int SK = KQ * KW, Ld = SK + 4;                    // rows padded: 16 rows at one k hit all banks
  static constexpr int T = 512;
  static constexpr int Items = (BM + BN) * (SK / 4) / T;             // 16-byte pieces of a stage per thread
  static constexpr int BufFloats = (BM + BN) * Ld;
  static constexpr int LdR = BN + 4;
  static constexpr int Outs = BM * BN / T;                           // outputs per thread
  static constexpr int TsOff = KQ * BM * LdR;                        // after the sums: t of the rows (of two sites), 32 ranks at a time
  static constexpr int LdsBytes = (2 * BufFloats > TsOff + 2 * BM * 32 ? 2 * BufFloats : TsOff + 2 * BM * 32) * 4;
  static_assert((BM + BN) * (SK / 4) % T == 0 && BM * BN % T == 0 && KW % 8 == 0 && 2 * LdsBytes <= 158 * 1024, "tile shape");
};
typedef GenCfg<32, 32, 16> GenSmall;
typedef GenCfg<64, 64, 32> GenLarge;
constexpr int kGenLargeTiles = 128;
constexpr int kGenGroupM = 8;  // row tiles of a column tile before the next one

// GATED: the columns of a tile are as many of the gate (W, t) and then of the up projection (W2, t of the next site): Y = silu(g) u, with g
// and u in fp32, which go to gate_out and up_out, if given.
template <typename T, class C, bool WIDE, bool GATED>
__global__ void __launch_bounds__(C::T, 4) linear_tile_kernel(const T* __restrict__ X, int64_t M, int d1, int d2, int col0,
                                                           const int32_t* __restrict__ row_to_req, const T* __restrict__ W,
                                                           const T* __restrict__ W2, const T* __restrict__ bias, AdapterView ad, int site,
                                                           const int32_t* __restrict__ tenant_id,
                                                           const uint8_t* __restrict__ route, int B,
                                                           const float* __restrict__ t, int64_t t_site, T* __restrict__ Y,
                                                           float* __restrict__ gate_out, float* __restrict__ up_out, int tiles_m, int tiles_n) {
  constexpr int kSites = GATED ? 2 : 1, kOutN = C::BN / kSites;
  extern __shared__ __attribute__((aligned(16))) float buf[];
  __shared__ int s_rank[kSites][C::BM], s_ten[kSites][C::BM], s_most[kSites];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, lh = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q = w / (C::WM * C::WN), wm = w % (C::WM * C::WN) % C::WM, wn = w % (C::WM * C::WN) / C::WM;
  // workgroup -> tile: ids go round-robin over the 8 XCDs; each XCD takes a contiguous run of an order that walks kGenGroupM row tiles of one column
  // tile before the next column tile, so that its L2 serves the re-reads of W (gated block, 300 rows of 1000 x 2730, columns first: 52 us without
  // LoRA rows).  The small tiles of a linear, a turn or so of them, go columns first: rows of a high rank then do not meet on one compute unit (300
  // rows of 1000 x 1000, a quarter of them of rank 64: 26 us a call, in the other order 32).
  const int total = tiles_m * tiles_n, per = (total + 7) >> 3;
  int row_tile, col_tile;
  if constexpr (GATED || C::Outs > 2) {
    const int id = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || id >= total) return;
    const int first = id / (kGenGroupM * tiles_n) * kGenGroupM, in_group = id % (kGenGroupM * tiles_n);
    const int gsz = tiles_m - first < kGenGroupM ? tiles_m - first : kGenGroupM;
    row_tile = first + in_group % gsz;
    col_tile = in_group / gsz;
  } else {
    row_tile = (int)blockIdx.x / tiles_n;
    col_tile = (int)blockIdx.x % tiles_n;
    if (row_tile >= tiles_m) return;
  }
  const int64_t m0 = (int64_t)row_tile * C::BM;
  const int n0 = col0 + col_tile * kOutN;

  const T* src[C::Items];
  const int kq = tid % (C::SK / 4) * 4;
  int dst[C::Items];
#pragma unroll
  for (int i = 0; i < C::Items; ++i) {
    const int row = tid / (C::SK / 4) + i * (C::T / (C::SK / 4));
    if (row < C::BM) {
      const int64_t m = m0 + row < M ? m0 + row : M - 1;  // past the edge: the last row again, its results are dropped
      src[i] = X + (size_t)m * d1;
    } else {
      const int c = row - C::BM, n = n0 + c % kOutN < d2 ? n0 + c % kOutN : d2 - 1;
      src[i] = (GATED && c >= kOutN ? W2 : W) + (size_t)n * d1;
    }
    dst[i] = row * C::Ld + kq;
  }
  const int stages = (d1 + C::SK - 1) / C::SK;
  constexpr int kSets = 4;
  f32x4 r[kSets][C::Items];
  auto load = [&](int st, f32x4 (&v)[C::Items]) __attribute__((always_inline)) {
    const int k = (st < stages ? st : stages - 1) * C::SK + kq;  // past the end: the last stage again, never stored
#pragma unroll
    for (int i = 0; i < C::Items; ++i) v[i] = WIDE ? load4(src[i] + (k < d1 - 4 ? k : d1 - 4)) : load4_end(src[i], k, d1);
    __builtin_amdgcn_sched_barrier(0);  // the sets in their order: the oldest can then be waited for alone
  };
  auto store = [&](int st, f32x4 (&r)[C::Items]) __attribute__((always_inline)) {
    const int shift = st * C::SK + kq - (d1 - 4);  // k by which a load past d1 - 4 was moved back
    if (WIDE && (st + 1) * C::SK > d1)
#pragma unroll
      for (int i = 0; i < C::Items; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = shift <= 0 ? r[i][e] : 0.f;
#pragma unroll
          for (int h = 1; e + h < 4; ++h) v = shift == h ? r[i][e + h] : v;
          r[i][e] = v;
        }
#pragma unroll
    for (int i = 0; i < C::Items; ++i) *reinterpret_cast<f32x4*>(buf + (st & 1) * C::BufFloats + dst[i]) = r[i];
  };
  f32x16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  const int xo = (wm * 32 + l32) * C::Ld + q * C::KW + lh * 4, wo = (C::BM + wn * 32 + l32) * C::Ld + q * C::KW + lh * 4;
  auto compute = [&](int b) __attribute__((always_inline)) {
    const float* const s = buf + b * C::BufFloats;
#pragma unroll
    for (int k = 0; k < C::KW; k += 8) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(s + xo + k), v = *reinterpret_cast<const f32x4*>(s + wo + k);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], x[e], acc, 0, 0, 0);
    }
  };
#pragma unroll
  for (int j = 0; j < kSets; ++j) load(j, r[j]);
  if (tid < kSites) s_most[tid] = 0;
  store(0, r[0]);
  load(kSets, r[0]);
  __syncthreads();
  if (tid < C::BM) {  // which rows carry a LoRA term
    const int64_t m = m0 + tid;
#pragma unroll
    for (int s = 0; s < kSites; ++s) {
      int tenant = 0, r = 0;
      if (m < M) {
        const int64_t req = row_to_req ? (int64_t)row_to_req[m] : m;
        r = (req >= 0 && req < B) ? routed_rank(ad, tenant_id, route, (int)req, B, site + s, &tenant) : 0;
      }
      s_rank[s][tid] = r;
      s_ten[s][tid] = tenant;
      if (r) atomicMax(&s_most[s], r);
    }
  }
  for (int s0 = 0; s0 < stages; s0 += kSets) {
#pragma unroll
    for (int j = 0; j < kSets; ++j) {
      const int st = s0 + j;
      if (st >= stages) break;
      compute(j & 1);
      if (st + 1 < stages) store(st + 1, r[(j + 1) % kSets]);
      load(st + 1 + kSets, r[(j + 1) % kSets]);
      __syncthreads();
    }
  }

  // the groups' sums meet in LDS (lane: row l % 32 of the 32 x 32 tile; registers 4 g .. + 3: columns 8 g + 4 (l / 32) ..)
#pragma unroll
  for (int g = 0; g < 4; ++g)
    *reinterpret_cast<f32x4*>(buf + (size_t)(q * C::BM + wm * 32 + l32) * C::LdR + wn * 32 + g * 8 + lh * 4) =
        f32x4{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
  __syncthreads();
  const int nc = tid % C::BN, r0 = tid / C::BN * C::Outs, n = n0 + nc % kOutN, my = GATED ? nc / kOutN : 0;
  const int ns = n < d2 ? n : d2 - 1;
  const float bv = bias ? Elem<T>::load(bias, ns) : 0.f;
  float val[C::Outs];
#pragma unroll
  for (int i = 0; i < C::Outs; ++i) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < C::KQ; ++k) v += buf[(size_t)(k * C::BM + r0 + i) * C::LdR + nc];
    val[i] = v + bv;
  }

  // LoRA expand, 32 ranks at a time: t of the rows by way of LDS; a thread's rows follow one another, so that they mostly belong to one tenant, whose
  // sixteen rows of W^B it reads once for all of its outputs, tenant by tenant.  Where the rows of some thread belong to more than a few tenants, and for
  // two rows a thread: eight rows of W^B for each output, all outputs' on their way together (`apart`).  300 rows of 1000 x 2730 in fp32, every row
  // routed, us a call tenant by tenant / apart: one tenant, rank 8 33.3 / 37.1, rank 32 36.7 / 46.3; rows dealt to 4 tenants in turn, rank 8
  // 38.0 / 35.5, rank 32 43.6 / 46.3; to 16, rank 8 41.7 / 36.0, rank 32 51.8 / 46.3; in bf16, where a row of W^B is half as long, to 16, rank 8
  // 46.7 / 41.6, rank 32 70.8 / 78.7.  The gated block goes tenant by tenant (its rows are a call's prompts; one tenant 56.7, with the choice in it
  // 58.5).
  float* const ts = buf + C::TsOff;  // [site][row][32]
  int most = s_most[0];
  if (GATED) most = s_most[kSites - 1] > most ? s_most[kSites - 1] : most;
  const float* const tr = ts + (my * C::BM + r0) * 32;
  auto bring_t = [&](int c0) __attribute__((always_inline)) {
    for (int e = tid; e < kSites * C::BM * 32; e += C::T) {
      const int s = e / (C::BM * 32), row = e / 32 % C::BM, c = c0 + (e & 31);
      ts[e] = c < s_rank[s][row] ? t[s * t_site + (size_t)(m0 + row) * ad.r_max + c] : 0.f;
    }
    __syncthreads();
  };
  bool apart = !GATED && C::Outs <= 2;
  if (!GATED && !apart && most > 0) {  // (a lane counts the tenants of some thread's rows; every wave comes to the same answer)
    const int g = lane % (C::BM / C::Outs) * C::Outs;
    int ten[C::Outs], tenants = 0;
#pragma unroll
    for (int i = 0; i < C::Outs; ++i) ten[i] = s_rank[0][g + i] ? s_ten[0][g + i] : -1;
#pragma unroll
    for (int i = 0; i < C::Outs; ++i) {
      bool seen = ten[i] < 0;
#pragma unroll
      for (int k = 0; k < i; ++k) seen |= ten[k] == ten[i];
      tenants += !seen;
    }
    apart = __any(tenants > (most <= 8 ? 3 : 4)) && (sizeof(T) == 4 || most <= 8);
  }
  if (!GATED && most > 0 && apart) {
    const T* Bm[C::Outs];
    int last[C::Outs];
#pragma unroll
    for (int i = 0; i < C::Outs; ++i) {
      last[i] = s_rank[my][r0 + i] - 1;
      Bm[i] = last[i] >= 0 ? (const T*)ad.B[s_ten[my][r0 + i] * MILORA_NUM_SITES + site + my] + ns : nullptr;
    }
    for (int c0 = 0; c0 < most; c0 += 32) {
      bring_t(c0);
      for (int c1 = 0; c1 < 32 && c0 + c1 < most; c1 += 8) {
        float b[C::Outs][8];
#pragma unroll
        for (int i = 0; i < C::Outs; ++i)
#pragma unroll
          for (int u = 0; u < 8; ++u) b[i][u] = c0 + c1 + u <= last[i] ? Elem<T>::load(Bm[i], (size_t)(c0 + c1 + u) * d2) : 0.f;
#pragma unroll
        for (int i = 0; i < C::Outs; ++i)
#pragma unroll
          for (int u = 0; u < 8; ++u) val[i] += tr[i * 32 + c1 + u] * b[i][u];
      }
      __syncthreads();
    }
  } else if (most > 0) {
    for (int c0 = 0; c0 < most; c0 += 32) {
      bring_t(c0);
      unsigned left = 0;  // rows whose term is still to be added
#pragma unroll
      for (int i = 0; i < C::Outs; ++i)
        if (s_rank[my][r0 + i] > c0) left |= 1u << i;
      while (__any(left != 0)) {
        const int row = r0 + (left ? __builtin_ctz(left) : 0), ten = s_ten[my][row], ranks = left ? s_rank[my][row] - c0 : 0;
        const T* const b1 = ranks > 0 ? (const T*)ad.B[ten * MILORA_NUM_SITES + site + my] + (size_t)c0 * d2 + ns : nullptr;
        unsigned mine = 0;
#pragma unroll
        for (int i = 0; i < C::Outs; ++i)
          if ((left >> i & 1) && s_ten[my][r0 + i] == ten) mine |= 1u << i;
        for (int c1 = 0; __any(c1 < ranks) && c1 < 32; c1 += 16) {
          float b[16];
#pragma unroll
          for (int u = 0; u < 16; ++u) b[u] = c1 + u < ranks ? Elem<T>::load(b1, (size_t)(c1 + u) * d2) : 0.f;
#pragma unroll
          for (int i = 0; i < C::Outs; ++i)
            if (mine >> i & 1)
#pragma unroll
              for (int u = 0; u < 16; ++u) val[i] += tr[i * 32 + c1 + u] * b[u];  // (past the rank both are zero)
        }
        left &= ~mine;
      }
      __syncthreads();
    }
  }
#pragma unroll
  for (int i = 0; i < C::Outs; ++i) {
    const int64_t m = m0 + r0 + i;
    if constexpr (GATED) {
      const float up = __shfl_xor(val[i], kOutN, 64);
      if (m >= M || n >= d2) continue;
      const size_t at = (size_t)m * d2 + n;
      float* const save = my ? up_out : gate_out;
      if (save) save[at] = val[i];
      if (my == 0) Elem<T>::store(Y, at, silu(val[i]) * up);
    } else {
      if (m < M && n < d2) Elem<T>::store(Y, (size_t)m * d2 + n, val[i]);
    }
  }
}

struct TileArgs {
  const void* X;
  int64_t M;
  int d1, d2;
  const int32_t* row_to_req;
  const void *W, *W2, *bias;
  AdapterView ad;
  int site;
  const int32_t* tenant_id;
  const uint8_t* route;
  int B;
  const float* t;
  int64_t t_site;
  void* Y;
  float *gate_out, *up_out;
};

template <typename T, class C, bool WIDE, bool GATED>
int launch_tile(const TileArgs& g, hipStream_t stream) {
  static thread_local int lds_set_for = -1;
  int dev = 0;
  MILORA_HIP(hipGetDevice(&dev));
  if (lds_set_for != dev) {
    MILORA_HIP(hipFuncSetAttribute((const void*)linear_tile_kernel<T, C, WIDE, GATED>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LdsBytes));
    lds_set_for = dev;
  }
  constexpr int kOutN = GATED ? C::BN / 2 : C::BN;
  const int tiles_m = (int)((g.M + C::BM - 1) / C::BM);
  const int64_t most = (int64_t)1 << 22;  // tiles of a launch: a grid has to stay below 2^32 threads
  const int64_t cols_most = (most / tiles_m > 0 ? most / tiles_m : 1) * kOutN;
  int rc = MILORA_OK;
  for (int64_t col0 = 0; col0 < g.d2 && !rc; col0 += cols_most) {
    const int64_t cols = g.d2 - col0 < cols_most ? g.d2 - col0 : cols_most;
    const int tiles_n = (int)((cols + kOutN - 1) / kOutN);
    const int64_t grid = ((int64_t)tiles_m * tiles_n + 7) / 8 * 8;
    hipLaunchKernelGGL((linear_tile_kernel<T, C, WIDE, GATED>), dim3((unsigned)grid), dim3(C::T), C::LdsBytes, stream, (const T*)g.X, g.M, g.d1,
                       g.d2, (int)col0, g.row_to_req, (const T*)g.W, (const T*)g.W2, (const T*)g.bias, g.ad, g.site, g.tenant_id, g.route, g.B,
                       g.t, g.t_site, (T*)g.Y, g.gate_out, g.up_out, tiles_m, tiles_n);
    rc = check_launch();
  }
  return rc;
}

// Tiles of more than kFewRows rows, from shrinks that are there.
template <typename T, bool GATED>
int launch_tiles_any(const TileArgs& g, hipStream_t stream) {
  const int64_t large = ((g.M + 63) / 64) * (((int64_t)g.d2 * (GATED ? 2 : 1) + 63) / 64);
  if (g.d1 < 4) return launch_tile<T, GenLarge, false, GATED>(g, stream);
  if (large >= kGenLargeTiles) return launch_tile<T, GenLarge, true, GATED>(g, stream);
  return launch_tile<T, GenSmall, true, GATED>(g, stream);
}

}  // namespace

int launch_shrink(const void* X, int64_t ldx, int64_t M, int d1, int dtype, const int32_t* row_to_req, const AdapterView& ad,
                  int site, int sites, const int32_t* tenant_id, const uint8_t* route, int B, float* t, hipStream_t stream) {
  if (dtype == MILORA_BF16)
    hipLaunchKernelGGL((shrink_rows_kernel<bf16_t>), dim3((unsigned)M, sites), dim3(kShrinkT), 0, stream, (const bf16_t*)X,
                       ldx, M, d1, row_to_req, ad, site, tenant_id, route, B, t);
  else
    hipLaunchKernelGGL((shrink_rows_kernel<float>), dim3((unsigned)M, sites), dim3(kShrinkT), 0, stream, (const float*)X, ldx,
                       M, d1, row_to_req, ad, site, tenant_id, route, B, t);
  return check_launch();
}

template <typename T, int W, bool FUSED>
static int launch_few_rows_t(FewArgs& g, int sites, int mode, hipStream_t st) {
  int rc = MILORA_OK;
  for (int64_t col0 = 0; col0 < g.d2 && !rc; col0 += kLaunchCols) {
    const int cols = g.d2 - col0 < kLaunchCols ? (int)(g.d2 - col0) : kLaunchCols;
    const dim3 grid((unsigned)((cols + 15) / 16), (unsigned)sites);
    g.col0 = (int)col0;
    switch (mode) {
      case kFewPlain: hipLaunchKernelGGL((few_rows_kernel<T, kFewPlain, W, FUSED>), grid, dim3(W * 64), 0, st, g); break;
      case kFewResid: hipLaunchKernelGGL((few_rows_kernel<T, kFewResid, W, FUSED>), grid, dim3(W * 64), 0, st, g); break;
      case kFewGateUp: hipLaunchKernelGGL((few_rows_kernel<T, kFewGateUp, W, FUSED>), dim3(grid.x), dim3(W * 64), 0, st, g); break;
      case kFewGated: hipLaunchKernelGGL((few_rows_kernel<T, kFewGated, W, FUSED>), dim3(grid.x), dim3(W * 64), 0, st, g); break;
      default: hipLaunchKernelGGL((few_rows_kernel<T, kFewDown, W, FUSED>), grid, dim3(W * 64), 0, st, g); break;
    }
    rc = check_launch();
  }
  return rc;
}

// Shrinks inside the launch spare one of its own (3 to 4 us) and cost every wave about 0.7 us per routed row and round trip, a trip
// taking d1 / 8 x rank in pieces of 64 lanes x 8 loads.  With every row routed the two meet at some 10 trips (fp32, 8 rows, 512 x
// 1376, rank 8: 11.3 us a call inside, 12.7 apart; 8 rows, 1000 x 2730: 16.6 and 13.2; 16 rows, 4100 x 11010, rank 16: 306 and
// 59).  In a layer's step a request has one of the seven sites, or a few: there it is some 45 trips of all rows (16 rows, d = 512,
// rank 8, 16 trips and 42 of the down projection: 40.2 and 45.3 us a step; d = 1000, rank 8, 31 and 85: 61.6 and 63.0; rank 16, 62 and
// 171: 80.6 and 70.0).
// (A trip is one of eight waves; four, where few_waves takes them, make one trip of a row's shrink as well.  The calls were made one
// by one from the host, where a second launch costs most; replayed from a graph the two meet sooner, fp32, 512 x 1359, rank 8: 4 rows
// 7.2 us inside and 7.2 apart, 8 rows 10.3 and 7.7, 16 rows 16.3 and 8.0.)
static int64_t shrink_work(int d1, int r_max) {  // of one row, in products
  int rpad = 1;
  while (rpad < r_max) rpad <<= 1;
  return (int64_t)d1 * rpad;
}
static constexpr int64_t shrink_trip(int waves) { return waves * 64 * 8; }

static bool fuse_shrink(int M, int d1, int r_max, bool layer) {
  if (r_max > kFuseRank) return false;
  const int64_t trip = shrink_trip(8), work = shrink_work(d1, r_max);
  return M * (work > trip ? work : trip) <= (layer ? 48 : 16) * trip;
}

// Waves of a launch with the shrinks inside.  Four where eight would each find two blocks of 16 k or fewer and where four form a
// row's shrink in one trip too: fp32, 1359 columns, all rows routed, d1 = 256: rank 8, 1, 8 and 16 rows 4.2, 8.8 and 14.3 us with four and
// 4.7, 10.2 and 16.1 with eight; d1 = 288: 4.6, 11.0, 18.3 and 4.7, 10.0, 16.2; rank 16, 343 columns, d1 = 200, 16 rows: 17.8 and
// 15.2.  Few rows of a layer's step, most of them without a term at a given site, take four up to any rank: d = 256, rank 16, 1 and
// 4 rows 16.9 and 21.4 us a step, 18.6 and 22.8 with eight; 16 rows with three sites each 55.6 and 52.0.
static int few_waves(int M, int d1, int r_max, bool layer) {
  return d1 <= kFewNarrow && (shrink_work(d1, r_max) <= shrink_trip(4) || (layer && M <= 4)) ? 4 : 8;
}

int launch_few_rows(const FewArgs& args, int dtype, int sites, int mode, float* t, hipStream_t st) {
  FewArgs g = args;
  g.t = nullptr;
  const bool layer = sites > 1 || mode != kFewPlain;
  // (the gated block by itself: a linear whose rows are routed to both sites at worst, and twice the sums: fp32, 8 rows, 512 x 1376, rank 8: 18.4 us
  // inside, 10.0 apart; 4 rows, 955 x 2297: 17.8 and 13.2)
  if (!fuse_shrink(mode == kFewGated ? 4 * g.M : g.M, g.d1, g.ad.r_max, layer && mode != kFewGated)) {
    const int rc = launch_shrink(g.X, g.ldx, g.M, g.d1, dtype, g.row_to_req, g.ad, g.site[0], sites, g.tenant_id, g.route, g.B, t, st);
    if (rc) return rc;
    g.t = t;
  }
  const bool bf = dtype == MILORA_BF16;
  if (g.t) return bf ? launch_few_rows_t<bf16_t, 8, false>(g, sites, mode, st) : launch_few_rows_t<float, 8, false>(g, sites, mode, st);
  if (few_waves(g.M, g.d1, g.ad.r_max, layer) == 4) return bf ? launch_few_rows_t<bf16_t, 4, true>(g, sites, mode, st) : launch_few_rows_t<float, 4, true>(g, sites, mode, st);
  return bf ? launch_few_rows_t<bf16_t, 8, true>(g, sites, mode, st) : launch_few_rows_t<float, 8, true>(g, sites, mode, st);
}

int launch_linear_generic(const void* X, int64_t M, int d1, int d2, int dtype, const int32_t* row_to_req,
                          const void* W, const void* bias, const AdapterView& ad, int site,
                          const int32_t* tenant_id, const uint8_t* route, int B, float* t, void* Y, hipStream_t stream) {
  if ((M + 63) / 64 > 65535) return MILORA_ERANGE;
  if (M <= kFewRows) {
    FewArgs g{};
    g.X = X; g.ldx = d1; g.M = (int)M; g.d1 = d1; g.d2 = d2;
    g.W[0] = W; g.bias = bias; g.Y[0] = Y; g.ldy = d2; g.site[0] = site;
    g.row_to_req = row_to_req; g.tenant_id = tenant_id; g.route = route; g.B = B; g.ad = ad;
    return launch_few_rows(g, dtype, 1, kFewPlain, t, stream);
  }
  const int rc = launch_shrink(X, d1, M, d1, dtype, row_to_req, ad, site, 1, tenant_id, route, B, t, stream);
  if (rc) return rc;
  const TileArgs g{X, M, d1, d2, row_to_req, W, nullptr, bias, ad, site, tenant_id, route, B, t, 0, Y, nullptr, nullptr};
  return dtype == MILORA_BF16 ? launch_tiles_any<bf16_t, false>(g, stream) : launch_tiles_any<float, false>(g, stream);
}

int launch_gated_generic(const void* X, int64_t M, int d, int F, int dtype, const int32_t* row_to_req, const void* Wg, const void* Wu,
                         const AdapterView& ad, int site, const int32_t* tenant_id, const uint8_t* route, int B, float* t, void* Y,
                         float* gate_out, float* up_out, hipStream_t stream) {
  if ((M + 63) / 64 > 65535) return MILORA_ERANGE;
  if (M <= kFewRows) {
    FewArgs g{};
    g.X = X; g.ldx = d; g.M = (int)M; g.d1 = d; g.d2 = F;
    g.W[0] = Wg; g.W[1] = Wu; g.Y[0] = Y; g.ldy = F; g.site[0] = site; g.site[1] = site + 1;
    g.row_to_req = row_to_req; g.tenant_id = tenant_id; g.route = route; g.B = B; g.ad = ad;
    g.gate_out = gate_out; g.up_out = up_out;
    return launch_few_rows(g, dtype, 2, kFewGated, t, stream);
  }
  const int rc = launch_shrink(X, d, M, d, dtype, row_to_req, ad, site, 2, tenant_id, route, B, t, stream);
  if (rc) return rc;
  const TileArgs g{X, M, d, F, row_to_req, Wg, Wu, nullptr, ad, site, tenant_id, route, B, t, M * ad.r_max, Y, gate_out, up_out};
  return dtype == MILORA_BF16 ? launch_tiles_any<bf16_t, true>(g, stream) : launch_tiles_any<float, true>(g, stream);
}

}  // namespace milora

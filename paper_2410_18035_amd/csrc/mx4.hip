// Base weights of 4 bits: w = E2M1(code) * 2^(s - 127), one scale byte s for 32 inputs of a column (the OCP microscaling
// format MXFP4).  A power-of-two scale leaves every weight a bf16 number, so the matrix cores see the weights exactly and the
// chip converts two of them in one instruction (v_cvt_scalef32_pk_bf16_fp4, the scale in it).
//
// Quantise: s = floor(log2 of the group's largest magnitude) - 2 + 127, kept within 2 .. 252 (no value of a group is then a
// denormal or beyond bf16), codes rounded to nearest, ties to even, magnitudes above 6 to 6; a group that holds Inf or NaN gets
// s = 255, its weights are NaN.
#include "mx4.h"

namespace milora {
namespace {

typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---- conversion ---------------------------------------------------------------------------------------------------------
// Four lanes share a group of 32, eight values each.  Bound: HBM.
constexpr int kQuantT = 256;
constexpr int kQuantU = 2;  // groups of a lane on their way

template <typename T>
__device__ __forceinline__ void load_eight(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load_eight<bf16_t>(const bf16_t* p, float (&v)[8]) {
  const u32x4 w = *reinterpret_cast<const u32x4_a2*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(w[e] << 16);
    v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
}
template <>
__device__ __forceinline__ void load_eight<float>(const float* p, float (&v)[8]) {
  typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4 w = reinterpret_cast<const f32x4_a4*>(p)[h];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * h + e] = w[e];
  }
}

template <typename T>
__global__ void __launch_bounds__(kQuantT) mx4_quantize_kernel(const T* __restrict__ src, uint32_t* __restrict__ codes,
                                                               uint8_t* __restrict__ scales, int64_t eighths) {
  const int64_t i0 = (int64_t)blockIdx.x * (kQuantT * kQuantU) + threadIdx.x;
  float v[kQuantU][8];
#pragma unroll
  for (int u = 0; u < kQuantU; ++u) {  // (a wave's lanes past the end take the last eight again and store nothing)
    const int64_t i = i0 + u * kQuantT;
    load_eight<T>(src + (i < eighths ? i : eighths - 1) * 8, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kQuantU; ++u) {
    const int64_t i = i0 + u * kQuantT;
    uint32_t top = 0;  // the largest magnitude's bits: they compare as the magnitudes do, Inf and NaN above all
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t b = __float_as_uint(v[u][e]) & 0x7fffffffu;
      top = b > top ? b : top;
    }
#pragma unroll
    for (int off = 1; off < 4; off <<= 1) {
      const uint32_t o = __shfl_xor(top, off, 64);
      top = o > top ? o : top;
    }
    const int biased = (int)(top >> 23);  // (of a denormal: 0, below the least scale in any case)
    int s = biased - 2;
    s = s < 2 ? 2 : s;
    const bool finite = biased < 255;
    const float scale = __uint_as_float((uint32_t)s << 23);
    uint32_t c = 0;
    if (finite) {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][0], v[u][1], scale, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][2], v[u][3], scale, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][4], v[u][5], scale, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[u][6], v[u][7], scale, 3);
    }
    if (i < eighths) {
      codes[i] = c;
      if ((threadIdx.x & 3) == 0) scales[i >> 2] = finite ? (uint8_t)s : (uint8_t)255;
    }
  }
}

// A thread takes eight codes at a time.  PACKED: in the order of the packed layout (16 columns x 32 inputs a block).  Bound: HBM.
template <typename T, bool PACKED>
__global__ void __launch_bounds__(kQuantT) mx4_dequantize_kernel(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                 T* __restrict__ dst, int64_t eighths, int d1) {
  const int64_t i0 = (int64_t)blockIdx.x * (kQuantT * kQuantU) + threadIdx.x;
  uint32_t c[kQuantU], s[kQuantU];
#pragma unroll
  for (int u = 0; u < kQuantU; ++u) {
    const int64_t i = i0 + u * kQuantT;
    int64_t from = i < eighths ? i : eighths - 1;
    if (PACKED) {
      const int KT = d1 >> 5, ln = (int)(from & 63);
      const int64_t blk = from >> 6, nt = blk / KT, kt = blk % KT;
      from = ((nt * 16 + (ln & 15)) * KT + kt) * 4 + (ln >> 4);
    }
    c[u] = codes[from];
    s[u] = scales[from >> 2];
  }
#pragma unroll
  for (int u = 0; u < kQuantU; ++u) {
    const int64_t i = i0 + u * kQuantT;
    if (i >= eighths) continue;
    const u32x4 b = mx4_bf16(c[u], mx4_scale(s[u]));
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x4_a2*>(dst + i * 8) = b;
    } else {
      typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
      for (int h = 0; h < 2; ++h)
        reinterpret_cast<f32x4_a4*>(dst + i * 8)[h] =
            f32x4{__uint_as_float(b[2 * h] << 16), __uint_as_float(b[2 * h] & 0xffff0000u), __uint_as_float(b[2 * h + 1] << 16),
                  __uint_as_float(b[2 * h + 1] & 0xffff0000u)};
    }
  }
}

// ---- few rows: two launches a level -----------------------------------------------------------------------------------------
// First launch: the base products and the LoRA shrinks, which do not depend on each other.  A workgroup of eight waves takes 256 / KW columns, 32 a
// wave, and KW x NL x 64 inputs, all of them at once: a lane holds NL groups of 32 inputs, 16 bytes of codes each, straight
// from global memory, every load on its way together; KW waves share the columns and split the inputs, so that few rows, whose X is small, need few
// parts of the reduction or none.  X goes through LDS, 32 rows at a time; with more rows the codes stay in registers and the next rows' X is on its
// way while these are multiplied.  Matrix instructions of 8 inputs a lane multiply the groups (which inputs stand at which place does not matter
// as long as both operands agree), those of 16 x 16 up to 16 rows, which take half the time.  The waves' sums meet in LDS, those of the parts in memory, in fp32.
// Second launch: adds the parts in part order, the LoRA term t W^B, bias and glue, and rounds once.
// Bound: the stream of the codes; what short reductions cost is their sums' way through memory.  Tried: stages of 256 inputs with the next ones on
// their way over a longer reduction (M = 64, 4096 x 4096: 23 us a call against 15), the whole reduction and the term in one launch with 2 x 8
// waves a compute unit (gated, 32 rows of 4096 x 11008: 60 us against 28).
constexpr int kMxW = 8;
constexpr int kMxT = kMxW * 64;
constexpr int kMxCols = kMxW * 32;

// What a row has at a site: W^B and rank, or rank 0.
struct MxTerm {
  const bf16_t* B;
  int r, unused;
};

struct MxBase {
  const bf16_t* X;
  int64_t ldx;
  int M, d1, d2;
  const unsigned char* W[3];
  int sites, col_groups, row_groups, row_split, parts;  // row groups of 32; a workgroup takes every row_split-th
  float* partial;  // [site][part][M][d2]
  int shrink_parts, shrink_z;  // the shrink: parts of a row, workgroups in all (a multiple of 8)
  ShrinkArgs shrink;
  const bf16_t* second;  // SECOND: second rows of the shrink's X
  MxTerm* terms;  // [site][M]
};

constexpr int kMxShrinkK = 1024;
// Workgroup `id` of those in front: the shrink of one row, site and 1024 inputs; most rows have no term and end at once.  SECOND: X is the sum of the
// row and its second one (a choice in the loop would have every load waited for by itself: one row of 4096 x 4096 12.2 us a call for 11.0).
template <bool SECOND>
__device__ __forceinline__ void mx4_shrink_row(const MxBase& g, int id, unsigned char* lds) {
  const ShrinkArgs& sh = g.shrink;
  const int tid = threadIdx.x, lane = tid & 63, d1 = g.d1;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int M = (int)sh.M;
  if (id >= M * g.sites * g.shrink_parts) return;
  const int part = id % g.shrink_parts, m = id / g.shrink_parts % M, s = id / (g.shrink_parts * M), site = sh.site + s;
  const int64_t req = sh.row_to_req ? (int64_t)sh.row_to_req[m] : m;
  int ten = -1;
  const int r = req >= 0 && req < sh.B ? routed_rank(sh.ad, sh.tenant_id, sh.route, (int)req, sh.B, site, &ten) : 0;
  if (part == 0 && tid == 0) g.terms[s * sh.lora_site + m] = MxTerm{r ? (const bf16_t*)sh.ad.B[ten * MILORA_NUM_SITES + site] : nullptr, r, 0};
  if (r == 0) return;
  gbf16* const A = in_global(sh.ad.A[ten * MILORA_NUM_SITES + site]);
  const bf16_t* const x = sh.X + (size_t)m * sh.ldx;
  const bf16_t* const x2 = SECOND ? g.second + (size_t)m * sh.ldx : nullptr;
  // lane: eight ranks (piece) of every kpl-th input of the wave's 128
  const int pieces = (r + 7) >> 3;
  int p2 = 1;
  while (p2 < pieces) p2 <<= 1;
  const int piece = lane & (p2 - 1), kpl = 64 / p2, left = r - piece * 8;
  const int k0 = part * kMxShrinkK + w * (kMxShrinkK / kMxW), k1 = k0 + kMxShrinkK / kMxW < d1 ? k0 + kMxShrinkK / kMxW : d1;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  if (left > 0)
    for (int k = k0 + lane / p2; k < k1; k += 8 * kpl) {
      u32x4 a[8];
      float xv[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int kk = k + u * kpl < k1 ? k + u * kpl : k;
        gbf16* const q = A + (size_t)kk * r + piece * 8;
        if (left >= 8) a[u] = *(gu32x4_any*)q;
        else a[u] = load8(q, left, false);
        xv[u] = bf16_to_f32(x[kk]);
        if constexpr (SECOND) xv[u] += bf16_to_f32(x2[kk]);  // (16 bits of h, exact in fp32)
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (k + u * kpl < k1)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sum[2 * e] += xv[u] * __uint_as_float(a[u][e] << 16);
            sum[2 * e + 1] += xv[u] * __uint_as_float(a[u][e] & 0xffff0000u);
          }
    }
  float* const red = reinterpret_cast<float*>(lds);  // [wave][256]
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    for (int off = p2; off < 64; off <<= 1) sum[e] += __shfl_xor(sum[e], off, 64);
    if (lane < p2) red[w * 256 + lane * 8 + e] = sum[e];
  }
  __syncthreads();
  if (tid < r) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kMxW; ++k) v += red[k * 256 + tid];
    sh.t[s * sh.t_site + part * sh.t_stride + (size_t)m * sh.ad.r_max + tid] = v;
  }
}

// MORE: more than 32 rows.  XM: pieces of X a thread brings; with four the registers allow three workgroups a compute unit (gated, one row of
// 4096 x 11008, 688 workgroups: 15.4 us a call, with two 20.3); up to 64 of them with the shorter parts four (what the shrink of second rows takes more
// would leave three: one request of 5120 x 13824 56.1 us a decode step for 54.6).
// SECOND (MxArgs::second): kBehind: the second rows follow the first ones among the M rows; kPlanes: a row group's second rows go through LDS after its
// first ones and are added to the same sums.
enum MxSecond { kNone, kBehind, kPlanes };
template <int KW, int NL, bool MORE, int XM, MxSecond SECOND>
__global__ void __launch_bounds__(kMxT, NL < 8 && SECOND == kBehind ? 8 : XM <= 4 ? 6 : 4) mx4_base_kernel(const MxBase g) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int d1 = g.d1;
  int id = blockIdx.x;
  if (id < g.shrink_z) {
    mx4_shrink_row<SECOND != kNone>(g, id, lds);
    return;
  }
  // workgroup -> tile: ids go round-robin over the 8 XCDs (those in front are a multiple of 8); with more than 32 rows an XCD takes a contiguous
  // run of an order in which the workgroups of the same codes follow one another, so that its L2 serves them after the first
  id -= g.shrink_z;
  const int row_split = MORE ? g.row_split : 1;
  const int total = g.sites * g.col_groups * row_split * g.parts, per = (total + 7) >> 3;
  if (MORE) id = (id & 7) * per + (id >> 3);
  if (id >= total) return;
  constexpr int kCols = kMxCols / KW, kPart = KW * NL * 64;  // columns and inputs of the workgroup
  constexpr int kScalePitch = KW * NL * 2 + 16, kScaleArea = kCols * kScalePitch;  // scales in LDS, [column][..], in front of X
  constexpr int kPitch = kPart * 2 + 16;                     // a row of X in LDS: 16 bytes past a multiple of all banks
  // Up to 16 rows: matrix instructions of 16 x 16, 32 inputs.  A lane's group g of a column: inputs 32 g of every kG x 32, kH columns a lane
  constexpr bool k16 = KW >= 4;
  constexpr int kSide = k16 ? 16 : 32, kG = 64 / kSide, kH = 32 / kSide, kS = NL / kH;  // kS steps of kG groups
  const int ln = lane & (kSide - 1), lg = lane / kSide, kw = w % KW, cw = w / KW;
  int rg = id % row_split;
  const int part = id / row_split % g.parts, cg = id / (row_split * g.parts) % g.col_groups, site = id / (row_split * g.parts * g.col_groups);
  const int n0 = cg * kCols + cw * 32, k_part = part * kPart, k0 = k_part + kw * NL * 64;

  // ---- X: [row][kPart], asked for in front of the codes, which may come later ----
  constexpr int kPieces = kPart / 8, kXMost = XM;  // (rows x kPieces is kXMost x kMxT at most)
  u32x4 x[kXMost];
  auto ask_x = [&](const bf16_t* X, int m0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kXMost; ++u) {
      const int e = tid + u * kMxT, m = m0 + e / kPieces, p = e % kPieces;
      x[u] = u32x4{0u, 0u, 0u, 0u};
      if (e < 32 * kPieces && m < g.M && k_part + p * 8 < d1) x[u] = *reinterpret_cast<const u32x4*>(X + (size_t)m * g.ldx + k_part + p * 8);
    }
  };
  // ---- scales: whole lines of the workgroup's columns, into LDS with the first rows of X ----
  constexpr int kScales = KW * NL * 2, kScalePieces = kScales / 16;  // bytes of a column, and pieces
  u32x4 scales = u32x4{0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
  const int scale_col = tid / kScalePieces, scale_piece = tid % kScalePieces;
  if (scale_col < kCols) {
    int col = cg * kCols + scale_col;
    col = col < g.d2 ? col : g.d2 - 1;  // (columns past the end: results dropped)
    const int from = (k_part >> 5) + scale_piece * 16, left = (d1 >> 5) - from;
    const uint8_t* const sp = g.W[site] + (size_t)d1 * g.d2 / 2 + (size_t)col * (d1 >> 5) + from;
    typedef uint32_t u32x4_a1 __attribute__((ext_vector_type(4), aligned(1)));
    if (left >= 16) {
      scales = *reinterpret_cast<const u32x4_a1*>(sp);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < left) scales[e >> 2] = (scales[e >> 2] & ~(255u << (8 * (e & 3)))) | ((uint32_t)sp[e] << (8 * (e & 3)));
    }
  }
  ask_x(g.X, rg * 32);
  __builtin_amdgcn_sched_barrier(0);
  // ---- codes: NL steps ----
  u32x4 c[kH][kS];
#pragma unroll
  for (int h = 0; h < kH; ++h) {
    int col = n0 + h * kSide + ln;
    col = col < g.d2 ? col : g.d2 - 1;  // (columns past the end: results dropped)
    const unsigned char* const wp = g.W[site] + (size_t)col * (d1 >> 1) + lg * 16 + (k0 >> 1);
    if (k0 + NL * 64 <= d1) {
#pragma unroll
      for (int i = 0; i < kS; ++i) c[h][i] = *reinterpret_cast<const u32x4*>(wp + i * kG * 16);
    } else {  // zeros past the end of the reduction
#pragma unroll
      for (int i = 0; i < kS; ++i) {
        const int at = k0 + (i * kG + lg) * 32;
        c[h][i] = u32x4{0u, 0u, 0u, 0u};
        if (at < d1) c[h][i] = *reinterpret_cast<const u32x4*>(wp + i * kG * 16);
      }
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  auto barrier = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0xc07f);  // LDS reads and writes done; what is on its way from memory stays so
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  constexpr int Ld = kMxCols + 4;  // a row of all waves' columns: [row][wave][32]
  float* const red = reinterpret_cast<float*>(lds + kScaleArea);
  if (scale_col < kCols) *reinterpret_cast<u32x4*>(lds + scale_col * kScalePitch + scale_piece * 16) = scales;
  typedef typename std::conditional<k16, uint32_t, uint16_t>::type scales_t;  // of a step: kG bytes
  typename std::conditional<k16, f32x4, f32x16>::type acc[kH];
  bool second = false;  // (kPlanes) second rows are being multiplied
  for (;;) {
    const int m0 = rg * 32, rows = g.M - m0 < 32 ? g.M - m0 : 32;
#pragma unroll
    for (int u = 0; u < kXMost; ++u) {
      const int e = tid + u * kMxT, r = e / kPieces, p = e % kPieces;
      if (r < rows) *reinterpret_cast<u32x4*>(lds + kScaleArea + r * kPitch + p * 16) = x[u];
    }
    barrier();
    const bool again = SECOND == kPlanes && !second;  // the second rows of these come next
    if (!again) rg += row_split;
    const bool more = again || (MORE && rg < g.row_groups);
    if (more) ask_x(again ? g.second : g.X, rg * 32);
    if (!second)
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int e = 0; e < (k16 ? 4 : 16); ++e) acc[h][e] = 0.f;
    if (n0 < g.d2 && k0 < d1) {
      const int row = ln < rows ? ln : rows - 1;  // (rows past the end: results dropped)
      const unsigned char* const xr = lds + kScaleArea + row * kPitch + kw * NL * 128 + lg * 64;
      const scales_t* const sr = reinterpret_cast<const scales_t*>(lds + (cw * 32 + ln) * kScalePitch + kw * NL * 2);
#pragma unroll
      for (int i = 0; i < kS; ++i) {
        float scale[kH];
#pragma unroll
        for (int h = 0; h < kH; ++h) scale[h] = mx4_scale(((uint32_t)sr[h * kSide * (kScalePitch / (int)sizeof(scales_t)) + i] >> (8 * lg)) & 255u);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bf16x8 xv = *reinterpret_cast<const bf16x8*>(xr + i * kG * 64 + e * 16);
#pragma unroll
          for (int h = 0; h < kH; ++h) {
            const bf16x8 wv = __builtin_bit_cast(bf16x8, mx4_bf16(c[h][i][e], scale[h]));
            if constexpr (k16) acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xv, acc[h], 0, 0, 0);
            else acc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wv, xv, acc[h], 0, 0, 0);
          }
        }
      }
    }
    barrier();
    if (SECOND == kPlanes) second = again;
    if (again) continue;
    // ---- the waves' sums ----
    if (ln < rows)
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int q = 0; q < (k16 ? 1 : 4); ++q)
          *reinterpret_cast<f32x4*>(red + ln * Ld + w * 32 + h * kSide + q * 8 + lg * 4) =
              f32x4{acc[h][4 * q], acc[h][4 * q + 1], acc[h][4 * q + 2], acc[h][4 * q + 3]};
    barrier();
    float* const out = g.partial + ((size_t)(site * g.parts + part) * g.M + m0) * g.d2 + cg * kCols;
    for (int e = tid; e < rows * (kCols / 4); e += kMxT) {
      const int r = e / (kCols / 4), n = e % (kCols / 4) * 4;
      if (cg * kCols + n >= g.d2) continue;
      const float* const q = red + r * Ld + (n / 32) * KW * 32 + n % 32;
      f32x4 v = *reinterpret_cast<const f32x4*>(q);
#pragma unroll
      for (int k = 1; k < KW; ++k) v += *reinterpret_cast<const f32x4*>(q + k * 32);
      st_through(reinterpret_cast<f32x4*>(out + (size_t)r * g.d2 + n), v);  // (left in the L2, the launch ends by writing it back: 96 rows 33 us a call, so 31)
    }
    if (!more) return;
    barrier();
  }
}

// ---- second launch: a workgroup takes 256 columns of a row (GATED: of both projections), its four waves a quarter of the parts and of the
// ranks each, so that everything a row needs is on its way together ----
constexpr int kFinT = 256, kFinCols = 256;
struct MxFinish {
  MxArgs a;
  int parts, rows;  // rows of a part: a.M, or twice that (kBehind)
  const float* partial;
  const float* t;  // [site][t_parts][M][r_max]
  size_t t_part, t_site;
  int t_parts;
  const MxTerm* terms;  // [site][M]
};
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x2_a8 __attribute__((ext_vector_type(2)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

template <bool GATED>
__global__ void __launch_bounds__(kFinT, 4) mx4_finish_kernel(const MxFinish f) {
  constexpr int kSites = GATED ? 2 : 1;
  __shared__ float ts[kSites][MILORA_MAX_RANK];
  __shared__ float ss[kFinT / 64];
  __shared__ f32x4 red[kFinT / 64][kSites][64];
  const MxArgs& g = f.a;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, m = blockIdx.y, s0 = GATED ? 0 : blockIdx.z;
  const int n = blockIdx.x * kFinCols + lane * 4;
  const bool in = n < g.d2;
  MxTerm tr[kSites];
#pragma unroll
  for (int s = 0; s < kSites; ++s) tr[s] = f.terms[(size_t)(s0 + s) * g.M + m];
  // ---- this wave's parts ----
  f32x4 v[kSites];
#pragma unroll
  for (int s = 0; s < kSites; ++s) {
    v[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    const size_t stride = (size_t)f.rows * g.d2;
    const float* const q = f.partial + ((size_t)(s0 + s) * f.parts * f.rows + m) * g.d2 + (in ? n : 0);
    for (int p = w; p < f.parts; p += 16) {
      f32x4 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = *reinterpret_cast<const f32x4*>(q + (p + 4 * u < f.parts ? p + 4 * u : p) * stride);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (p + 4 * u < f.parts) v[s] += x[u];
      if (f.rows > g.M) {
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = *reinterpret_cast<const f32x4*>(q + (size_t)g.M * g.d2 + (p + 4 * u < f.parts ? p + 4 * u : p) * stride);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (p + 4 * u < f.parts) v[s] += x[u];
      }
    }
  }
  // ---- normalisation of the level's input: a factor of the row, applied to its products ----
  const bool norm = g.norm_x || g.norm_h;
  if (norm) {
    float sum = 0.f;
    if (g.norm_x) {
      const bf16_t* const x = g.norm_x + (size_t)m * g.d1;
      for (int i = tid * 8; i < g.d1; i += kFinT * 8) {
        const u32x4 q = *reinterpret_cast<const u32x4*>(x + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float a = __uint_as_float(q[e] << 16), b = __uint_as_float(q[e] & 0xffff0000u);
          sum += a * a + b * b;
        }
      }
    } else {
      const float* const h = g.norm_h + (size_t)m * g.d1;
      for (int i = tid * 4; i < g.d1; i += kFinT * 4) {
        const f32x4 q = *reinterpret_cast<const f32x4*>(h + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += q[e] * q[e];
      }
    }
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) ss[w] = sum;
  }
  // ---- LoRA: t of the row, this wave's ranks of W^B ----
  const bool lora = tr[0].r || tr[kSites - 1].r;
  if (lora) {
    gbf16* b[kSites];
#pragma unroll
    for (int s = 0; s < kSites; ++s)
      b[s] = in_global(tr[s].B) + (in ? n : 0);
#pragma unroll
    for (int s = 0; s < kSites; ++s)
      if (tid < tr[s].r) {
        const float* const tp = f.t + (s0 + s) * f.t_site + (size_t)m * g.ad.r_max + tid;
        float x = 0.f;
        for (int p = 0; p < f.t_parts; p += 4) {
          float q[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) q[u] = tp[(p + u < f.t_parts ? p + u : p) * f.t_part];
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (p + u < f.t_parts) x += q[u];
        }
        ts[s][tid] = x;
      }
    constexpr int kU = 8;
    u32x2_a2 first[kSites][kU];
#pragma unroll
    for (int s = 0; s < kSites; ++s)
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int c = w + 4 * u;
        if (tr[s].r) first[s][u] = *(__attribute__((address_space(1))) const u32x2_a2*)(b[s] + (size_t)(c < tr[s].r ? c : 0) * g.d2);
      }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kSites; ++s) {
      const int r = tr[s].r;
      auto add = [&](int c, u32x2_a2 x) __attribute__((always_inline)) {
        if (c >= r) return;
        const float t = ts[s][c];
        v[s][0] += t * __uint_as_float(x[0] << 16);
        v[s][1] += t * __uint_as_float(x[0] & 0xffff0000u);
        v[s][2] += t * __uint_as_float(x[1] << 16);
        v[s][3] += t * __uint_as_float(x[1] & 0xffff0000u);
      };
      if (r)
#pragma unroll
        for (int u = 0; u < kU; ++u) add(w + 4 * u, first[s][u]);
      for (int c0 = w + 4 * kU; c0 < r; c0 += 4 * kU) {
        u32x2_a2 x[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) x[u] = *(__attribute__((address_space(1))) const u32x2_a2*)(b[s] + (size_t)(c0 + 4 * u < r ? c0 + 4 * u : 0) * g.d2);
#pragma unroll
        for (int u = 0; u < kU; ++u) add(c0 + 4 * u, x[u]);
      }
    }
  }
  // ---- glue, by the first wave ----
#pragma unroll
  for (int s = 0; s < kSites; ++s) red[w][s][lane] = v[s];
  __syncthreads();
  if (w || !in) return;
#pragma unroll
  for (int s = 0; s < kSites; ++s) v[s] = (red[0][s][lane] + red[1][s][lane]) + (red[2][s][lane] + red[3][s][lane]);
  if (norm) {
    const float inv = rsqrtf((ss[0] + ss[1] + ss[2] + ss[3]) / (float)g.d1 + 1e-5f);
#pragma unroll
    for (int s = 0; s < kSites; ++s) v[s] *= inv;
  }
  const size_t at = (size_t)m * g.d2 + n;
  f32x4 y;
  if constexpr (GATED) {
    if (g.gate_out) *reinterpret_cast<f32x4_a4*>(g.gate_out + at) = v[0];
    if (g.up_out) *reinterpret_cast<f32x4_a4*>(g.up_out + at) = v[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = silu(v[0][e]) * v[1][e];
  } else {
    y = v[0];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (g.bias) y[e] += bf16_to_f32(g.bias[n + e]);
      if (g.res) y[e] += bf16_to_f32(g.res[at + e]);
    }
    if (g.res) *reinterpret_cast<f32x4*>(g.h_out + at) = y;
    if (g.h_in) y += *reinterpret_cast<const f32x4*>(g.h_in + at);
  }
  u32x2_a8 o;
  o[0] = pack_bf16x2(y[0], y[1]);
  o[1] = pack_bf16x2(y[2], y[3]);
  *reinterpret_cast<u32x2_a8*>(g.Y[s0] + (size_t)m * g.ldy + n) = o;
  if (!GATED && g.left_out) {
    u32x2_a8 left;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      left[e] = pack_bf16x2(rest_of(y[2 * e], __uint_as_float(o[e] << 16)), rest_of(y[2 * e + 1], __uint_as_float(o[e] & 0xffff0000u)));
    *reinterpret_cast<u32x2_a8*>(g.left_out + at) = left;
  }
}

constexpr int kMxSteps = 8;
template <int KW, int NL, bool MORE, int XM, MxSecond SECOND>
int launch_base(const MxBase& b, hipStream_t st) {
  constexpr int kPart = KW * NL * 64, kRed = 32 * (kMxCols + 4) * 4;
  const int rows = b.M < 32 ? b.M : 32, x = rows * (kPart * 2 + 16), red = rows * (kMxCols + 4) * 4;
  int bytes = x > red ? x : red;
  constexpr int kScaleArea = kMxCols / KW * (KW * NL * 2 + 16);
  bytes += kScaleArea;
  if (bytes < kMxW * 256 * 4) bytes = kMxW * 256 * 4;  // (the shrink's sums)
  static thread_local int lds_set_for = -1;
  int dev = 0;
  MILORA_HIP(hipGetDevice(&dev));
  if (lds_set_for != dev) {
    const int most = (32 * (kPart * 2 + 16) > kRed ? 32 * (kPart * 2 + 16) : kRed) + kScaleArea;
    MILORA_HIP(hipFuncSetAttribute((const void*)mx4_base_kernel<KW, NL, MORE, XM, SECOND>, hipFuncAttributeMaxDynamicSharedMemorySize, most < 160 * 1024 ? most : 160 * 1024));
    lds_set_for = dev;
  }
  const int64_t total = (int64_t)b.sites * b.col_groups * b.row_split * b.parts, grid = b.shrink_z + (total + 7) / 8 * 8;
  hipLaunchKernelGGL((mx4_base_kernel<KW, NL, MORE, XM, SECOND>), dim3((unsigned)grid), dim3(kMxT), bytes, st, b);
  return check_launch();
}

// (kBehind: two to sixteen rows; kPlanes: more than kMxBehind)
template <MxSecond SECOND>
int launch_base_of(const MxBase& b, int rows, int kw, bool half, hipStream_t st) {
  if constexpr (SECOND != kBehind) {
    if (kw == 2) return b.row_groups == 1 ? launch_base<2, kMxSteps, false, 8, SECOND>(b, st) : launch_base<2, kMxSteps, true, 8, SECOND>(b, st);
  }
  if constexpr (SECOND != kPlanes) {
    static_assert(kMxBehind >= 8, "rows of mx4_waves");
    if (rows <= 2) return launch_base<8, kMxSteps / 2, false, 1, SECOND>(b, st);
    if (kw == 8 && half) return launch_base<8, kMxSteps / 2, false, 4, SECOND>(b, st);
    if (kw == 8 && rows <= 4) return launch_base<8, kMxSteps, false, 4, SECOND>(b, st);
    if (kw == 8) return launch_base<8, kMxSteps, false, 8, SECOND>(b, st);
  }
  return half ? launch_base<4, kMxSteps / 2, false, 4, SECOND>(b, st) : launch_base<4, kMxSteps, false, 8, SECOND>(b, st);
}

// How the first launch cuts a call; functions of the sizes alone.  Waves that share columns: X of a row group is rows x KW x NL x 128 bytes, 64 KB
// of LDS at most (two workgroups a compute unit), and few parts.  Up to 16 rows parts of half the length where they let more workgroups run at once:
// one and two rows always (us a call, one row, 4096 x 4096 8.0 for 8.8, 4096 x 12288 11.1 for 12.0, gated 4096 x 11008 14.7 for 14.9), the
// others where whole ones are more than two for each compute unit (gated 4096 x 11008, 8 rows 18.4 for 22.6, 16 rows 21.9 for 24.0; where they
// are not: 4096 x 12288, 4 rows 14.5 for 13.9, 16 rows 16.0 for 15.4).
int mx4_waves(int64_t M) { return M <= 8 ? 8 : M <= 16 ? 4 : 2; }
bool mx4_short(int64_t M, int d1, int d2, int sites) {
  const int kw = mx4_waves(M), cols = kMxCols / kw, part = kw * kMxSteps * 64;
  return M <= 2 || (M <= 16 && (int64_t)sites * (((int64_t)d2 + cols - 1) / cols) * ((d1 + part - 1) / part) > 512);
}
// (with the shorter parts where they can be: no size lowers it)
size_t mx4_partial_floats(int64_t M, int d1, int d2, int sites) {
  const int part = mx4_waves(M) * kMxSteps * 64 / (M <= 16 ? 2 : 1);
  return (size_t)M * d2 * sites * ((d1 + part - 1) / part);
}
int mx4_shrink_parts(int d1) { return (d1 + kMxShrinkK - 1) / kMxShrinkK; }

struct MxCut {
  int kw;     // waves that share columns
  bool half;  // parts of half the length
  int parts, col_groups, row_groups, row_split;
};
// rows: of X, the second ones among them
MxCut mx4_cut(int64_t rows, int d1, int d2, int sites) {
  MxCut c;
  c.kw = mx4_waves(rows);
  c.half = mx4_short(rows, d1, d2, sites);
  const int part = c.kw * kMxSteps * 64 / (c.half ? 2 : 1);
  c.parts = (d1 + part - 1) / part;
  c.col_groups = (int)(((int64_t)d2 + kMxCols / c.kw - 1) / (kMxCols / c.kw));
  // row groups of the same codes in one workgroup once the workgroups are two for each compute unit: the codes are then read once
  c.row_groups = (int)((rows + 31) / 32);
  const int64_t units = (int64_t)sites * c.col_groups * c.parts;
  c.row_split = (int)(512 / units < 1 ? 1 : 512 / units < c.row_groups ? 512 / units : c.row_groups);
  return c;
}

// Groups of eight of one launch: a grid has to stay below 2^32 threads.
constexpr int64_t kQuantSlice = (int64_t)1 << 30;

}  // namespace

int mx4_quantize(const void* src, int dtype, void* dst, int d1, int d2, hipStream_t st) {
  const int64_t eighths = (int64_t)d1 * d2 / 8;
  uint32_t* const codes = (uint32_t*)dst;
  uint8_t* const scales = (uint8_t*)dst + mx4_code_bytes(d1, d2);
  int rc = MILORA_OK;
  for (int64_t i = 0; i < eighths && !rc; i += kQuantSlice) {
    const int64_t n = eighths - i < kQuantSlice ? eighths - i : kQuantSlice;
    const dim3 grid((unsigned)((n + kQuantT * kQuantU - 1) / (kQuantT * kQuantU)));
    if (dtype == MILORA_BF16)
      hipLaunchKernelGGL(mx4_quantize_kernel<bf16_t>, grid, dim3(kQuantT), 0, st, (const bf16_t*)src + i * 8, codes + i, scales + i / 4, n);
    else
      hipLaunchKernelGGL(mx4_quantize_kernel<float>, grid, dim3(kQuantT), 0, st, (const float*)src + i * 8, codes + i, scales + i / 4, n);
    rc = check_launch();
  }
  return rc;
}

int mx4_dequantize(const void* src, void* dst, int dtype, int d1, int d2, bool packed, hipStream_t st) {
  const int64_t eighths = (int64_t)d1 * d2 / 8;
  const uint32_t* const codes = (const uint32_t*)src;
  const uint8_t* const scales = (const uint8_t*)src + mx4_code_bytes(d1, d2);
  if (packed) {
    if (eighths > kQuantSlice) return MILORA_ERANGE;
    hipLaunchKernelGGL((mx4_dequantize_kernel<bf16_t, true>), dim3((unsigned)((eighths + kQuantT * kQuantU - 1) / (kQuantT * kQuantU))), dim3(kQuantT),
                       0, st, codes, scales, (bf16_t*)dst, eighths, d1);
    return check_launch();
  }
  int rc = MILORA_OK;
  for (int64_t i = 0; i < eighths && !rc; i += kQuantSlice) {
    const int64_t n = eighths - i < kQuantSlice ? eighths - i : kQuantSlice;
    const dim3 grid((unsigned)((n + kQuantT * kQuantU - 1) / (kQuantT * kQuantU)));
    if (dtype == MILORA_BF16)
      hipLaunchKernelGGL((mx4_dequantize_kernel<bf16_t, false>), grid, dim3(kQuantT), 0, st, codes + i, scales + i / 4, (bf16_t*)dst + i * 8, n, d1);
    else
      hipLaunchKernelGGL((mx4_dequantize_kernel<float, false>), grid, dim3(kQuantT), 0, st, codes + i, scales + i / 4, (float*)dst + i * 8, n, d1);
    rc = check_launch();
  }
  return rc;
}

size_t mx4_rows_workspace_bytes(int64_t M, int d1, int d2, int r_max, int sites, bool second) {
  // (second rows: the largest need of up to M rows, so that it never falls with M)
  const int64_t rows = !second ? M : M <= kMxBehind ? 2 * M : M > 2 * kMxBehind ? M : 2 * kMxBehind;
  return align_up((size_t)M * mx4_shrink_parts(d1) * r_max * sites * sizeof(float), 256) + align_up((size_t)M * sites * sizeof(MxTerm), 256) +
         align_up(mx4_partial_floats(rows, d1, d2, sites) * sizeof(float), 256);
}

bool mx4_rows_fit(int64_t M, int d1, int d2, int sites, bool second) {
  const MxCut c = mx4_cut(second && M <= kMxBehind ? 2 * M : M, d1, d2, sites);
  const int64_t shrinks = M * sites * mx4_shrink_parts(d1), tiles = (int64_t)sites * c.col_groups * c.row_split * c.parts;
  return shrinks + tiles <= ((int64_t)1 << 22) - 16;  // (a grid has to stay below 2^32 threads)
}

int launch_mx4_rows(const MxArgs& g, int sites, bool gated, void* workspace, hipStream_t st) {
  const int r_max = g.ad.r_max, t_parts = mx4_shrink_parts(g.d1);
  float* const t = (float*)workspace;
  MxTerm* const terms = (MxTerm*)((char*)t + align_up((size_t)g.M * r_max * t_parts * sites * sizeof(float), 256));
  float* const partial = (float*)((char*)terms + align_up((size_t)g.M * sites * sizeof(MxTerm), 256));
  const bool behind = g.second && g.M <= kMxBehind;
  const int rows = behind ? 2 * g.M : g.M;
  MxBase b{};
  b.X = g.X; b.ldx = g.ldx; b.M = rows; b.d1 = g.d1; b.d2 = g.d2;
  for (int s = 0; s < sites; ++s) b.W[s] = g.W[s];
  b.sites = sites;
  const MxCut cut = mx4_cut(rows, g.d1, g.d2, sites);
  const int kw = cut.kw;
  const bool half = cut.half;
  b.parts = cut.parts; b.col_groups = cut.col_groups; b.row_groups = cut.row_groups; b.row_split = cut.row_split;
  b.partial = partial;
  b.shrink = ShrinkArgs{g.X, g.ldx, g.M, 0, g.d1, g.site[0], g.B, g.row_to_req, g.tenant_id, g.route, g.ad, t, (size_t)g.M * r_max, nullptr, nullptr,
                        sites, (size_t)g.M * r_max * t_parts, (size_t)g.M, 0};
  b.second = g.second ? g.X + (size_t)g.M * g.ldx : nullptr;
  b.terms = terms;
  b.shrink_parts = t_parts;
  b.shrink_z = (g.M * sites * t_parts + 7) / 8 * 8;
  const int rc = behind     ? launch_base_of<kBehind>(b, rows, kw, half, st)
                 : g.second ? launch_base_of<kPlanes>(b, rows, kw, half, st)
                            : launch_base_of<kNone>(b, rows, kw, half, st);
  if (rc) return rc;
  MxFinish f{g, b.parts, rows, partial, t, (size_t)g.M * r_max, (size_t)g.M * r_max * t_parts, t_parts, terms};
  const dim3 grid((unsigned)((g.d2 + kFinCols - 1) / kFinCols), (unsigned)g.M, gated ? 1 : sites);
  if (gated) hipLaunchKernelGGL(mx4_finish_kernel<true>, grid, dim3(kFinT), 0, st, f);
  else hipLaunchKernelGGL(mx4_finish_kernel<false>, grid, dim3(kFinT), 0, st, f);
  return check_launch();
}

}  // namespace milora

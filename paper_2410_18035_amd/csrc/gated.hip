// The gated block of a layer with the LoRA terms of its two sites (paper Sec. 3.1, Eq. 1): g = X W_gate + [routed] (X A4) B4,
// u = X W_up + [routed] (X A5) B5, Y = silu(g) u, g and u in fp32 up to the one rounding of Y.  And its backward pass against a frozen base:
//   dg = dY u s (1 + g (1 - s)), du = dY g s, s = 1 / (1 + e^-g)
//   dX = dg W_gate^T + du W_up^T + sum over the two sites of low A^T,  low = dz B^T (routed rows)
//   dA = sum over the tenant's rows of x^T low,  dB = sum of (x A)^T dz
//
// Forward: bf16 takes the matrix-core tiles with gate and up columns side by side (tiles.hip, prefill.hip), 4-bit weights of few rows
// mx4.hip, of more the same tiles, on the codes or on the weights written out in bf16, whichever is reckoned shorter; everything else the
// any-shape kernels of linear_generic.hip.  Backward: the 256 x 256 tiles of prefill.hip for dX, on the codes of 4-bit weights too
// (d % 128 == 0; others are written out first), and the bf16 matrix cores below for dA and dB; everything else the any-shape
// kernels below, fp32 matrix instructions.
#include "gated.h"
#include "mx4.h"
#include "tiles.h"

namespace milora {

// prefill.hip
bool prefill_supported(int64_t M, int d1, int d2, const void* X, const void* W, const void* Y);
int launch_shrink_sites(const bf16_t* X, int64_t ldx, int64_t M, int d1, const int32_t* row_to_req, const AdapterView& ad, int site, int sites,
                        const int32_t* tenant_id, const uint8_t* route, int B, float* t, int2* row_lora, int* clear, hipStream_t stream);
int launch_low_sites(const bf16_t* dz, int64_t M, int F, const int32_t* row_to_req, const AdapterView& ad, const int32_t* tenant_id,
                     const uint8_t* route, int B, float* low, hipStream_t stream);

namespace {

constexpr int kGate = 4;  // site; the up projection's is the next
constexpr int kThreads = 256;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
static_assert(kThreads * 8 == 2048, "columns of gated_dz8_kernel");

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// What of a workspace a call needs, in the order of its calls.
struct Carver {
  char* base;
  size_t off = 0;
  template <typename T>
  T* take(size_t n) {
    T* const p = (T*)(base + off);
    off += align_up(n * sizeof(T), 256);
    return p;
  }
};

// The scales of the ranks (X W^A, dz W^B^T: fp32, [site][part][M][r_max]) as two bf16 halves, about 17 of their bits: zero past the rank and for
// rows without a term.  A row's 32 ranks by 32 lanes.  An Inf or NaN is a high half by itself (its low half would be Inf - Inf); LATER: it becomes zero
// and marks its row, whose products with it the tiles then form in fp32 (where zero columns stand beside those of the site, it would reach them).
constexpr int kHalvesRowsWg = kThreads / 32;
struct HalvesOf {
  const float* v;
  int parts;
  Halves out;
};
template <bool LATER>
__global__ void __launch_bounds__(kThreads) gated_halves_kernel(HalvesOf first, HalvesOf second, size_t part, int64_t M, int r_max, int2* row_lora,
                                                                int sites) {
  const int64_t i = (int64_t)blockIdx.x * kHalvesRowsWg + (threadIdx.x >> 5);  // line
  if (i > M) return;
  const bool other = (int)blockIdx.z >= sites;
  const float* const v = other ? second.v : first.v;
  const int parts = other ? second.parts : first.parts;
  const Halves out = other ? second.out : first.out;
  const int chunk = blockIdx.y, s = (int)blockIdx.z - (other ? sites : 0), c = chunk * 32 + (threadIdx.x & 31);
  float x = 0.f;
  if (i > 0 && c < (row_lora[s * M + i - 1].y & (kLaterBit - 1))) {
    const float* const q = v + (size_t)s * part * parts + (size_t)(i - 1) * r_max + c;
    for (int p = 0; p < parts; ++p) x += q[p * part];
  }
  if (LATER && !finite_f32(x)) {
    x = 0.f;
    atomicOr(&row_lora[s * M + i - 1].y, kLaterBit);
  }
  const bf16_t hi = f32_to_bf16(x);
  bf16_t* const line = out.at + s * out.site + chunk * out.chunk + (size_t)i * 64 + (threadIdx.x & 31);
  line[0] = hi;
  line[32] = f32_to_bf16(rest_of(x, bf16_to_f32(hi)));
}

// ---- forward ---------------------------------------------------------------------------------------------------------------
}  // namespace

static int launch_halves_of(const HalvesOf& first, const HalvesOf* second, int64_t M, int r_max, int2* row_lora, int sites, bool later, hipStream_t st) {
  const dim3 grid((unsigned)((M + kHalvesRowsWg) / kHalvesRowsWg), (unsigned)((r_max + 31) / 32), (unsigned)(second ? 2 * sites : sites));
  const HalvesOf& other = second ? *second : first;
  if (later) hipLaunchKernelGGL(gated_halves_kernel<true>, grid, dim3(kThreads), 0, st, first, other, (size_t)M * r_max, M, r_max, row_lora, sites);
  else hipLaunchKernelGGL(gated_halves_kernel<false>, grid, dim3(kThreads), 0, st, first, other, (size_t)M * r_max, M, r_max, row_lora, sites);
  return check_launch();
}

int launch_halves(const float* v, int parts, int64_t M, int r_max, int2* row_lora, int sites, const Halves& out, hipStream_t st) {
  return launch_halves_of(HalvesOf{v, parts, out}, nullptr, M, r_max, row_lora, sites, true, st);
}

// (2 F is below 2^31: the entry points refuse larger ones)
static size_t gated_partial_bytes(int64_t M, int d, int F) {
  const size_t parts = partial_bytes_bound(M, d, 2 * F), cut = cut_bytes_bound(M, 2 * (int64_t)((F + 127) / 128) * 128);
  return parts > cut ? parts : cut;
}

size_t gated_workspace_bytes(int64_t M, int d, int F, int dtype, bool mx4, int r_max) {
  size_t most = 0;
  if (dtype == MILORA_BF16) {  // control words, shrinks of both sites, look-ups, partial tiles, 4-bit weights in bf16
    Carver c{nullptr};
    c.take<char>(kStreamCtrlBytes);
    c.take<float>(shrink_rows_bound(M, d, 2) * r_max * 2);
    c.take<int2>((size_t)M * 2);
    c.take<char>(gated_partial_bytes(M, d, F));
    c.take<bf16_t>(halves_of(nullptr, M, r_max).site * 2);
    if (mx4 && M > kMxAlwaysFew) c.take<bf16_t>((size_t)d * F * 2);
    most = c.off;
    if (mx4) {
      const size_t few = mx4_rows_workspace_bytes(M < kMxMostFew ? M : kMxMostFew, d, F, r_max, 2);
      if (M <= kMxAlwaysFew) return few;
      most = few > most ? few : most;
    }
  }
  const size_t any = align_up((size_t)M * r_max * 2 * sizeof(float), 256);  // (bf16 too: whatever the alignment of its tensors)
  return any > most ? any : most;
}

int run_gated(const GatedCall& g, void* Y, float* gate_out, float* up_out, void* workspace, hipStream_t st) {
  const int64_t M = g.M;
  int rc;
  if (g.mx4 && mx4_few_rows(M, g.d, 2 * (int64_t)g.F)) {
    if (!mx4_rows_fit(M, g.d, g.F, 2)) return MILORA_ERANGE;
    MxArgs a{};
    a.X = (const bf16_t*)g.X; a.ldx = g.d; a.M = (int)M; a.d1 = g.d; a.d2 = g.F;
    a.W[0] = (const unsigned char*)g.Wg; a.W[1] = (const unsigned char*)g.Wu; a.Y[0] = (bf16_t*)Y; a.ldy = g.F;
    a.gate_out = gate_out; a.up_out = up_out;
    a.ad = g.ad; a.site[0] = kGate; a.row_to_req = g.row_to_req; a.tenant_id = g.tenant_id; a.route = g.route; a.B = g.B;
    return launch_mx4_rows(a, 2, true, workspace, st);
  }
  const bool packed = g.mx4 && g.d % 64 != 0;  // the layout 4-bit weights are written out in: the row-major tiles take whole 64 of a reduction
  const void* const like = g.mx4 ? (const void*)(uintptr_t)256 : nullptr;  // (in the workspace: aligned)
  const void *Wg = like ? like : g.Wg, *Wu = like ? like : g.Wu;
  const bool small = g.dtype == MILORA_BF16 && g.F < 1 << 30 && tiles_supported(M, g.d, 2 * g.F, packed, g.X, Wg, Y) && aligned16(Wu) && g.F % 16 == 0;
  const bool large = g.dtype == MILORA_BF16 && !packed && M <= kHalvesRows && (uint64_t)g.d * 512u < (1ull << 32) &&  // (offsets of a tile's 256 rows)
                     prefill_supported(M, g.d, g.F, g.X, Wg, Y) && aligned16(Wu);
  if (small || large) {
    Carver c{(char*)workspace};
    char* const ctrl = c.take<char>(kStreamCtrlBytes);
    const int parts = shrink_parts(M, g.d, 2);
    GatedTileArgs a{};
    a.d = g.d; a.F = g.F; a.packed = packed; a.ad = g.ad; a.tenant_id = g.tenant_id; a.route = g.route; a.B = g.B;
    a.t_stride = (size_t)M * g.ad.r_max; a.t_site = a.t_stride * parts; a.parts = parts; a.lora_site = (size_t)M;
    a.cnt = (int*)(ctrl + kTileCtrlOffset);
    float* const t = c.take<float>(shrink_rows_bound(M, g.d, 2) * g.ad.r_max * 2);
    int2* const looked_up = c.take<int2>((size_t)M * 2);
    a.partial = c.take<float>(gated_partial_bytes(M, g.d, g.F) / sizeof(float));
    a.halves = halves_of(nullptr, M, g.ad.r_max);
    a.halves.at = c.take<bf16_t>(a.halves.site * 2);
    // slices of rows where the smaller tiles are the only ones and the call has more than a launch of them takes
    int64_t slice = large || M <= kTileMaxRows ? M : kTileMaxRows;
    TilePlan first = plan_tiles(slice, g.d, 2 * g.F, small, large, true, kCut);
    if (g.mx4 && mx4_prefill_supported(M, g.d, g.F)) {  // the codes themselves by 256 x 256 tiles, unless smaller ones make up for writing them out
      const TilePlan direct = plan_tiles(M, g.d, 2 * g.F, false, true, true, kCutMx4);
      if (direct.time <= first.time + 2 * write_out_time(g.d, g.F)) {
        first = direct;
        slice = M;
        a.mx4 = true;
        Wg = g.Wg;
        Wu = g.Wu;
      }
    }
    if (g.mx4 && !a.mx4) {
      bf16_t* const w = c.take<bf16_t>((size_t)g.d * g.F * 2);
      rc = mx4_dequantize(g.Wg, w, MILORA_BF16, g.d, g.F, packed, st);
      if (!rc) rc = mx4_dequantize(g.Wu, w + (size_t)g.d * g.F, MILORA_BF16, g.d, g.F, packed, st);
      if (rc) return rc;
      Wg = w;
      Wu = w + (size_t)g.d * g.F;
    }
    a.Wg = (const bf16_t*)Wg;
    a.Wu = (const bf16_t*)Wu;
    const bool big = first.shape == kTiles256;
    int2* const row_lora = large && !big ? nullptr : looked_up;
    rc = launch_shrink_sites((const bf16_t*)g.X, g.d, M, g.d, g.row_to_req, g.ad, kGate, 2, g.tenant_id, g.route, g.B, t, row_lora,
                             big || row_lora || first.S > 1 ? a.cnt : nullptr, st);
    if (!rc && big) rc = launch_halves(t, parts, M, g.ad.r_max, looked_up, 2, a.halves, st);
    for (int64_t m0 = 0; m0 < M && !rc; m0 += slice) {
      a.M = M - m0 < slice ? M - m0 : slice;
      a.row_base = m0;
      a.X = (const bf16_t*)g.X + (size_t)m0 * g.d;
      a.Y = (bf16_t*)Y + (size_t)m0 * g.F;
      a.gate_out = gate_out ? gate_out + (size_t)m0 * g.F : nullptr;
      a.up_out = up_out ? up_out + (size_t)m0 * g.F : nullptr;
      a.row_to_req = g.row_to_req ? g.row_to_req + m0 : nullptr;
      a.t = t + (size_t)m0 * g.ad.r_max;
      a.row_lora = row_lora ? row_lora + m0 : nullptr;
      const TilePlan pl = a.M == slice ? first : plan_tiles(a.M, g.d, 2 * g.F, small, large, true, kCut);
      rc = pl.shape == kTiles256 ? gated_prefill(a, st) : gated_tiles(a, pl, st);
    }
    return rc;
  }
  // any shape and type
  if (g.mx4) return MILORA_ERANGE;
  return launch_gated_generic(g.X, M, g.d, g.F, g.dtype, g.row_to_req, g.Wg, g.Wu, g.ad, kGate, g.tenant_id, g.route, g.B, (float*)workspace, Y,
                              gate_out, up_out, st);
}

// ---- backward --------------------------------------------------------------------------------------------------------------
namespace {

// dz = [dg | du], rows of 2 F: a workgroup takes kDzCols columns of a row.
constexpr int kDzCols = 2048;
template <typename T>
__global__ void __launch_bounds__(kThreads) gated_dz_kernel(const T* __restrict__ dy, const float* __restrict__ g, const float* __restrict__ u,
                                                            int F, int pieces, T* __restrict__ dz) {
  const int64_t m = blockIdx.x / pieces;
  const int j0 = blockIdx.x % pieces * kDzCols;
  for (int j = j0 + threadIdx.x; j < F && j < j0 + kDzCols; j += kThreads) {
    const int64_t i = m * F + j;
    const float y = Elem<T>::load(dy, i), gv = g[i], uv = u[i], s = 1.f / (1.f + __expf(-gv));
    T* const row = dz + m * 2 * F;
    Elem<T>::store(row, j, y * uv * s * (1.f + gv * (1.f - s)));
    Elem<T>::store(row, F + j, y * gv * s);
  }
}

// The same eight columns a thread (bf16, F % 8 == 0, 16-byte aligned): bound by HBM, 14 bytes an element.
__global__ void __launch_bounds__(kThreads) gated_dz8_kernel(const bf16_t* __restrict__ dy, const float* __restrict__ g, const float* __restrict__ u,
                                                             int F, int pieces, bf16_t* __restrict__ dz) {
  const int64_t m = blockIdx.x / pieces;
  const int j = blockIdx.x % pieces * kDzCols + threadIdx.x * 8;
  if (j >= F) return;
  const int64_t i = m * F + j;
  const u32x4 y = *(const u32x4*)(dy + i);
  f32x4 gv[2], uv[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    gv[h] = __builtin_nontemporal_load((const f32x4*)(g + i) + h);
    uv[h] = __builtin_nontemporal_load((const f32x4*)(u + i) + h);
  }
  u32x4 dg, du;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a[2], b[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float yv = __uint_as_float(k ? y[e] & 0xffff0000u : y[e] << 16), x = gv[e >> 1][2 * (e & 1) + k], v = uv[e >> 1][2 * (e & 1) + k];
      const float s = 1.f / (1.f + __expf(-x));
      a[k] = yv * v * s * (1.f + x * (1.f - s));
      b[k] = yv * x * s;
    }
    dg[e] = pack_bf16x2(a[0], a[1]);
    du[e] = pack_bf16x2(b[0], b[1]);
  }
  bf16_t* const row = dz + m * 2 * F;
  *(u32x4*)(row + j) = dg;
  *(u32x4*)(row + F + j) = du;
}

template <typename T>
int launch_dz(const void* dY, const float* gate, const float* up, int64_t M, int F, void* dz, hipStream_t st) {
  const int pieces = (F + kDzCols - 1) / kDzCols;
  const int64_t slice = ((int64_t)1 << 23) / pieces;  // rows of a launch: a grid has to stay below 2^32 threads
  if (slice < 1) return MILORA_ERANGE;
  int rc = MILORA_OK;
  for (int64_t m = 0; m < M && !rc; m += slice) {
    const int64_t rows = M - m < slice ? M - m : slice;
    if (sizeof(T) == 2 && F % 8 == 0 && aligned16(dY) && aligned16(gate) && aligned16(up))
      hipLaunchKernelGGL(gated_dz8_kernel, dim3((unsigned)(rows * pieces)), dim3(kThreads), 0, st, (const bf16_t*)dY + m * F, gate + m * F, up + m * F, F,
                         pieces, (bf16_t*)dz + m * 2 * F);
    else
      hipLaunchKernelGGL(gated_dz_kernel<T>, dim3((unsigned)(rows * pieces)), dim3(kThreads), 0, st, (const T*)dY + m * F, gate + m * F, up + m * F, F,
                       pieces, (T*)dz + m * 2 * F);
    rc = check_launch();
  }
  return rc;
}

// Tenant and rank of every row at the two sites, [site][M], and the least and the largest tenant among 64 rows, [site][M / 64].
__global__ void __launch_bounds__(kThreads) gated_rows_kernel(int64_t M, const int32_t* __restrict__ row_to_req, AdapterView ad,
                                                              const int32_t* __restrict__ tenant_id, const uint8_t* __restrict__ route, int B,
                                                              int2* __restrict__ row_lora, int2* __restrict__ among, int* __restrict__ clear) {
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < kShrinkClear; i += kThreads) clear[i] = 0;
  const int64_t m = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t req = m < M ? (row_to_req ? (int64_t)row_to_req[m] : m) : -1;
  for (int s = 0; s < 2; ++s) {
    int tenant = -1;
    const int r = req >= 0 && req < B ? routed_rank(ad, tenant_id, route, (int)req, B, kGate + s, &tenant) : 0;
    if (m < M) row_lora[s * M + m] = int2{r ? tenant : -1, r};
    int lo = r ? tenant : 0x7fffffff, hi = r ? tenant : -1;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int a = __shfl_xor(lo, off, 64), b = __shfl_xor(hi, off, 64);
      lo = a < lo ? a : lo;
      hi = b > hi ? b : hi;
    }
    if ((threadIdx.x & 63) == 0 && m < M) among[s * ((M + 63) / 64) + (m >> 6)] = int2{lo, hi};
  }
}

// low[site][m][c] = sum_j dz[m][site F + j] B[c][j] for the routed rows.  A workgroup takes four rows and four ranks of a site, a wave a quarter of
// the columns, so that eight loads feed sixteen products; rows of different tenants one tenant after the other.  Bound: the caches, which send W^B
// once for four rows (500 rows x 2730 columns, ranks 8 and 20: 15 us; a rank a wave, row by row, 62).
constexpr int kLowU = 4;  // columns of a lane on their way
template <typename T>
__global__ void __launch_bounds__(kThreads) gated_low_kernel(const T* __restrict__ dz, int64_t M, int F, const int2* __restrict__ row_lora, AdapterView ad,
                                                             float* __restrict__ low) {
  __shared__ float red[kThreads / 64][16];
  const int64_t m0 = (int64_t)blockIdx.x * 4;
  const int s = blockIdx.y, c0 = blockIdx.z * 4, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int2 tr[4];
  const T* z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = m0 + i < M ? m0 + i : M - 1;
    tr[i] = m0 + i < M ? row_lora[s * M + m] : int2{-1, 0};
    z[i] = dz + m * 2 * F + (int64_t)s * F;
  }
  const int per = (F + 3) / 4, j_end = (w + 1) * per < F ? (w + 1) * per : F;
#pragma unroll
  for (int first = 0; first < 4; ++first) {
    bool seen = tr[first].y <= c0;  // no such ranks, or done with a row in front
    for (int i = 0; i < first; ++i) seen |= tr[i].x == tr[first].x;
    if (seen) continue;
    const T* const B = (const T*)ad.B[tr[first].x * MILORA_NUM_SITES + kGate + s];
    const int r = tr[first].y;
    const T* b[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) b[c] = B + (size_t)(c0 + c < r ? c0 + c : r - 1) * F;
    float sum[4][4] = {};
    for (int j = w * per + lane; j < j_end; j += 64 * kLowU) {
      float zv[kLowU][4], bv[kLowU][4];
#pragma unroll
      for (int u = 0; u < kLowU; ++u) {
        const int at = j + u * 64 < j_end ? j + u * 64 : j;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          zv[u][i] = Elem<T>::load(z[i], at);
          bv[u][i] = Elem<T>::load(b[i], at);
        }
      }
#pragma unroll
      for (int u = 0; u < kLowU; ++u)
        if (j + u * 64 < j_end)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[i][c] += zv[u][i] * bv[u][c];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        for (int off = 32; off > 0; off >>= 1) sum[i][c] += __shfl_xor(sum[i][c], off, 64);
        if (lane == 0) red[w][i * 4 + c] = sum[i][c];
      }
    __syncthreads();
    if (threadIdx.x < 16) {
      const int i = threadIdx.x >> 2, c = c0 + (threadIdx.x & 3);
      int ten = -1;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k == i) ten = tr[k].x;
      if (ten == tr[first].x && c < r)
        low[((size_t)s * M + m0 + i) * ad.r_max + c] = (red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]);
    }
    __syncthreads();
  }
}

// dX of any shape and type: 64 x 64 tiles, 32 of the reduction (2 F, cut into `parts`) at a time through LDS, the next 32 on their way, fp32 matrix
// instructions; the LoRA part of a row after them, or after the parts' sums have been added by the launch behind.  Bound: the matrix instructions
// (500 rows of 1000 x 2730 in fp32: 90 us and 18 for the sums; the whole reduction by one workgroup, one step at a time, 842; 11 rows of 989 x 3026: 16 and 8 against 715).
constexpr int kNnK = 32, kDxUnits = 1024, kDxParts = 32;  // workgroups of a cut launch, parts of a reduction, at most
__host__ __device__ inline int dx_steps(int F) { return (F + kNnK - 1) / kNnK; }  // of one weight
inline int dx_parts(int64_t M, int d, int F) {
  const int64_t tiles = ((M + 63) / 64) * ((d + 63) / 64), steps = 2 * (int64_t)dx_steps(F);
  int64_t parts = kDxUnits / tiles;
  if (parts > kDxParts) parts = kDxParts;
  if (parts > steps / 4) parts = steps / 4;
  if (parts < 2) return 1;
  const int64_t each = (steps + parts - 1) / parts;
  return (int)((steps + each - 1) / each);
}
// never less for larger sizes
inline size_t dx_partial_floats(int64_t M, int d) {
  const size_t by_units = (size_t)kDxUnits * 64 * 64, by_parts = (size_t)kDxParts * M * d;
  return by_units < by_parts ? by_units : by_parts;
}

template <typename T>
__device__ __forceinline__ float dx_lora(int64_t m, int n, int64_t M, const int2* __restrict__ row_lora, const AdapterView& ad, const float* __restrict__ low,
                                         float v) {
  for (int s = 0; s < 2; ++s) {
    const int2 tr = row_lora[s * M + m];
    if (tr.y == 0) continue;
    const T* const A = (const T*)ad.A[tr.x * MILORA_NUM_SITES + kGate + s] + (size_t)n * tr.y;
    const float* const lw = low + ((size_t)s * M + m) * ad.r_max;
    float sum = 0.f;
    for (int c = 0; c < tr.y; ++c) sum += lw[c] * Elem<T>::load(A, c);
    v += sum;
  }
  return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 4) gated_dx_kernel(const T* __restrict__ dz, int64_t M, int d, int F, const T* __restrict__ Wg,
                                                               const T* __restrict__ Wu, const int2* __restrict__ row_lora, AdapterView ad,
                                                               const float* __restrict__ low, float* __restrict__ partial, T* __restrict__ dX) {
  __shared__ float zs[2][64][kNnK + 1], ws[2][kNnK][64 + 4];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, l32 = lane & 31, lh = lane >> 5;
  const int64_t m0 = (int64_t)blockIdx.y * 64;
  const int n0 = blockIdx.x * 64, wm = w & 1, wn = w >> 1;
  const int half = dx_steps(F), each = (2 * half + (int)gridDim.z - 1) / (int)gridDim.z;
  const int from = blockIdx.z * each, end = from + each < 2 * half ? from + each : 2 * half;
  constexpr int kN = 64 * kNnK / kThreads;
  float z[kN], wv[kN];
  auto ask = [&](int step) __attribute__((always_inline)) {
    const bool up = step >= half;
    const int k0 = (up ? step - half : step) * kNnK;
    const T* const W = up ? Wu : Wg;
    const T* const zr = dz + (up ? F : 0);
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      const int e = tid + u * kThreads, row = e / kNnK, k = k0 + e % kNnK, col = n0 + e % 64, kw = k0 + e / 64;
      z[u] = m0 + row < M && k < F ? Elem<T>::load(zr, (m0 + row) * 2 * F + k) : 0.f;
      wv[u] = col < d && kw < F ? Elem<T>::load(W, (size_t)kw * d + col) : 0.f;
    }
  };
  f32x16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  ask(from);
  for (int step = from, buf = 0; step < end; ++step, buf ^= 1) {
#pragma unroll
    for (int u = 0; u < kN; ++u) {
      const int e = tid + u * kThreads;
      zs[buf][e / kNnK][e % kNnK] = z[u];
      ws[buf][e / 64][e % 64] = wv[u];
    }
    __syncthreads();  // (the buffer written next was read before this)
    if (step + 1 < end) ask(step + 1);
#pragma unroll
    for (int k = 0; k < kNnK; k += 2)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(ws[buf][k + lh][wn * 32 + l32], zs[buf][wm * 32 + l32][k + lh], acc, 0, 0, 0);
  }
  // (lane: row l % 32, registers 4 g .. + 3: columns 8 g + 4 (l / 32) ..)
  const int64_t m = m0 + wm * 32 + l32;
  if (m >= M) return;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int n = n0 + wn * 32 + (e >> 2) * 8 + lh * 4 + (e & 3);
    if (n >= d) continue;
    if (gridDim.z > 1) partial[(blockIdx.z * (size_t)M + m) * d + n] = acc[e];
    else Elem<T>::store(dX, (size_t)m * d + n, dx_lora<T>(m, n, M, row_lora, ad, low, acc[e]));
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) gated_dx_sum_kernel(const float* __restrict__ partial, int parts, int64_t M, int d, const int2* __restrict__ row_lora,
                                                                AdapterView ad, const float* __restrict__ low, T* __restrict__ dX) {
  const int64_t m = blockIdx.y;
  const int n = blockIdx.x * kThreads + threadIdx.x;
  if (n >= d) return;
  const float* const q = partial + (size_t)m * d + n;
  const size_t stride = (size_t)M * d;
  float v = 0.f;
  for (int p = 0; p < parts; p += 4) {
    float x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = q[(p + u < parts ? p + u : p) * stride];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (p + u < parts) v += x[u];
  }
  Elem<T>::store(dX, (size_t)m * d + n, dx_lora<T>(m, n, M, row_lora, ad, low, v));
}

// Gradients of the tenants' matrices: out[col][c] = sum over the tenant's rows m of P[m][col] s[m][c], with (P, s) = (X, low) for dA and
// (dz of the site, x A) for dB.  A workgroup takes 64 columns and 32 ranks of one of the tenant's four matrices; its rows, in order, 32 at a time.
struct GradArgs {
  const void *X, *dz;
  int64_t M;
  int d, F, tiles_a, tiles_b;  // tiles of 64 columns of dA and dB
  const int2 *row_lora, *among;
  AdapterView ad;
  const float *low, *t;  // [site][M][r_max]
  void* const* dA;
  void* const* dB;
};
template <typename T>
__global__ void __launch_bounds__(kThreads) gated_grad_kernel(const GradArgs g) {
  __shared__ float ps[32][64 + 4], ss[32][32 + 4];
  __shared__ int rows[64 + kThreads];
  __shared__ int span[2];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, l32 = lane & 31, lh = lane >> 5;
  const int tile = blockIdx.x % (g.tiles_a + g.tiles_b), c0 = blockIdx.x / (g.tiles_a + g.tiles_b) * 32;
  const int s = blockIdx.y & 1, ten = blockIdx.y >> 1;
  const bool is_b = tile >= g.tiles_a;
  void* const* const table = is_b ? g.dB : g.dA;
  T* const out = table ? (T*)table[ten * MILORA_NUM_SITES + kGate + s] : nullptr;
  const int r = g.ad.rank[ten];
  if (!out || r < 1 || r > g.ad.r_max || c0 >= r) return;
  const int cols = is_b ? g.F : g.d, n0 = (is_b ? tile - g.tiles_a : tile) * 64;
  const T* const P = is_b ? (const T*)g.dz + (int64_t)s * g.F : (const T*)g.X;
  const int64_t ldp = is_b ? 2 * (int64_t)g.F : g.d;
  const float* const sc = (is_b ? g.t : g.low) + (size_t)s * g.M * g.ad.r_max;
  // the first and the last 64 rows that can hold one of the tenant's
  const int blocks = (int)((g.M + 63) / 64);
  if (tid == 0) { span[0] = blocks; span[1] = 0; }
  __syncthreads();
  {
    int first = blocks, end = 0;
    for (int i = tid; i < blocks; i += kThreads) {
      const int2 a = g.among[(size_t)s * blocks + i];
      if (ten < a.x || ten > a.y) continue;
      first = first < i ? first : i;
      end = i + 1;
    }
    if (first < end) {
      atomicMin(&span[0], first);
      atomicMax(&span[1], end);
    }
  }
  __syncthreads();
  const int64_t m_end = (int64_t)span[1] * 64 < g.M ? (int64_t)span[1] * 64 : g.M;
  f32x16 acc;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  int have = 0;
  for (int64_t m0 = (int64_t)span[0] * 64; m0 < m_end || have > 0;) {
    // list the tenant's rows among the next ones, in their order
    while (have < 32 && m0 < m_end) {
      const int64_t m = m0 + tid;
      const bool mine = m < m_end && g.row_lora[s * g.M + m].x == ten;
      const unsigned long long votes = __ballot(mine);
      __shared__ int counts[kThreads / 64];
      if (lane == 0) counts[w] = __popcll(votes);
      __syncthreads();
      int at = have;
      for (int i = 0; i < w; ++i) at += counts[i];
      if (mine) rows[at + __popcll(votes & ((1ull << lane) - 1))] = (int)m;
      for (int i = 0; i < kThreads / 64; ++i) have += counts[i];
      m0 += kThreads;
      __syncthreads();
    }
    if (have == 0) break;
    const int n = have < 32 ? have : 32;
    for (int e = tid; e < 32 * 64; e += kThreads) {
      const int k = e >> 6, col = n0 + (e & 63);
      ps[k][e & 63] = k < n && col < cols ? Elem<T>::load(P, (size_t)rows[k] * ldp + col) : 0.f;
    }
    for (int e = tid; e < 32 * 32; e += kThreads) {
      const int k = e >> 5, c = c0 + (e & 31);
      ss[k][e & 31] = k < n && c < r ? sc[(size_t)rows[k] * g.ad.r_max + c] : 0.f;
    }
    __syncthreads();
    if (w < 2)
#pragma unroll
      for (int k = 0; k < 32; k += 2) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(ss[k + lh][l32], ps[k + lh][w * 32 + l32], acc, 0, 0, 0);
    // the rows that are left move to the front
    int keep = 0;
    if (tid < have - n) keep = rows[n + tid];
    __syncthreads();
    if (tid < have - n) rows[tid] = keep;
    have -= n;
    __syncthreads();
  }
  if (w >= 2) return;
  const int col = n0 + w * 32 + l32;
  if (col >= cols) return;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int c = c0 + (e >> 2) * 8 + lh * 4 + (e & 3);
    if (c < r) Elem<T>::store(out, is_b ? (size_t)c * g.F + col : (size_t)col * r + c, acc[e]);
  }
}

// ---- the same on the bf16 matrix cores -------------------------------------------------------------------------------------
// out[col][c] = sum over the tenant's rows of P[m][col] s[m][c]: a workgroup of kGradW waves takes 64 columns and 32 ranks of one of a
// tenant's matrices, a wave every kGradW-th 64 rows of the call: two waves up to kGradFewRows, so that all workgroups are resident (a training step
// of 4096 x 11008 with 16 / 534 / 1111 rows: 155 / 394 / 567 us, with eight 168 / 407 / 579), eight beyond (5120 x 13824, 8192 rows: 4422 us, with
// two 4448).  A wave lists the tenant's rows among its own and takes 32 of them at a time: their 128 bytes
// of P and of s go through registers (the next 32 rows' are on their way while these are multiplied) into the wave's LDS, and the
// transposing read makes operands of both.  The waves' sums meet in LDS at the end.  Bound: the reads of P (HBM) and s (L2).
struct GradTileArgs {
  const bf16_t *X, *dz;
  int64_t M;
  int d, F, tiles_a, tiles_b;  // tiles of 64 columns
  const int2 *row_lora, *among;
  AdapterView ad;
  Halves low, t;
  void* const* dA;
  void* const* dB;
};
// 16-column pieces (32 bytes) of a 128-byte row k: permuted so that four rows of two pieces, which half a wave reads at once, hit all banks
__device__ __forceinline__ int grad_swz(int k) { return ((k >> 1) & 1) * 2; }

constexpr int64_t kGradFewRows = 2048;
template <int kGradW>
__global__ void __launch_bounds__(kGradW * 64, 4) gated_grad_tile_kernel(const GradTileArgs g) {
  __shared__ __attribute__((aligned(16))) unsigned char lds[kGradW * 8192];
  __shared__ int lists[kGradW][128];
  __shared__ int span[2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int tiles = g.tiles_a + g.tiles_b, tile = blockIdx.x % tiles, chunk = blockIdx.x / tiles, c0 = chunk * 32;
  const int s = blockIdx.y & 1, ten = blockIdx.y >> 1;
  const bool is_b = tile >= g.tiles_a;
  void* const* const table = is_b ? g.dB : g.dA;
  bf16_t* const out = table ? (bf16_t*)table[ten * MILORA_NUM_SITES + kGate + s] : nullptr;
  const int r = g.ad.rank[ten];
  if (!out || r < 1 || r > g.ad.r_max || c0 >= r) return;
  const int cols = is_b ? g.F : g.d, n0 = (is_b ? tile - g.tiles_a : tile) * 64;
  const bf16_t* const P = is_b ? g.dz + (int64_t)s * g.F : g.X;
  const int64_t ldp = is_b ? 2 * (int64_t)g.F : g.d;
  const Halves& half = is_b ? g.t : g.low;
  const bf16_t* const sc = half.at + s * half.site + chunk * half.chunk + 64;  // (behind the zero line)
  const int blocks = (int)((g.M + 63) / 64);
  if (tid == 0) { span[0] = blocks; span[1] = 0; }
  __syncthreads();
  {
    int first = blocks, end = 0;
    for (int i = tid; i < blocks; i += kGradW * 64) {
      const int2 a = g.among[(size_t)s * blocks + i];
      if (ten < a.x || ten > a.y) continue;
      first = first < i ? first : i;
      end = i + 1;
    }
    if (first < end) {
      atomicMin(&span[0], first);
      atomicMax(&span[1], end);
    }
  }
  __syncthreads();
  const int b_end = span[1];
  int blk = span[0] + w;
  int* const list = lists[w];
  unsigned char* const mine = lds + w * 8192;
  const uint32_t mine_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)mine;
  f32x16 acc[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;

  // rows 8 it + lane / 8 of 32, piece lane % 8 of 16 bytes
  const int piece = lane & 7;
  const bool p_in = n0 + piece * 8 < cols;  // (cols % 16 == 0)
  u32x4 pv[4], sv[4];
  auto ask = [&](int n) __attribute__((always_inline)) {  // the first n of the list
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int k = it * 8 + (lane >> 3);
      pv[it] = sv[it] = u32x4{0u, 0u, 0u, 0u};
      if (k < n) {
        const int64_t m = list[k];
        if (p_in) pv[it] = *(const u32x4*)(P + m * ldp + n0 + piece * 8);
        sv[it] = *(const u32x4*)(sc + m * 64 + piece * 8);
      }
    }
  };
  int have = 0;
  // fills the list up to 32 rows or the end; the rows asked for before leave it
  auto next = [&](int drop) __attribute__((always_inline)) {
    if (drop) {
      const int keep = drop + lane < have ? list[drop + lane] : 0;
      __builtin_amdgcn_s_waitcnt(0xc07f);
      asm volatile("" ::: "memory");
      if (drop + lane < have) list[lane] = keep;
      have -= drop;
    }
    while (have < 32 && blk < b_end) {
      const int64_t m = (int64_t)blk * 64 + lane;
      const bool ours = m < g.M && g.row_lora[s * g.M + m].x == ten;
      const unsigned long long votes = __ballot(ours);
      if (ours) list[have + __popcll(votes & ((1ull << lane) - 1))] = (int)m;
      have += __popcll(votes);
      blk += kGradW;
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
    return have < 32 ? have : 32;
  };
  const int k_of = (lane >> 5) * 8 + ((lane & 15) >> 2), col_half = (lane >> 4) & 1;
  auto read_tr = [&](uint32_t base, int ks, int pair) __attribute__((always_inline)) {  // rows 16 ks + 8 (l / 32) .., pieces 2 pair, 2 pair + 1
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    s16x4 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = ks * 16 + k_of + 4 * h;
      v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(base + k * 128 + ((2 * pair + col_half) ^ grad_swz(k)) * 32 + (lane & 3) * 8));
    }
    return __builtin_bit_cast(bf16x8, v);
  };
  int n = next(0);
  if (n) ask(n);
  while (n) {
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int k = it * 8 + (lane >> 3);
      unsigned char* const at = mine + k * 128 + ((piece >> 1) ^ grad_swz(k)) * 32 + (piece & 1) * 16;
      *(u32x4*)at = pv[it];
      *(u32x4*)(at + 4096) = sv[it];
    }
    const int left = next(n);
    if (left) ask(left);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // the wave's own LDS writes
    asm volatile("" ::: "memory");
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const bf16x8 hi = read_tr(mine_at + 4096, ks, 0), lo = read_tr(mine_at + 4096, ks, 1);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bf16x8 p = read_tr(mine_at, ks, j);
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, p, acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, p, acc[j], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
    n = left;
  }
  // (lane: column l % 32, registers 4 q .. + 3: ranks 8 q + 4 (l / 32) ..)
  __syncthreads();
  float* const sums = (float*)lds;  // [wave][rank][64 columns]
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[(w * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3)) * 64 + j * 32 + (lane & 31)] = acc[j][e];
  __syncthreads();
  for (int e = tid; e < 32 * 64; e += kGradW * 64) {
    // dB: columns next to one another are next to one another in memory; dA: ranks
    const int c = is_b ? e >> 6 : e & 31, col = is_b ? e & 63 : e >> 5;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kGradW; ++k) v += sums[(k * 32 + c) * 64 + col];
    if (c0 + c < r && n0 + col < cols) out[is_b ? (size_t)(c0 + c) * g.F + n0 + col : (size_t)(n0 + col) * r + c0 + c] = f32_to_bf16(v);
  }
}

struct BackWs {
  void* dz;        // [M][2 F] dtype
  float* low;      // [2][M][r_max]
  float* t;        // [2][part][M][r_max]
  int2* row_lora;  // [2][M]
  int2* among;     // [2][M / 64]
  void* W;         // 4-bit weights in bf16
  Halves low_halves, t_halves;  // of the bf16 matrix cores
  float* partial;
  int* cnt;        // of cut tiles
  size_t bytes;
};

BackWs carve_back(void* base, int64_t M, int d, int F, int dtype, bool mx4, int r_max) {
  Carver c{(char*)base};
  BackWs w;
  w.dz = c.take<char>((size_t)M * F * 2 * dtype_size(dtype));
  w.low = c.take<float>(shrink_rows_bound(M, F, 2) * r_max * 2);
  w.t = c.take<float>(shrink_rows_bound(M, d, 2) * r_max * 2);
  w.row_lora = c.take<int2>((size_t)M * 2);
  w.among = c.take<int2>((size_t)((M + 63) / 64) * 2);
  w.W = c.take<bf16_t>(mx4 ? (size_t)d * F * 2 : 0);
  const bool tiles = dtype == MILORA_BF16;  // (whatever the other sizes: none may go down when one goes up)
  w.low_halves = w.t_halves = halves_of(nullptr, M, r_max);
  w.low_halves.at = c.take<bf16_t>(tiles ? w.low_halves.site * 2 : 0);
  w.t_halves.at = c.take<bf16_t>(tiles ? w.t_halves.site * 2 : 0);
  const size_t any = dx_partial_floats(M, d), by_tiles = tiles ? back_partial_floats(M, d, F) : 0;
  w.partial = c.take<float>(any > by_tiles ? any : by_tiles);
  w.cnt = c.take<int>(kShrinkClear);
  w.bytes = c.off;
  return w;
}

template <typename T>
int backward_any(const GatedCall& g, const void* dY, const float* gate, const float* up, void* dX, void* const* dA, void* const* dB, const BackWs& w,
                 hipStream_t st) {
  const int64_t M = g.M;
  const int tenants = g.ad.n_tenants;
  int rc = launch_dz<T>(dY, gate, up, M, g.F, w.dz, st);
  if (rc) return rc;
  hipLaunchKernelGGL(gated_rows_kernel, dim3((unsigned)((M + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, M, g.row_to_req, g.ad, g.tenant_id,
                     g.route, g.B, w.row_lora, w.among, w.cnt);
  if ((rc = check_launch())) return rc;
  hipLaunchKernelGGL(gated_low_kernel<T>, dim3((unsigned)((M + 3) / 4), 2, (unsigned)((g.ad.r_max + 3) / 4)), dim3(kThreads), 0, st, (const T*)w.dz, M, g.F, w.row_lora, g.ad, w.low);
  if ((rc = check_launch())) return rc;
  const T *Wg = (const T*)g.Wg, *Wu = (const T*)g.Wu;
  if (g.mx4) {
    Wg = (const T*)w.W;
    Wu = Wg + (size_t)g.d * g.F;
  }
  if (dX) {
    const int parts = dx_parts(M, g.d, g.F);  // (up to kDxUnits tiles where there are several: rows fit a grid's y)
    hipLaunchKernelGGL(gated_dx_kernel<T>, dim3((unsigned)((g.d + 63) / 64), (unsigned)((M + 63) / 64), (unsigned)parts), dim3(kThreads), 0, st,
                       (const T*)w.dz, M, g.d, g.F, Wg, Wu, w.row_lora, g.ad, w.low, w.partial, (T*)dX);
    if ((rc = check_launch())) return rc;
    if (parts > 1) {
      hipLaunchKernelGGL(gated_dx_sum_kernel<T>, dim3((unsigned)((g.d + kThreads - 1) / kThreads), (unsigned)M), dim3(kThreads), 0, st, w.partial, parts, M,
                         g.d, w.row_lora, g.ad, w.low, (T*)dX);
      if ((rc = check_launch())) return rc;
    }
  }
  if (dA || dB) {
    GradArgs a{};
    a.X = g.X; a.dz = w.dz; a.M = M; a.d = g.d; a.F = g.F;
    a.tiles_a = dA ? (g.d + 63) / 64 : 0;
    a.tiles_b = dB ? (g.F + 63) / 64 : 0;
    const int chunks = (g.ad.r_max + 31) / 32;
    a.row_lora = w.row_lora; a.among = w.among; a.ad = g.ad; a.low = w.low; a.t = w.t;
    a.dA = dA; a.dB = dB;
    rc = launch_shrink(g.X, g.d, M, g.d, g.dtype, g.row_to_req, g.ad, kGate, 2, g.tenant_id, g.route, g.B, w.t, st);
    if (rc) return rc;
    hipLaunchKernelGGL(gated_grad_kernel<T>, dim3((unsigned)((a.tiles_a + a.tiles_b) * chunks), (unsigned)(2 * tenants)), dim3(kThreads), 0, st, a);
    rc = check_launch();
  }
  return rc;
}

// (4-bit weights) Does the product behind both projections read the codes?  Scales of 128 inputs are copied four bytes at a time.
bool direct_back(const GatedCall& g) { return g.d % 128 == 0; }

// bf16 of whole 32 of F and d, 16-byte aligned: everything on the bf16 matrix cores.
int backward_tiles(const GatedCall& g, const void* dY, const float* gate, const float* up, void* dX, void* const* dA, void* const* dB, const BackWs& w,
                   hipStream_t st) {
  const int64_t M = g.M;
  const int tenants = g.ad.n_tenants, r_max = g.ad.r_max;
  const bf16_t* const dz = (const bf16_t*)w.dz;
  int rc = launch_dz<bf16_t>(dY, gate, up, M, g.F, w.dz, st);
  if (!rc) rc = launch_low_sites(dz, M, g.F, g.row_to_req, g.ad, g.tenant_id, g.route, g.B, w.low, st);
  if (rc) return rc;
  hipLaunchKernelGGL(gated_rows_kernel, dim3((unsigned)((M + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, M, g.row_to_req, g.ad, g.tenant_id,
                     g.route, g.B, w.row_lora, w.among, w.cnt);
  if ((rc = check_launch())) return rc;
  const int low_parts = shrink_parts(M, g.F, 2);
  const size_t row_floats = (size_t)M * r_max;
  const HalvesOf low{w.low, low_parts, w.low_halves}, t{w.t, shrink_parts(M, g.d, 2), w.t_halves};
  if (dB) {
    rc = launch_shrink_sites((const bf16_t*)g.X, g.d, M, g.d, g.row_to_req, g.ad, kGate, 2, g.tenant_id, g.route, g.B, w.t, nullptr, nullptr, st);
    if (rc) return rc;
  }
  if ((rc = launch_halves_of(low, dB ? &t : nullptr, M, r_max, w.row_lora, 2, false, st))) return rc;
  if (dX) {
    GatedBackArgs a{};
    a.dz = dz; a.M = M; a.d = g.d; a.F = g.F; a.row_to_req = g.row_to_req; a.ad = g.ad; a.tenant_id = g.tenant_id; a.route = g.route; a.B = g.B;
    a.mx4 = g.mx4 && direct_back(g);
    a.Wg = g.mx4 && !a.mx4 ? (const bf16_t*)w.W : (const bf16_t*)g.Wg;
    a.Wu = g.mx4 && !a.mx4 ? (const bf16_t*)w.W + (size_t)g.d * g.F : (const bf16_t*)g.Wu;
    a.row_lora = w.row_lora; a.lora_site = (size_t)M; a.halves = w.low_halves;
    a.low = w.low; a.low_stride = row_floats; a.low_site = row_floats * low_parts; a.parts = low_parts;
    a.partial = w.partial; a.cnt = w.cnt; a.dX = (bf16_t*)dX;
    if ((rc = gated_dx_tiles(a, st))) return rc;
  }
  if (!dA && !dB) return rc;
  const int chunks = (r_max + 31) / 32;
  GradTileArgs a{};
  a.X = (const bf16_t*)g.X; a.dz = dz; a.M = M; a.d = g.d; a.F = g.F;
  a.tiles_a = dA ? (g.d + 63) / 64 : 0;
  a.tiles_b = dB ? (g.F + 63) / 64 : 0;
  a.row_lora = w.row_lora; a.among = w.among; a.ad = g.ad; a.low = w.low_halves; a.t = w.t_halves; a.dA = dA; a.dB = dB;
  const dim3 grid((unsigned)((a.tiles_a + a.tiles_b) * chunks), (unsigned)(2 * tenants));
  if (M <= kGradFewRows) hipLaunchKernelGGL(gated_grad_tile_kernel<2>, grid, dim3(2 * 64), 0, st, a);
  else hipLaunchKernelGGL(gated_grad_tile_kernel<8>, grid, dim3(8 * 64), 0, st, a);
  return check_launch();
}

}  // namespace

size_t gated_backward_workspace_bytes(int64_t M, int d, int F, int dtype, bool mx4, int r_max) {
  return carve_back(nullptr, M, d, F, dtype, mx4, r_max).bytes;
}

int run_gated_backward(const GatedCall& g, const void* dY, const float* gate, const float* up, void* dX, void* const* dA, void* const* dB,
                       void* workspace, hipStream_t st) {
  const BackWs w = carve_back(workspace, g.M, g.d, g.F, g.dtype, g.mx4, g.ad.r_max);
  const bf16_t* const Wg = g.mx4 ? (const bf16_t*)w.W : (const bf16_t*)g.Wg;
  const bf16_t* const Wu = g.mx4 ? Wg + (size_t)g.d * g.F : (const bf16_t*)g.Wu;
  if (g.M > (int64_t)65535 * 64 || g.ad.n_tenants > 32767) return MILORA_ERANGE;
  const bool tiles = g.dtype == MILORA_BF16 && g.d % 32 == 0 && aligned16(g.X) &&
                     back_supported(g.M, g.d, g.F, w.dz, Wg, Wu, dX);
  if (g.mx4 && dX && !(tiles && direct_back(g))) {
    int rc = mx4_dequantize(g.Wg, w.W, MILORA_BF16, g.d, g.F, false, st);
    if (!rc) rc = mx4_dequantize(g.Wu, (bf16_t*)w.W + (size_t)g.d * g.F, MILORA_BF16, g.d, g.F, false, st);
    if (rc) return rc;
  }
  if (tiles)
    return backward_tiles(g, dY, gate, up, dX, dA, dB, w, st);
  return g.dtype == MILORA_BF16 ? backward_any<bf16_t>(g, dY, gate, up, dX, dA, dB, w, st) : backward_any<float>(g, dY, gate, up, dX, dA, dB, w, st);
}

}  // namespace milora

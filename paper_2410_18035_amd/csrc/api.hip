// C ABI of the routed-LoRA library: argument validation, workspace carving and dispatch between
// the decode kernels (bf16, packed weights), the matrix-core tiles (bf16, row-major weights or packed ones
// of many rows) and the any-shape path (fp32 and everything else).
#include "gated.h"
#include "mx4.h"
#include "tiles.h"

namespace milora {

thread_local int g_last_hip_error = 0;

// decode.hip
size_t decode_packed_workspace_bytes(int M, int d, int F, int r_max);
int layer_decode_packed(const bf16_t* x, int B, int d, int F, const milora_layer_weights* wts, const AdapterView& ad,
                        const int32_t* tenant_id, const uint8_t* route, uint32_t flags, const bf16_t* attn_out,
                        bf16_t* y, bf16_t* qkv_out, void* workspace, hipStream_t st, LaunchMarks* marks);
int routed_linear_packed(const bf16_t* X, int M, int d1, int d2, const int32_t* row_to_req, const bf16_t* W,
                         const bf16_t* bias, const AdapterView& ad, int site, const int32_t* tenant_id,
                         const uint8_t* route, int B, bf16_t* Y, void* workspace, hipStream_t st);
size_t routed_linear_packed_workspace_bytes(int M, int d1, int d2, int r_max);
int pack_weight(const void* src, void* dst, int d1, int d2, hipStream_t st);
int set_wait_limit(int polls);
size_t decode_trace_bytes();
int decode_trace_dims(int* stages_max, int* waves, int* slots);
int layer_decode_packed_static(const bf16_t* x, int B, int d, int F, const milora_layer_weights* wts, const AdapterView& ad,
                               const int32_t* tenant_id, const uint8_t* route, uint32_t flags, const bf16_t* attn_out,
                               bf16_t* y, bf16_t* qkv_out, hipStream_t st);
int static_scratch_status(int* status, hipStream_t st);
// prefill.hip
int decode_workspace_status(const void* workspace, int* status, hipStream_t st);
bool prefill_supported(int64_t M, int d1, int d2, const void* X, const void* W, const void* Y);
int launch_shrink_tiles(const bf16_t* X, int64_t M, int d1, const int32_t* row_to_req, const AdapterView& ad, int site,
                        const int32_t* tenant_id, const uint8_t* route, int B, float* t, int2* row_lora, int* clear,
                        hipStream_t stream);
int launch_shrink_sites(const bf16_t* X, int64_t ldx, int64_t M, int d1, const int32_t* row_to_req, const AdapterView& ad, int site, int sites,
                        const int32_t* tenant_id, const uint8_t* route, int B, float* t, int2* row_lora, int* clear, hipStream_t stream);
int routed_linear_prefill(const bf16_t* X, int64_t M, int d1, int d2, const int32_t* row_to_req, const bf16_t* W,
                          const bf16_t* bias, const AdapterView& ad, int site, const int32_t* tenant_id,
                          const uint8_t* route, int B, const float* t, bf16_t* Y, hipStream_t st);

namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float block_sum(float v, float* sh) {
  for (int off = 32; off > 0; off >>= 1) v += __shfl_down(v, off, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < kThreads / 64; ++w) s += sh[w];
  __syncthreads();
  return s;
}

// out[m] = T(n(in[m])) with n = weightless RMS normalisation (one workgroup per row).
template <typename Tin, typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_rows_kernel(const Tin* __restrict__ in, int d, T* __restrict__ out) {
  __shared__ float sh[kThreads / 64];
  const size_t m = blockIdx.x;
  float ss = 0.f;
  for (int i = threadIdx.x; i < d; i += kThreads) {
    const float v = Elem<Tin>::load(in, m * d + i);
    ss += v * v;
  }
  const float inv = rsqrtf(block_sum<T>(ss, sh) / (float)d + 1e-5f);
  for (int i = threadIdx.x; i < d; i += kThreads) Elem<T>::store(out, m * d + i, Elem<Tin>::load(in, m * d + i) * inv);
}

// h = x + o in fp32; hn = T(n(h)) or T(h).
template <typename T>
__global__ void __launch_bounds__(kThreads) resid_norm_kernel(const T* __restrict__ x, const T* __restrict__ o, int d,
                                                              int norm, float* __restrict__ h, T* __restrict__ hn) {
  __shared__ float sh[kThreads / 64];
  const size_t m = blockIdx.x;
  float ss = 0.f;
  for (int i = threadIdx.x; i < d; i += kThreads) {
    const float v = Elem<T>::load(x, m * d + i) + Elem<T>::load(o, m * d + i);
    h[m * d + i] = v;
    ss += v * v;
  }
  const float tot = block_sum<T>(ss, sh);
  const float inv = norm ? rsqrtf(tot / (float)d + 1e-5f) : 1.f;
  for (int i = threadIdx.x; i < d; i += kThreads) Elem<T>::store(hn, m * d + i, h[m * d + i] * inv);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) silu_mul_kernel(const T* __restrict__ g, const T* __restrict__ u, size_t n,
                                                            T* __restrict__ out) {
  const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) Elem<T>::store(out, i, silu(Elem<T>::load(g, i)) * Elem<T>::load(u, i));
}

template <typename T>
__global__ void __launch_bounds__(kThreads) add_f32_kernel(const float* __restrict__ h, const T* __restrict__ dn, size_t n,
                                                           T* __restrict__ y) {
  const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) Elem<T>::store(y, i, h[i] + Elem<T>::load(dn, i));
}

template <typename T>
__global__ void __launch_bounds__(kThreads) interleave_qkv_kernel(const T* __restrict__ qkv3, int B, int d, T* __restrict__ out) {
  const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
  const size_t n = (size_t)3 * B * d;
  if (i >= n) return;
  const size_t s = i / ((size_t)B * d), rem = i % ((size_t)B * d);
  const size_t b = rem / d, c = rem % d;
  out[(b * 3 + s) * d + c] = qkv3[i];
}

// Workspace of the any-shape layer path.
struct GenericWs {
  float* t;   // [3][B][r_max]
  float* h;   // [B][d]
  char* xn;   // [B][d]   T
  char* qkv;  // [3][B][d] T
  char* o;    // [B][d]   T
  char* hn;   // [B][d]   T
  char* g;    // [B][F]   T
  char* u;    // [B][F]   T
  char* mm;   // [B][F]   T
  char* dn;   // [B][d]   T
  size_t bytes;
};

GenericWs carve_generic(void* base, int B, int d, int F, int r_max, size_t es) {
  size_t off = 0;
  auto take = [&](size_t n) { size_t o = off; off += align_up(n, 256); return o; };
  char* b = (char*)base;
  GenericWs w;
  w.t = (float*)(b + take((size_t)3 * B * r_max * 4));
  w.h = (float*)(b + take((size_t)B * d * 4));
  w.xn = b + take((size_t)B * d * es);
  w.qkv = b + take((size_t)3 * B * d * es);
  w.o = b + take((size_t)B * d * es);
  w.hn = b + take((size_t)B * d * es);
  w.g = b + take((size_t)B * F * es);
  w.u = b + take((size_t)B * F * es);
  w.mm = b + take((size_t)B * F * es);
  w.dn = b + take((size_t)B * d * es);
  w.bytes = off;
  return w;
}

// Up to kFewRows rows: four launches with the glue in their stores (two more with normalisation).
template <typename T>
int layer_decode_few(const void* x, int B, int d, int F, int dtype, const milora_layer_weights* wts, const AdapterView& ad,
                     const int32_t* tenant_id, const uint8_t* route, int norm, const void* attn_out, void* y, void* qkv_out,
                     const GenericWs& w, hipStream_t st) {
  int rc;
  FewArgs g{};
  g.M = g.B = B;
  g.tenant_id = tenant_id;
  g.route = route;
  g.ad = ad;
  auto run = [&](int site0, int sites, int mode, const void* in, int64_t ldx) {
    g.X = in;
    g.ldx = ldx;
    site_dims(site0, d, F, &g.d1, &g.d2);
    for (int s = 0; s < sites; ++s) { g.site[s] = site0 + s; g.W[s] = wts->W[site0 + s]; }
    return launch_few_rows(g, dtype, sites, mode, w.t, st);
  };
  const void* xin = x;
  if (norm) {
    hipLaunchKernelGGL((rmsnorm_rows_kernel<T, T>), dim3(B), dim3(kThreads), 0, st, (const T*)x, d, (T*)w.xn);
    if ((rc = check_launch())) return rc;
    xin = w.xn;
  }
  T* const qkv = qkv_out ? (T*)qkv_out : (T*)w.qkv;  // [B][3 d]
  for (int s = 0; s < 3; ++s) g.Y[s] = qkv + (size_t)s * d;
  g.ldy = 3 * (int64_t)d;
  if ((rc = run(0, 3, kFewPlain, xin, d))) return rc;
  const bool h_is_input = !norm && sizeof(T) == 4;
  g.x_res = x;
  g.h = w.h;
  g.Y[0] = norm || h_is_input ? nullptr : w.hn;
  rc = attn_out ? run(3, 1, kFewResid, attn_out, d) : run(3, 1, kFewResid, qkv + 2 * (size_t)d, 3 * (int64_t)d);
  if (rc) return rc;
  if (norm) {
    hipLaunchKernelGGL((rmsnorm_rows_kernel<float, T>), dim3(B), dim3(kThreads), 0, st, w.h, d, (T*)w.hn);
    if ((rc = check_launch())) return rc;
  }
  g.Y[0] = w.mm;
  g.ldy = F;
  if ((rc = run(4, 2, kFewGateUp, h_is_input ? (const void*)w.h : (const void*)w.hn, d))) return rc;
  g.Y[0] = y;
  return run(6, 1, kFewDown, w.mm, F);
}

template <typename T>
int layer_decode_generic(const void* x, int B, int d, int F, int dtype, const milora_layer_weights* wts,
                         const AdapterView& ad, const int32_t* tenant_id, const uint8_t* route, uint32_t flags,
                         const void* attn_out, void* y, void* qkv_out, void* workspace, hipStream_t st) {
  GenericWs w = carve_generic(workspace, B, d, F, ad.r_max, sizeof(T));
  const int norm = (flags & MILORA_LAYER_RMSNORM) ? 1 : 0;
  if (B <= kFewRows)
    return layer_decode_few<T>(x, B, d, F, dtype, wts, ad, tenant_id, route, norm, attn_out, y, qkv_out, w, st);
  int rc;
  auto lin = [&](const void* in, int site, void* out) -> int {
    int d1, d2;
    site_dims(site, d, F, &d1, &d2);
    return launch_linear_generic(in, B, d1, d2, dtype, nullptr, wts->W[site], nullptr, ad, site, tenant_id, route, B,
                                 w.t, out, st);
  };
  const void* xin = x;
  if (norm) {
    hipLaunchKernelGGL((rmsnorm_rows_kernel<T, T>), dim3(B), dim3(kThreads), 0, st, (const T*)x, d, (T*)w.xn);
    if ((rc = check_launch())) return rc;
    xin = w.xn;
  }
  T* q3 = (T*)w.qkv;
  for (int s = 0; s < 3; ++s)
    if ((rc = lin(xin, s, q3 + (size_t)s * B * d))) return rc;
  if (qkv_out) {
    const size_t n = (size_t)3 * B * d;
    hipLaunchKernelGGL(interleave_qkv_kernel<T>, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, st,
                       (const T*)q3, B, d, (T*)qkv_out);
    if ((rc = check_launch())) return rc;
  }
  const void* a = attn_out ? attn_out : (const void*)(q3 + (size_t)2 * B * d);
  if ((rc = lin(a, 3, w.o))) return rc;
  hipLaunchKernelGGL(resid_norm_kernel<T>, dim3(B), dim3(kThreads), 0, st, (const T*)x, (const T*)w.o, d, norm, w.h,
                     (T*)w.hn);
  if ((rc = check_launch())) return rc;
  if ((rc = lin(w.hn, 4, w.g))) return rc;
  if ((rc = lin(w.hn, 5, w.u))) return rc;
  const size_t nF = (size_t)B * F, nd = (size_t)B * d;
  hipLaunchKernelGGL(silu_mul_kernel<T>, dim3((unsigned)((nF + kThreads - 1) / kThreads)), dim3(kThreads), 0, st,
                     (const T*)w.g, (const T*)w.u, nF, (T*)w.mm);
  if ((rc = check_launch())) return rc;
  if ((rc = lin(w.mm, 6, w.dn))) return rc;
  hipLaunchKernelGGL(add_f32_kernel<T>, dim3((unsigned)((nd + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, w.h,
                     (const T*)w.dn, nd, (T*)y);
  return check_launch();
}

// ---- a decode step on 4-bit weights: two launches a level, the glue in the second ----
struct MxLayerWs {
  float* h;     // [B][d]
  bf16_t* qkv;  // [B][3 d]
  bf16_t* hn;   // [2][B][d]: h as two bf16 values, rounded and the rest (16 bits of it)
  bf16_t* mm;   // [B][F]
  char* level;  // workspace of a level
  size_t bytes;
};

MxLayerWs carve_mx4(void* base, int B, int d, int F, int r_max) {
  size_t off = 0;
  auto take = [&](size_t n) { size_t o = off; off += align_up(n, 256); return o; };
  char* b = (char*)base;
  MxLayerWs w;
  w.h = (float*)(b + take((size_t)B * d * 4));
  w.qkv = (bf16_t*)(b + take((size_t)B * d * 6));
  w.hn = (bf16_t*)(b + take((size_t)B * d * 4));
  w.mm = (bf16_t*)(b + take((size_t)B * F * 2));
  size_t level = 0;
  const struct { int d1, d2, sites; } levels[4] = {{d, d, 3}, {d, d, 1}, {d, F, 2}, {F, d, 1}};
  for (const auto& l : levels) {
    const size_t n = mx4_rows_workspace_bytes(B, l.d1, l.d2, r_max, l.sites, l.sites == 2);
    level = n > level ? n : level;
  }
  w.level = b + take(level);
  w.bytes = off;
  return w;
}

int layer_decode_mx4(const bf16_t* x, int B, int d, int F, const milora_layer_weights* wts, const AdapterView& ad, const int32_t* tenant_id,
                     const uint8_t* route, uint32_t flags, const bf16_t* attn_out, bf16_t* y, bf16_t* qkv_out, void* workspace, hipStream_t st) {
  const MxLayerWs w = carve_mx4(workspace, B, d, F, ad.r_max);
  const bool norm = (flags & MILORA_LAYER_RMSNORM) != 0;
  MxArgs g{};
  g.M = g.B = B; g.ad = ad; g.tenant_id = tenant_id; g.route = route;
  // level of `sites` linears from site0 on
  auto level = [&](int site0, int sites, const bf16_t* in, int64_t ldx, bool gated, int64_t ldy) {
    site_dims(site0, d, F, &g.d1, &g.d2);
    g.X = in; g.ldx = ldx; g.ldy = ldy;
    for (int s = 0; s < sites; ++s) { g.site[s] = site0 + s; g.W[s] = (const unsigned char*)wts->W[site0 + s]; }
    return launch_mx4_rows(g, sites, gated, w.level, st);
  };
  bf16_t* const qkv = qkv_out ? qkv_out : w.qkv;
  for (int s = 0; s < 3; ++s) g.Y[s] = qkv + (size_t)s * d;
  g.norm_x = norm ? x : nullptr;
  int rc = level(0, 3, x, d, false, 3 * (int64_t)d);
  if (rc) return rc;
  g.norm_x = nullptr;
  g.Y[0] = w.hn;
  g.res = x;
  g.h_out = w.h;
  g.left_out = w.hn + (size_t)B * d;
  if ((rc = attn_out ? level(3, 1, attn_out, d, false, d) : level(3, 1, qkv + 2 * (size_t)d, 3 * (int64_t)d, false, d))) return rc;
  g.res = nullptr;
  g.left_out = nullptr;
  g.Y[0] = w.mm;
  g.norm_h = norm ? w.h : nullptr;
  g.second = true;
  if ((rc = level(4, 2, w.hn, d, true, F))) return rc;
  g.second = false;
  g.norm_h = nullptr;
  g.Y[0] = y;
  g.h_in = w.h;
  return level(6, 1, w.mm, F, false, d);
}

bool valid_dtype(int dt) { return dt == MILORA_BF16 || dt == MILORA_F32; }
bool valid_layout(int l) { return l == MILORA_W_ROWMAJOR || l == MILORA_W_PACKED || l == MILORA_W_MX4; }

int check_adapters(const milora_adapters* a) {
  if (!a || !a->rank || !a->A || !a->B) return MILORA_EINVAL;
  if (a->n_tenants < 1 || a->r_max < 1) return MILORA_EINVAL;
  if (a->r_max > MILORA_MAX_RANK) return MILORA_ERANGE;
  return MILORA_OK;
}

// How milora_routed_linear serves a call whose arguments it has accepted.
struct LinearPlan {
  int kind;        // MILORA_KERNEL_GENERIC, MILORA_KERNEL_STREAM, or MILORA_KERNEL_TILES: matrix-core tiles of any size
  bool small, large;
  int64_t slice;   // rows of a launch of the tiles
  TilePlan tiles;  // of the first slice
};

LinearPlan plan_linear(int64_t M, int d1, int d2, int dtype, bool packed, const void* X, const void* W, const void* Y) {
  LinearPlan p{MILORA_KERNEL_GENERIC, false, false, M, TilePlan{}};
  if (dtype != MILORA_BF16) return p;
  p.small = tiles_supported(M, d1, d2, packed, X, W, Y);
  p.large = !packed && prefill_supported(M, d1, d2, X, W, Y);
  if (packed && (M <= kStreamRows || !p.small)) {
    p.kind = MILORA_KERNEL_STREAM;
  } else if (p.small || p.large) {
    p.kind = MILORA_KERNEL_TILES;
    // more rows than a launch of the smaller tiles takes, and no larger ones for this weight: slices of rows
    if (!p.large && M > kTileMaxRows) p.slice = kTileMaxRows;
    p.tiles = plan_tiles(p.slice, d1, d2, p.small, p.large);
  }
  return p;
}

bool packed_shape_ok(int d1, int d2) { return d1 % 32 == 0 && d2 % 16 == 0; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// A call whose arguments have been accepted.
int run_linear(const void* X, int64_t M, int d1, int d2, int dtype, const int32_t* row_to_req, const void* W, bool packed,
               const void* bias, const AdapterView& ad, int site, const int32_t* tenant_id, const uint8_t* route, int B, void* Y,
               void* workspace, hipStream_t st) {
  int rc = MILORA_OK;
  const LinearPlan pl = plan_linear(M, d1, d2, dtype, packed, X, W, Y);
  if (pl.kind == MILORA_KERNEL_STREAM)
    // (more rows on reductions too long for the tiles: rows are independent, slices of them each read W again)
    for (int64_t m0 = 0;; m0 += kStreamRows) {
      const int mc = (int)(M - m0 < kStreamRows ? M - m0 : kStreamRows);
      const int64_t b0 = row_to_req ? 0 : m0;  // (unmapped rows: the slice's requests)
      rc = routed_linear_packed((const bf16_t*)X + m0 * d1, mc, d1, d2, row_to_req ? row_to_req + m0 : nullptr,
                                (const bf16_t*)W, (const bf16_t*)bias, ad, site, tenant_id + b0, route + b0, (int)(B - b0),
                                (bf16_t*)Y + m0 * d2, workspace, st);
      if (rc || m0 + mc >= M) return rc;
    }
  int* const cnt = (int*)((char*)workspace + kTileCtrlOffset);
  float* const t = (float*)((char*)workspace + kStreamCtrlBytes);
  if (pl.kind == MILORA_KERNEL_TILES) {
    const int parts = shrink_parts(M, d1);
    const size_t t_stride = (size_t)M * ad.r_max;
    int2* const looked_up = (int2*)((char*)t + align_up(t_stride * sizeof(float) * parts, 256));
    float* const partial = (float*)((char*)looked_up + align_up((size_t)M * sizeof(int2), 256));
    // Where the 256 x 256 kernel is no choice, the LoRA term is added in fp32 row by row: few rows and packed weights, where many
    // tenants meet, and weights beyond that kernel's offsets.
    int2* const row_lora = pl.large ? nullptr : looked_up;
    // Part counters start from zero in every call: what the workspace held before does not matter here.
    int* const clear = row_lora || pl.tiles.S > 1 ? cnt : nullptr;
    rc = launch_shrink_tiles((const bf16_t*)X, M, d1, row_to_req, ad, site, tenant_id, route, B, t, row_lora, clear, st);
    for (int64_t m0 = 0; m0 < M && !rc; m0 += pl.slice) {
      const int64_t mc = M - m0 < pl.slice ? M - m0 : pl.slice;
      const TilePlan tiles = mc == pl.slice ? pl.tiles : plan_tiles(mc, d1, d2, pl.small, pl.large);
      const bf16_t* const x = (const bf16_t*)X + (size_t)m0 * d1;
      bf16_t* const y = (bf16_t*)Y + (size_t)m0 * d2;
      const int32_t* const map = row_to_req ? row_to_req + m0 : nullptr;
      if (tiles.shape == kTiles256)
        rc = routed_linear_prefill(x, mc, d1, d2, map, (const bf16_t*)W, (const bf16_t*)bias, ad, site, tenant_id, route, B, t, y, st);
      else
        rc = routed_linear_tiles(x, mc, d1, d2, map, (const bf16_t*)W, packed, row_lora ? row_lora + m0 : nullptr,
                                 (const bf16_t*)bias, ad, site, tenant_id, route, B, t + (size_t)m0 * ad.r_max, t_stride, parts,
                                 tiles, cnt, partial, y, st);
    }
    return rc;
  }
  return launch_linear_generic(X, M, d1, d2, dtype, row_to_req, W, bias, ad, site, tenant_id, route, B, t, Y, st);
}

// ---- 4-bit weights ----
// Few rows: the kernels of mx4.hip multiply the codes.  More: 256 x 256 tiles do, or the weight is written out in bf16 once per call, row-major or,
// where the row-major tiles do not take its reduction, packed.
bool mx4_rowmajor(int d1) { return d1 % 64 == 0; }  // the layout a weight is written out in

// Do 256 x 256 tiles multiply the codes themselves?  Unless other tiles (pl) make up for writing the weight out.
bool mx4_linear_direct(int64_t M, int d1, int d2, const LinearPlan& pl) {
  if (!mx4_prefill_supported(M, d1, d2)) return false;
  const int64_t other = pl.kind == MILORA_KERNEL_TILES && pl.slice == M ? pl.tiles.time : INT64_MAX / 2;
  return plan_tiles(M, d1, d2, false, true, false, kCutMx4).time <= other + write_out_time(d1, d2);
}

// Is there a kernel for these sizes?  Not where only the weight-streaming kernel would be left for the weight written out (packed, reductions too long
// or columns too many for the tiles): its hand-over words have to be zero before their first use, which a workspace of any contents does not
// promise.  Nor where the rows of one large tile are beyond the offsets.
bool mx4_linear_fits(int64_t M, int d1, int d2) {
  if (mx4_few_rows(M, d1, d2)) return mx4_rows_fit(M, d1, d2, 1);
  const void* aligned = (const void*)(uintptr_t)256;
  const LinearPlan pl = plan_linear(M, d1, d2, MILORA_BF16, !mx4_rowmajor(d1), aligned, aligned, aligned);
  return mx4_linear_direct(M, d1, d2, pl) || (pl.kind != MILORA_KERNEL_STREAM && !(pl.large && !pl.small && (uint64_t)d1 * 512u >= (1ull << 32)));
}

int run_linear_mx4(const bf16_t* X, int64_t M, int d1, int d2, const int32_t* row_to_req, const void* W, const bf16_t* bias,
                   const AdapterView& ad, int site, const int32_t* tenant_id, const uint8_t* route, int B, bf16_t* Y, void* workspace,
                   hipStream_t st) {
  if (mx4_few_rows(M, d1, d2)) {
    MxArgs g{};
    g.X = X; g.ldx = d1; g.M = (int)M; g.d1 = d1; g.d2 = d2; g.W[0] = (const unsigned char*)W; g.bias = bias; g.Y[0] = Y; g.ldy = d2;
    g.ad = ad; g.site[0] = site; g.row_to_req = row_to_req; g.tenant_id = tenant_id; g.route = route; g.B = B;
    return launch_mx4_rows(g, 1, false, workspace, st);
  }
  const bool packed = !mx4_rowmajor(d1);
  const LinearPlan pl = plan_linear(M, d1, d2, MILORA_BF16, packed, X, (const void*)(uintptr_t)256, Y);
  if (mx4_linear_direct(M, d1, d2, pl)) {
    GatedTileArgs a{};
    const int parts = shrink_parts(M, d1);
    float* const t = (float*)((char*)workspace + kStreamCtrlBytes);
    int2* const looked_up = (int2*)((char*)t + align_up((size_t)M * ad.r_max * parts * sizeof(float), 256));
    a.X = X; a.M = M; a.d = d1; a.F = d2; a.row_to_req = row_to_req; a.Wg = (const bf16_t*)W; a.mx4 = true;
    a.row_lora = looked_up; a.lora_site = (size_t)M; a.halves = halves_of(nullptr, M, ad.r_max);
    a.halves.at = (bf16_t*)((char*)looked_up + align_up((size_t)M * sizeof(int2), 256));
    a.ad = ad; a.tenant_id = tenant_id; a.route = route; a.B = B; a.t = t; a.t_stride = (size_t)M * ad.r_max; a.t_site = a.t_stride * parts; a.parts = parts;
    a.Y = Y;
    a.cnt = (int*)((char*)workspace + kTileCtrlOffset);
    a.partial = (float*)((char*)a.halves.at + align_up(a.halves.site * sizeof(bf16_t), 256));
    int rc = launch_shrink_sites(X, d1, M, d1, row_to_req, ad, site, 1, tenant_id, route, B, t, looked_up, a.cnt, st);
    if (!rc) rc = launch_halves(t, parts, M, ad.r_max, looked_up, 1, a.halves, st);
    return rc ? rc : linear_prefill_mx4(a, bias, site, st);
  }
  const int rc = mx4_dequantize(W, workspace, MILORA_BF16, d1, d2, packed, st);
  if (rc) return rc;
  return run_linear(X, M, d1, d2, MILORA_BF16, row_to_req, workspace, packed, bias, ad, site, tenant_id, route, B, Y,
                    (char*)workspace + align_up((size_t)d1 * d2 * 2, 256), st);
}

}  // namespace
}  // namespace milora

using namespace milora;

extern "C" const char* milora_version(void) { return "milora-mi355x 0.1 (gfx950)"; }

extern "C" const char* milora_status_string(int status) {
  switch (status) {
    case MILORA_OK: return "ok";
    case MILORA_EINVAL: return "invalid argument";
    case MILORA_ERANGE: return "size beyond a documented limit";
    case MILORA_EUNSUPPORTED: return "combination not supported";
    case MILORA_EHIP: return "HIP call failed";
    case MILORA_EWORKSPACE: return "workspace missing or too small";
    default: return "unknown status";
  }
}

extern "C" int milora_last_hip_error(void) { return g_last_hip_error; }

extern "C" size_t milora_routed_linear_workspace_bytes(int64_t M, int d1, int d2, int r_max) {
  if (M < 1 || d1 < 1 || d2 < 1 || r_max < 1) return 0;
  // Control words, LoRA shrinks, the rows' look-ups, partial tiles.  What a call needs of shrinks and tiles goes up and down with M (fewer rows are cut
  // into more parts); a caller sizes once for the largest call, so each is bounded by something that no size lowers.
  const size_t t_bytes = align_up(shrink_rows_bound(M, d1) * r_max * sizeof(float), 256);
  const size_t tiles = kStreamCtrlBytes + t_bytes + align_up((size_t)M * sizeof(int2), 256) + partial_bytes_bound(M, d1, d2);
  const size_t packed = routed_linear_packed_workspace_bytes(M <= kStreamRows ? (int)M : kStreamRows, d1, d2, r_max);
  return tiles > packed ? tiles : packed;
}

extern "C" size_t milora_quantized_linear_workspace_bytes(int64_t M, int d1, int d2, int r_max) {
  if (M < 1 || d1 < 1 || d2 < 1 || d1 > 0x3fffffff || r_max < 1) return 0;
  const size_t few = mx4_rows_workspace_bytes(M < kMxMostFew ? M : kMxMostFew, d1, d2, r_max, 1);
  if (M <= kMxAlwaysFew) return kStreamCtrlBytes + few;
  const size_t many = align_up((size_t)d1 * d2 * 2, 256) + milora_routed_linear_workspace_bytes(M, d1, d2, r_max);
  const size_t direct = kStreamCtrlBytes + cut_bytes_bound(M, d2) + align_up(shrink_rows_bound(M, d1) * r_max * sizeof(float), 256) + align_up((size_t)M * sizeof(int2), 256) +
                        align_up(halves_of(nullptr, M, r_max).site * sizeof(bf16_t), 256);
  const size_t most = many > direct ? many : direct;
  return kStreamCtrlBytes + (most > few ? most : few);  // (behind the words of the stream kernels: packed and 4-bit weights in turn)
}

extern "C" int milora_routed_linear_kernel(int64_t M, int d1, int d2, int dtype, int w_layout) {
  if (M < 1 || d1 < 1 || d2 < 1 || !valid_dtype(dtype)) return MILORA_EINVAL;
  if (!valid_layout(w_layout)) return MILORA_EINVAL;
  if (w_layout != MILORA_W_ROWMAJOR) {
    if (dtype != MILORA_BF16 || !packed_shape_ok(d1, d2)) return MILORA_EUNSUPPORTED;
    if (w_layout == MILORA_W_MX4 && (d1 > 0x3fffffff || M > 0x7fffffffLL || !mx4_linear_fits(M, d1, d2))) return MILORA_ERANGE;
    if (w_layout == MILORA_W_PACKED || mx4_few_rows(M, d1, d2)) return MILORA_KERNEL_STREAM;
    return MILORA_KERNEL_TILES;
  }
  const void* aligned = (const void*)(uintptr_t)256;
  if (dtype == MILORA_BF16 && prefill_supported(M, d1, d2, aligned, aligned, aligned)) return MILORA_KERNEL_TILES;
  return MILORA_KERNEL_GENERIC;
}

extern "C" int milora_routed_linear_tile(int64_t M, int d1, int d2, int dtype, int w_layout) {
  const int kernel = milora_routed_linear_kernel(M, d1, d2, dtype, w_layout);
  if (kernel < 0) return kernel;
  const void* aligned = (const void*)(uintptr_t)256;
  if (w_layout == MILORA_W_MX4 && kernel == MILORA_KERNEL_STREAM) return 0;
  const bool packed = w_layout == MILORA_W_PACKED || (w_layout == MILORA_W_MX4 && !mx4_rowmajor(d1));
  const LinearPlan p = plan_linear(M, d1, d2, dtype, packed, aligned, aligned, aligned);
  if (w_layout == MILORA_W_MX4 && mx4_linear_direct(M, d1, d2, p)) return 256;
  if (p.kind != MILORA_KERNEL_TILES) return 0;
  return p.tiles.shape == kTiles256 ? 256 : p.tiles.shape == kTiles128 ? 128 : 64;
}

extern "C" int milora_routed_linear(const void* X, int64_t M, int d1, int d2, int dtype, const int32_t* row_to_req,
                                    const void* W, int w_layout, const void* bias, const milora_adapters* adapters,
                                    int site, const int32_t* tenant_id, const uint8_t* route, int B, void* Y,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!X || !W || !Y || !tenant_id || !route) return MILORA_EINVAL;
  if (M < 1 || d1 < 1 || d2 < 1 || B < 1) return MILORA_EINVAL;
  if (!valid_dtype(dtype) || site < 0 || site >= MILORA_NUM_SITES) return MILORA_EINVAL;
  if (!valid_layout(w_layout)) return MILORA_EINVAL;
  if (!row_to_req && M != B) return MILORA_EINVAL;
  int rc = check_adapters(adapters);
  if (rc) return rc;
  if (M > 0x7fffffffLL) return MILORA_ERANGE;
  const bool mx4 = w_layout == MILORA_W_MX4;
  if (mx4 && d1 > 0x3fffffff) return MILORA_ERANGE;
  if (!workspace || workspace_bytes < (mx4 ? milora_quantized_linear_workspace_bytes(M, d1, d2, adapters->r_max)
                                           : milora_routed_linear_workspace_bytes(M, d1, d2, adapters->r_max)))
    return MILORA_EWORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const AdapterView ad = view_of(adapters);
  const bool packed = w_layout == MILORA_W_PACKED;
  if (packed || mx4) {
    if (dtype != MILORA_BF16 || !packed_shape_ok(d1, d2) || !aligned16(X) || !aligned16(W) || !aligned16(Y) ||
        (bias && !aligned16(bias)))
      return MILORA_EUNSUPPORTED;
    if (packed && !row_to_req && M > MILORA_MAX_DECODE_BATCH) return MILORA_ERANGE;
  }
  if (mx4 && !mx4_linear_fits(M, d1, d2)) return MILORA_ERANGE;
  if (mx4)
    return run_linear_mx4((const bf16_t*)X, M, d1, d2, row_to_req, W, (const bf16_t*)bias, ad, site, tenant_id, route, B, (bf16_t*)Y,
                          (char*)workspace + kStreamCtrlBytes, st);
  return run_linear(X, M, d1, d2, dtype, row_to_req, W, packed, bias, ad, site, tenant_id, route, B, Y, workspace, st);
}

// Arguments that the gated block and its backward pass share.
static int check_gated(int64_t M, int d, int F, int dtype, const int32_t* row_to_req, const void* Wg, const void* Wu, int w_layout,
                       const milora_adapters* adapters, const int32_t* tenant_id, const uint8_t* route, int B) {
  if (!Wg || !Wu || !tenant_id || !route) return MILORA_EINVAL;
  if (M < 1 || d < 1 || F < 1 || B < 1 || !valid_dtype(dtype) || !valid_layout(w_layout)) return MILORA_EINVAL;
  if (!row_to_req && M != B) return MILORA_EINVAL;
  const int rc = check_adapters(adapters);
  if (rc) return rc;
  if (M > 0x7fffffffLL || F > 0x3fffffff || d > 0x3fffffff) return MILORA_ERANGE;
  if (w_layout == MILORA_W_PACKED) return MILORA_EUNSUPPORTED;
  if (w_layout == MILORA_W_MX4 && (dtype != MILORA_BF16 || !packed_shape_ok(d, F) || !aligned16(Wg) || !aligned16(Wu))) return MILORA_EUNSUPPORTED;
  return MILORA_OK;
}

extern "C" size_t milora_gated_linear_workspace_bytes(int64_t M, int d, int F, int dtype, int w_layout, int r_max) {
  if (M < 1 || d < 1 || F < 1 || F > 0x3fffffff || d > 0x3fffffff || r_max < 1 || !valid_dtype(dtype) || !valid_layout(w_layout)) return 0;
  return gated_workspace_bytes(M, d, F, dtype, w_layout == MILORA_W_MX4, r_max);
}

extern "C" int milora_gated_linear(const void* X, int64_t M, int d, int F, int dtype, const int32_t* row_to_req, const void* W_gate,
                                   const void* W_up, int w_layout, const milora_adapters* adapters, const int32_t* tenant_id,
                                   const uint8_t* route, int B, void* Y, float* gate_out, float* up_out, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  if (!X || !Y) return MILORA_EINVAL;
  const int rc = check_gated(M, d, F, dtype, row_to_req, W_gate, W_up, w_layout, adapters, tenant_id, route, B);
  if (rc) return rc;
  if (w_layout == MILORA_W_MX4 && (!aligned16(X) || !aligned16(Y))) return MILORA_EUNSUPPORTED;
  if (!workspace || workspace_bytes < milora_gated_linear_workspace_bytes(M, d, F, dtype, w_layout, adapters->r_max)) return MILORA_EWORKSPACE;
  const GatedCall g{X, M, d, F, dtype, w_layout == MILORA_W_MX4, row_to_req, W_gate, W_up, view_of(adapters), tenant_id, route, B};
  return run_gated(g, Y, gate_out, up_out, workspace, (hipStream_t)stream);
}

extern "C" size_t milora_gated_linear_backward_workspace_bytes(int64_t M, int d, int F, int dtype, int w_layout, int r_max) {
  if (M < 1 || d < 1 || F < 1 || F > 0x3fffffff || d > 0x3fffffff || r_max < 1 || !valid_dtype(dtype) || !valid_layout(w_layout)) return 0;
  return gated_backward_workspace_bytes(M, d, F, dtype, w_layout == MILORA_W_MX4, r_max);
}

extern "C" int milora_gated_linear_backward(const void* dY, const void* X, const float* gate, const float* up, int64_t M, int d, int F,
                                            int dtype, const int32_t* row_to_req, const void* W_gate, const void* W_up, int w_layout,
                                            const milora_adapters* adapters, const int32_t* tenant_id, const uint8_t* route, int B,
                                            void* dX, const milora_gradients* gradients, void* workspace, size_t workspace_bytes,
                                            void* stream) {
  if (!dY || !X || !gate || !up) return MILORA_EINVAL;
  const int rc = check_gated(M, d, F, dtype, row_to_req, W_gate, W_up, w_layout, adapters, tenant_id, route, B);
  if (rc) return rc;
  if (!workspace || workspace_bytes < milora_gated_linear_backward_workspace_bytes(M, d, F, dtype, w_layout, adapters->r_max))
    return MILORA_EWORKSPACE;
  const GatedCall g{X, M, d, F, dtype, w_layout == MILORA_W_MX4, row_to_req, W_gate, W_up, view_of(adapters), tenant_id, route, B};
  return run_gated_backward(g, dY, gate, up, dX, gradients ? gradients->dA : nullptr, gradients ? gradients->dB : nullptr, workspace,
                            (hipStream_t)stream);
}

extern "C" int milora_packed_workspace_status(const void* workspace, int* status, void* stream) {
  if (!status) return MILORA_EINVAL;
  if (!workspace) return static_scratch_status(status, (hipStream_t)stream);
  return decode_workspace_status(workspace, status, (hipStream_t)stream);
}

extern "C" int milora_set_wait_limit(int polls) { return set_wait_limit(polls); }

extern "C" size_t milora_layer_decode_workspace_bytes(int B, int d, int F, int r_max) {
  if (B < 1 || d < 1 || F < 1 || r_max < 1 || B > MILORA_MAX_DECODE_BATCH) return 0;
  size_t a = carve_generic(nullptr, B, d, F, r_max, 4).bytes;
  size_t b = decode_packed_workspace_bytes(B, d, F, r_max);
  const size_t c = carve_mx4(nullptr, B, d, F, r_max).bytes;
  a = a > b ? a : b;
  return a > c ? a : c;
}

static int layer_decode_impl(const void* x, int B, int d, int F, int dtype, const milora_layer_weights* weights,
                             const milora_adapters* adapters, const int32_t* tenant_id, const uint8_t* route,
                             uint32_t flags, const void* attn_out, void* y, void* qkv_out, void* workspace,
                             size_t workspace_bytes, void* stream, LaunchMarks* marks) {
  if (!x || !y || !weights || !tenant_id || !route) return MILORA_EINVAL;
  if (B < 1 || d < 1 || F < 1 || !valid_dtype(dtype)) return MILORA_EINVAL;
  if (flags & ~MILORA_LAYER_RMSNORM) return MILORA_EINVAL;
  for (int m = 0; m < MILORA_NUM_SITES; ++m)
    if (!weights->W[m]) return MILORA_EINVAL;
  if (!valid_layout(weights->layout)) return MILORA_EINVAL;
  int rc = check_adapters(adapters);
  if (rc) return rc;
  if (B > MILORA_MAX_DECODE_BATCH) return MILORA_ERANGE;
  if (!workspace || workspace_bytes < milora_layer_decode_workspace_bytes(B, d, F, adapters->r_max))
    return MILORA_EWORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const AdapterView ad = view_of(adapters);
  if (weights->layout != MILORA_W_ROWMAJOR) {
    if (dtype != MILORA_BF16 || d % 32 != 0 || F % 32 != 0) return MILORA_EUNSUPPORTED;
    if (!aligned16(x) || (attn_out && !aligned16(attn_out)) || !aligned16(y) || (qkv_out && !aligned16(qkv_out)))
      return MILORA_EUNSUPPORTED;
    for (int m = 0; m < MILORA_NUM_SITES; ++m)
      if (!aligned16(weights->W[m])) return MILORA_EUNSUPPORTED;
    if (weights->layout == MILORA_W_MX4) {
      if (marks) return MILORA_EUNSUPPORTED;
      if (d > 0x3fffffff || F > 0x3fffffff) return MILORA_ERANGE;
      if (!mx4_rows_fit(B, d, d, 3) || !mx4_rows_fit(B, d, d, 1) || !mx4_rows_fit(B, d, F, 2, true) || !mx4_rows_fit(B, F, d, 1)) return MILORA_ERANGE;
      return layer_decode_mx4((const bf16_t*)x, B, d, F, weights, ad, tenant_id, route, flags, (const bf16_t*)attn_out, (bf16_t*)y,
                              (bf16_t*)qkv_out, workspace, st);
    }
    return layer_decode_packed((const bf16_t*)x, B, d, F, weights, ad, tenant_id, route, flags,
                               (const bf16_t*)attn_out, (bf16_t*)y, (bf16_t*)qkv_out, workspace, st, marks);
  }
  if (marks) return MILORA_EUNSUPPORTED;
  if (dtype == MILORA_BF16)
    return layer_decode_generic<bf16_t>(x, B, d, F, dtype, weights, ad, tenant_id, route, flags, attn_out, y, qkv_out,
                                        workspace, st);
  return layer_decode_generic<float>(x, B, d, F, dtype, weights, ad, tenant_id, route, flags, attn_out, y, qkv_out,
                                     workspace, st);
}

extern "C" int milora_layer_decode(const void* x, int B, int d, int F, int dtype, const milora_layer_weights* weights,
                                   const milora_adapters* adapters, const int32_t* tenant_id, const uint8_t* route,
                                   uint32_t flags, const void* attn_out, void* y, void* qkv_out, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  return layer_decode_impl(x, B, d, F, dtype, weights, adapters, tenant_id, route, flags, attn_out, y, qkv_out,
                           workspace, workspace_bytes, stream, nullptr);
}

extern "C" int milora_layer_decode_noalloc(const void* x, int B, int d, int F, int dtype,
                                           const milora_layer_weights* weights, const milora_adapters* adapters,
                                           const int32_t* tenant_id, const uint8_t* route, uint32_t flags,
                                           const void* attn_out, void* y, void* qkv_out, void* stream) {
  if (!x || !y || !weights || !tenant_id || !route) return MILORA_EINVAL;
  if (B < 1 || d < 1 || F < 1 || !valid_dtype(dtype)) return MILORA_EINVAL;
  if (flags & ~MILORA_LAYER_RMSNORM) return MILORA_EINVAL;
  for (int m = 0; m < MILORA_NUM_SITES; ++m)
    if (!weights->W[m]) return MILORA_EINVAL;
  int rc = check_adapters(adapters);
  if (rc) return rc;
  if (weights->layout != MILORA_W_PACKED || dtype != MILORA_BF16 || d % 32 != 0 || F % 32 != 0) return MILORA_EUNSUPPORTED;
  if (!aligned16(x) || (attn_out && !aligned16(attn_out)) || !aligned16(y) || (qkv_out && !aligned16(qkv_out)))
    return MILORA_EUNSUPPORTED;
  for (int m = 0; m < MILORA_NUM_SITES; ++m)
    if (!aligned16(weights->W[m])) return MILORA_EUNSUPPORTED;
  return layer_decode_packed_static((const bf16_t*)x, B, d, F, weights, view_of(adapters), tenant_id, route, flags,
                                    (const bf16_t*)attn_out, (bf16_t*)y, (bf16_t*)qkv_out, (hipStream_t)stream);
}

extern "C" int milora_layer_decode_profile(const void* x, int B, int d, int F, int dtype,
                                           const milora_layer_weights* weights, const milora_adapters* adapters,
                                           const int32_t* tenant_id, const uint8_t* route, uint32_t flags,
                                           const void* attn_out, void* y, void* qkv_out, void* workspace,
                                           size_t workspace_bytes, void* stream, int reps, float* slot_ms) {
  if (!slot_ms || reps < 1) return MILORA_EINVAL;
  hipStream_t st = (hipStream_t)stream;
  hipEvent_t ev[MILORA_PROFILE_SLOTS + 1];
  for (int i = 0; i <= MILORA_PROFILE_SLOTS; ++i) MILORA_HIP(hipEventCreate(&ev[i]));
  for (int i = 0; i < MILORA_PROFILE_SLOTS; ++i) slot_ms[i] = 0.f;
  LaunchMarks marks{ev + 1, MILORA_PROFILE_SLOTS};
  int rc = MILORA_OK;
  for (int r = 0; r < reps && rc == MILORA_OK; ++r) {
    MILORA_HIP(hipEventRecord(ev[0], st));
    rc = layer_decode_impl(x, B, d, F, dtype, weights, adapters, tenant_id, route, flags, attn_out, y, qkv_out,
                           workspace, workspace_bytes, stream, &marks);
    if (rc != MILORA_OK) break;
    MILORA_HIP(hipStreamSynchronize(st));
    for (int i = 0; i < MILORA_PROFILE_SLOTS; ++i) {
      float ms = 0.f;
      if (hipEventElapsedTime(&ms, ev[i], ev[i + 1]) == hipSuccess) slot_ms[i] += ms / (float)reps;
      else (void)hipGetLastError();
    }
  }
  for (int i = 0; i <= MILORA_PROFILE_SLOTS; ++i) (void)hipEventDestroy(ev[i]);
  return rc;
}

extern "C" size_t milora_layer_decode_trace_bytes(void) { return decode_trace_bytes(); }

extern "C" int milora_layer_decode_trace(const void* x, int B, int d, int F, int dtype,
                                         const milora_layer_weights* weights, const milora_adapters* adapters,
                                         const int32_t* tenant_id, const uint8_t* route, uint32_t flags,
                                         const void* attn_out, void* y, void* qkv_out, void* workspace,
                                         size_t workspace_bytes, void* stream, void* stamps, size_t stamps_bytes,
                                         int32_t* dims) {
  if (!stamps || !dims) return MILORA_EINVAL;
  if (stamps_bytes < decode_trace_bytes()) return MILORA_EWORKSPACE;
  if (!weights || weights->layout != MILORA_W_PACKED) return MILORA_EUNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  MILORA_HIP(hipMemsetAsync(stamps, 0, decode_trace_bytes(), st));
  LaunchMarks marks{nullptr, 0};
  marks.trace = (long long*)stamps;
  const int rc = layer_decode_impl(x, B, d, F, dtype, weights, adapters, tenant_id, route, flags, attn_out, y, qkv_out,
                                   workspace, workspace_bytes, stream, &marks);
  if (rc != MILORA_OK) return rc;
  MILORA_HIP(hipStreamSynchronize(st));
  int smax = 0, waves = 0, slots = 0;
  decode_trace_dims(&smax, &waves, &slots);
  dims[0] = marks.grid; dims[1] = marks.stages; dims[2] = smax; dims[3] = waves; dims[4] = slots;
  return MILORA_OK;
}

extern "C" size_t milora_quantized_weight_bytes(int d1, int d2) { return mx4_shape_ok(d1, d2) ? mx4_bytes(d1, d2) : 0; }

extern "C" int milora_quantize_weight(const void* src_rowmajor, int dtype, void* dst, int d1, int d2, void* stream) {
  if (!src_rowmajor || !dst || d1 < 1 || d2 < 1 || !valid_dtype(dtype)) return MILORA_EINVAL;
  if (!mx4_shape_ok(d1, d2) || !aligned16(dst)) return MILORA_EUNSUPPORTED;
  return mx4_quantize(src_rowmajor, dtype, dst, d1, d2, (hipStream_t)stream);
}

extern "C" int milora_dequantize_weight(const void* src, void* dst_rowmajor, int dtype, int d1, int d2, void* stream) {
  if (!src || !dst_rowmajor || d1 < 1 || d2 < 1 || !valid_dtype(dtype)) return MILORA_EINVAL;
  if (!mx4_shape_ok(d1, d2) || !aligned16(src)) return MILORA_EUNSUPPORTED;
  return mx4_dequantize(src, dst_rowmajor, dtype, d1, d2, false, (hipStream_t)stream);
}

extern "C" int milora_pack_weight(const void* src_rowmajor, void* dst_packed, int d1, int d2, void* stream) {
  if (!src_rowmajor || !dst_packed || d1 < 1 || d2 < 1) return MILORA_EINVAL;
  if (!packed_shape_ok(d1, d2) || !aligned16(src_rowmajor) || !aligned16(dst_packed)) return MILORA_EUNSUPPORTED;
  return pack_weight(src_rowmajor, dst_packed, d1, d2, (hipStream_t)stream);
}

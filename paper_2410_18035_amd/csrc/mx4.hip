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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1))) const bf16_t gbf16;

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

__device__ __forceinline__ float mx4_scale(uint32_t s) { return __uint_as_float(s << 23); }  // 255: the conversion gives NaN

// Eight codes to eight bf16.
__device__ __forceinline__ u32x4 mx4_bf16(uint32_t c, float scale) {
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
  return v;
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

// ---- few rows -------------------------------------------------------------------------------------------------------------
// A workgroup of eight waves takes NT tiles of 16 columns (GATED: half of them of the gate, half of the up projection, for the
// same outputs) and up to 16 MT rows.  The reduction is dealt to the waves in steps of 128 inputs: a lane loads the 32 codes of
// one group of one column (16 bytes), its scale and the same 32 inputs of a row of X, and multiplies them in four matrix
// instructions of 8 inputs a lane (which inputs stand at which place of an instruction does not matter as long as both
// operands agree).  The codes of a chunk of steps are on their way before the first is used: the whole of a weight of 4096 x 4096
// is then in flight at once.  The waves' sums meet in LDS.
// The LoRA term: t = X W^A comes from a launch of its own; the first ranks of W^B are asked for in front of the reduction.
constexpr int kMxW = 8;
constexpr int kMxT = kMxW * 64;

template <int MT, int NT, bool GATED>
struct MxCfg {
  static constexpr int U = MT * NT > 2 ? 2 : 4;  // steps of a chunk
  static constexpr int Ld = 16 * NT + 4;      // fp32 row of the sums in LDS
  static constexpr int Sites = GATED ? 2 : 1;
  static constexpr int Outs = MT * NT;        // outputs of a thread (two threads share each)
  static constexpr int Pre = Outs == 1 ? 16 : 16 / Outs;      // ranks of each asked for ahead
  static constexpr int RedBytes = kMxW * 16 * MT * Ld * 4;
};

template <int MT, int NT, bool GATED>
__global__ void __launch_bounds__(kMxT, 4) mx4_rows_kernel(const MxArgs g) {
  typedef MxCfg<MT, NT, GATED> C;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ int2 s_lora[C::Sites][16 * MT];
  float* const red = reinterpret_cast<float*>(lds);                 // [wave][row][Ld]
  float* const ts = reinterpret_cast<float*>(lds + C::RedBytes);    // [site][row][r_max]
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int s0 = GATED ? 0 : blockIdx.y;
  constexpr int kCols = GATED ? NT * 8 : NT * 16;  // outputs of the workgroup
  const int n0 = blockIdx.x * kCols;
  const int d1 = g.d1, r_max = g.ad.r_max;

  // ---- operands of this lane ----
  const unsigned char* wp[NT];
  const uint8_t* sp[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    int col = n0 + (GATED ? j / 2 : j) * 16 + li;
    col = col < g.d2 ? col : g.d2 - 1;  // (columns past the end: results dropped)
    const unsigned char* const base = g.W[GATED ? j & 1 : s0];
    wp[j] = base + (size_t)col * (d1 >> 1) + lq * 16;
    sp[j] = base + (size_t)d1 * g.d2 / 2 + (size_t)col * (d1 >> 5) + lq;
  }
  const bf16_t* xp[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int row = i * 16 + li < g.M ? i * 16 + li : g.M - 1;
    xp[i] = g.X + (size_t)row * g.ldx + lq * 32;
  }
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int full = d1 >> 7;  // whole steps
  u32x4 c[C::U][NT];
  uint32_t sc[C::U][NT];
  auto load = [&](int b0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < C::U; ++u) {
      const int b = b0 + u * kMxW < full ? b0 + u * kMxW : full - 1;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        c[u][j] = *reinterpret_cast<const u32x4*>(wp[j] + (size_t)b * 64);
        sc[u][j] = sp[j][b * 4];
      }
    }
  };
  auto load_x = [&](int b, u32x4 (&x)[MT][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[i][k] = *reinterpret_cast<const u32x4*>(xp[i] + (size_t)b * 128 + k * 8);
  };
  auto step = [&](const u32x4 (&cc)[NT], const uint32_t (&ss)[NT], const u32x4 (&xx)[MT][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const float scale = mx4_scale(ss[j]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bf16x8 wv = __builtin_bit_cast(bf16x8, mx4_bf16(cc[j][k], scale));
#pragma unroll
        for (int i = 0; i < MT; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, __builtin_bit_cast(bf16x8, xx[i][k]), acc[i][j], 0, 0, 0);
      }
    }
  };
  if (w < full) load(w);

  // ---- LoRA: tenants and ranks of the rows, t into LDS, the first ranks of W^B ----
  if (tid < 16 * MT)
#pragma unroll
    for (int s = 0; s < C::Sites; ++s)
      s_lora[s][tid] = tid < g.M ? g.row_lora[(s0 + s) * g.lora_site + tid] : int2{-1, 0};
  __syncthreads();
  const int n_out = tid & 15, m_out = (tid >> 4) & 15, half = tid >> 8;
  const bf16_t* bp[MT][NT];
  int rank[MT][NT];
  uint32_t pre[MT][NT][C::Pre];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int2 tr = s_lora[GATED ? j & 1 : 0][i * 16 + m_out];
      const int n = n0 + (GATED ? j / 2 : j) * 16 + n_out;
      rank[i][j] = n < g.d2 ? tr.y : 0;
      bp[i][j] = nullptr;
      if (rank[i][j] > 0) {
        bp[i][j] = (const bf16_t*)g.ad.B[tr.x * MILORA_NUM_SITES + g.site[s0] + (GATED ? j & 1 : 0)] + n;
#pragma unroll
        for (int u = 0; u < C::Pre; ++u) {  // this half's ranks: half, half + 2, ...
          const int r = 2 * u + half;
          pre[i][j][u] = ((gbf16*)bp[i][j])[(size_t)(r < rank[i][j] ? r : 0) * g.d2];
        }
      }
    }
  for (int e = tid; e < C::Sites * 16 * MT * r_max; e += kMxT) {
    const int s = e / (16 * MT * r_max), row = e / r_max % (16 * MT), r = e % r_max;
    float v = 0.f;
    if (r < s_lora[s][row].y) {
      const float* const tp = g.t + (s0 + s) * g.t_site + (size_t)row * r_max + r;
      for (int k = 0; k < g.parts; ++k) v += tp[k * g.t_part];
    }
    ts[e] = v;
  }

  // ---- base linear ----
  for (int b0 = w; b0 < full; b0 += kMxW * C::U) {
    if (b0 != w) load(b0);
#pragma unroll
    for (int u = 0; u < C::U; ++u)
      if (b0 + u * kMxW < full) {
        u32x4 x[MT][4];
        load_x(b0 + u * kMxW, x);
        step(c[u], sc[u], x);
      }
  }
  if ((d1 & 127) && w == full % kMxW) {  // the last groups: lanes past the end multiply zeros
    const bool in = full * 128 + lq * 32 < d1;
    u32x4 c1[NT], x1[MT][4];
    uint32_t s1[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      c1[j] = u32x4{0u, 0u, 0u, 0u};
      s1[j] = 127;
      if (in) {
        c1[j] = *reinterpret_cast<const u32x4*>(wp[j] + (size_t)full * 64);
        s1[j] = sp[j][full * 4];
      }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x1[i][k] = u32x4{0u, 0u, 0u, 0u};
        if (in) x1[i][k] = *reinterpret_cast<const u32x4*>(xp[i] + (size_t)full * 128 + k * 8);
      }
    step(c1, s1, x1);
  }
  // (lane: row li, columns 4 lq .. + 3 of the 16)
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
      *reinterpret_cast<f32x4*>(red + ((size_t)w * 16 * MT + i * 16 + li) * C::Ld + j * 16 + lq * 4) = acc[i][j];
  __syncthreads();

  // ---- sums: two threads an output, four waves' parts and every other rank each ----
  float val[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < kMxW / 2; ++k) v += red[((size_t)(half * (kMxW / 2) + k) * 16 * MT + i * 16 + m_out) * C::Ld + j * 16 + n_out];
      if (rank[i][j] > 0) {
        const float* const tr = ts + ((GATED ? j & 1 : 0) * 16 * MT + i * 16 + m_out) * r_max;
#pragma unroll
        for (int u = 0; u < C::Pre; ++u) {
          const int r = 2 * u + half;
          if (r < rank[i][j]) v += tr[r] * bf16_to_f32((bf16_t)pre[i][j][u]);
        }
        for (int r0 = 2 * C::Pre + half; r0 < rank[i][j]; r0 += 16) {
          bf16_t b[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) b[u] = ((gbf16*)bp[i][j])[(size_t)(r0 + 2 * u < rank[i][j] ? r0 + 2 * u : 0) * g.d2];
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if (r0 + 2 * u < rank[i][j]) v += tr[r0 + 2 * u] * bf16_to_f32(b[u]);
        }
      }
      val[i][j] = v;
    }
  __syncthreads();
  if (half == 1)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) red[(i * 16 + m_out) * C::Ld + j * 16 + n_out] = val[i][j];
  __syncthreads();
  if (half == 1) return;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = i * 16 + m_out;
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < NT; ++j) val[i][j] += red[m * C::Ld + j * 16 + n_out];
    if constexpr (GATED) {
#pragma unroll
      for (int j = 0; j < NT; j += 2) {
        const int n = n0 + j * 8 + n_out;
        if (n >= g.d2) continue;
        const float gate = val[i][j], up = val[i][j + 1];
        const size_t at = (size_t)m * g.d2 + n;
        if (g.gate_out) g.gate_out[at] = gate;
        if (g.up_out) g.up_out[at] = up;
        g.Y[0][(size_t)m * g.ldy + n] = f32_to_bf16(silu(gate) * up);
      }
    } else {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int n = n0 + j * 16 + n_out;
        if (n >= g.d2) continue;
        float v = val[i][j];
        if (g.bias) v += bf16_to_f32(g.bias[n]);
        const size_t at = (size_t)m * g.d2 + n;
        if (g.res) {
          v += bf16_to_f32(g.res[at]);
          g.h_out[at] = v;
        }
        if (g.h_in) v += g.h_in[at];
        if (g.Y[s0]) g.Y[s0][(size_t)m * g.ldy + n] = f32_to_bf16(v);
      }
    }
  }
}

template <int MT, int NT, bool GATED>
int launch_rows(const MxArgs& g, int sites, hipStream_t st) {
  typedef MxCfg<MT, NT, GATED> C;
  const int bytes = C::RedBytes + C::Sites * 16 * MT * g.ad.r_max * (int)sizeof(float);
  static thread_local int lds_set_for = -1;
  int dev = 0;
  MILORA_HIP(hipGetDevice(&dev));
  if (lds_set_for != dev) {
    const int most = C::RedBytes + C::Sites * 16 * MT * MILORA_MAX_RANK * (int)sizeof(float);
    MILORA_HIP(hipFuncSetAttribute((const void*)mx4_rows_kernel<MT, NT, GATED>, hipFuncAttributeMaxDynamicSharedMemorySize, most));
    lds_set_for = dev;
  }
  constexpr int kCols = GATED ? NT * 8 : NT * 16;
  hipLaunchKernelGGL((mx4_rows_kernel<MT, NT, GATED>), dim3((unsigned)((g.d2 + kCols - 1) / kCols), GATED ? 1 : sites), dim3(kMxT), bytes, st, g);
  return check_launch();
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

int launch_mx4_rows(const MxArgs& g, int sites, bool gated, hipStream_t st) {
  if (g.M <= 16) return gated ? launch_rows<1, 2, true>(g, 1, st) : launch_rows<1, 1, false>(g, sites, st);
  return gated ? launch_rows<2, 2, true>(g, 1, st) : launch_rows<2, 2, false>(g, sites, st);
}

}  // namespace milora

// Interface of the 4-bit base weights (mx4.hip): storage, conversion, the few-row linears.
#pragma once
#include "shrink.h"

namespace milora {

// Storage of a weight of d1 inputs and d2 columns (MILORA_W_MX4): codes [d2][d1 / 2], the even input of a byte in its low
// half, then one scale byte for 32 inputs of a column, [d2][d1 / 32].
constexpr int kMxGroup = 32;
inline bool mx4_shape_ok(int d1, int d2) { return d1 >= 1 && d2 >= 1 && d1 % kMxGroup == 0; }
inline size_t mx4_code_bytes(int d1, int d2) { return (size_t)d1 * d2 / 2; }
inline size_t mx4_bytes(int d1, int d2) { return mx4_code_bytes(d1, d2) + (size_t)d1 * d2 / kMxGroup; }

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

int mx4_quantize(const void* src, int dtype, void* dst, int d1, int d2, hipStream_t st);
// To [d2][d1] of `dtype`, or (bf16, d2 % 16 == 0) to the packed layout.
int mx4_dequantize(const void* src, void* dst, int dtype, int d1, int d2, bool packed, hipStream_t st);

// Few rows: the linears of up to three consecutive sites on the same X, or the gated block.
struct MxArgs {
  const bf16_t* X;  // M rows of ldx elements
  int64_t ldx;
  bool second;      // behind them M rows with what their rounding left, which the products take in as well (without: 32 requests 73.6 us a step for 77,
                    // 128 165 for 186, and y 0.0031 off its exact value for 0.0025)
  int M, d1, d2;
  const unsigned char* W[3];  // of the sites; gated: W[0] gate, W[1] up
  const bf16_t* bias;
  bf16_t* Y[3];     // rows of ldy elements
  int64_t ldy;
  float* gate_out;  // gated: [M][d2] or null
  float* up_out;
  const bf16_t* res;   // [M][d2] or null: h_out = res + linear, in fp32, and Y that rounded
  float* h_out;
  bf16_t* left_out;    // [M][d2] or null: what the rounding of Y left of h_out
  const float* h_in;   // [M][d2] or null: Y = h_in + linear
  const bf16_t* norm_x;  // [M][d1] or null: the products are of the rows divided by the root of their mean square (plus 1e-5)
  const float* norm_h;   // the same, rows in fp32
  AdapterView ad;
  int site[3];
  const int32_t* row_to_req;
  const int32_t* tenant_id;
  const uint8_t* route;
  int B;
};
// The few-row kernels read the codes for up to 128 rows, and for up to 512 while the products of all sites stay below 24e9.  Beyond, tiles are
// faster, whose time hardly falls below 256 rows (us, few-row kernels / tiles: 4096 x 11008, 320 rows 76 / 115, 512 rows 107 / 107, 768 rows
// 153 / 108; 5120 x 13824, 320 rows 115 / 136, 384 rows 137 / 131; gated 4096 x 11008, 256 rows 114 / 126, 320 rows 125 / 124).
constexpr int64_t kMxAlwaysFew = 128, kMxMostFew = 512;
inline bool mx4_few_rows(int64_t M, int d1, int64_t columns) {
  return M <= kMxAlwaysFew || (M <= kMxMostFew && (double)M * d1 * columns <= 24e9);
}
// Up to so many rows the second ones are rows of their own behind them: the matrix instructions of up to 16 rows have them to spare.  Beyond, they
// go through LDS after the first ones (us a decode step of 4096 x 11008, behind / after: 1 request 47.1 / 49.0, 5 52 / 56, 8 56 / 60, 9 66 / 61, 16 68 /
// 64, 32 82 / 77, 128 211 / 186).
constexpr int kMxBehind = 8;
size_t mx4_rows_workspace_bytes(int64_t M, int d1, int d2, int r_max, int sites, bool second = false);
// Does a launch take these sizes?
bool mx4_rows_fit(int64_t M, int d1, int d2, int sites, bool second = false);
// gated: sites = 2
int launch_mx4_rows(const MxArgs& g, int sites, bool gated, void* workspace, hipStream_t st);

}  // namespace milora

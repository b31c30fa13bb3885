// Many-row (prefill) routed LoRA linear on row-major bf16 weights (paper Eq. 1 with the layer-level gate of
// Sec. 3.3): Y = X W^T + bias + (X W^A) W^B for the rows whose request is routed to this site.
//
// One workgroup of four waves computes a 256 x 256 tile of Y with the bf16 matrix cores
// (v_mfma_f32_32x32x16_bf16, fp32 accumulators, 128 x 128 per wave; a kernel of nothing but this instruction
// sustains 2.3-2.4 PFLOP/s on the chip, one of nothing but the 16x16x32 form 1.45-1.5).  X and W are both contiguous along the
// reduction index: 16-row x 64-k blocks of either are copied from global memory straight into LDS
// (global_load_lds_dwordx4, no registers; whole 128-byte lines per row), in a ring of five half steps of
// 32 KB, and read back as matrix-core operands with one conflict-free 16-byte LDS load per lane, pair of blocks
// and 16 k.  A step's operands are all in registers after a quarter of its matrix work; its ring slots are
// refilled from there on, so that nearly the whole LDS is data on its way (the copies are bound by latency:
// bytes in flight over about two microseconds).
// The LoRA term enters as extra k steps: t = X W^A (fp32, computed beforehand) split into two bf16 halves
// (hi + lo, about 17 of its 24 bits) against W^B of the tenant, masked to that tenant's rows; Inf and NaN of W^B are kept
// out of the stages and added to those rows at the end.
// Bias is added and the result rounded once at the store.
#include <type_traits>

#include "mx4.h"
#include "tiles.h"

namespace milora {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_a8 __attribute__((ext_vector_type(4), aligned(8)));
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef __attribute__((address_space(1))) const u32x4_a2 gu32x4_a2;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
constexpr int kTM = 256, kTN = 256, kTK = 64;
constexpr int kThreadsP = 256;
constexpr int kBlocksM = kTM / 16, kBlocksN = kTN / 16;
constexpr int kBlockBytes = 16 * kTK * 2;                 // 16 rows x 64 k: 2 KiB, a row is one 128-byte line
constexpr int kHalfBytes = (kBlocksM + kBlocksN) / 2 * kBlockBytes;  // 8 X blocks + 8 W blocks: 32 KiB
constexpr int kHalves = 5;                                // ring of half steps
constexpr int kLdsBytesP = kHalves * kHalfBytes;
constexpr int kAccTilesRows = 3;
constexpr int kOutPitch = 128 * 2 + 16;                   // a row of a wave's results on their way out, padded: 16 rows at one column hit all banks
static_assert(4 * 128 * kOutPitch <= kLdsBytesP, "results of the four waves");
// Where the sixteen copy instructions of a k step sit among its 64 matrix instructions: those of the first half
// after instructions 0, kCopyAStride, ..., those of the second half from instruction kCopyB0 on (16 or later: the
// slot they fill is read until then).
constexpr int kCopyAStride = 2, kCopyB0 = 16, kCopyBStride = 3;
static_assert(kCopyB0 >= 16 && 7 * kCopyAStride < kCopyB0 && kCopyB0 + 7 * kCopyBStride < 64, "copy positions");
constexpr int kGroupM = 4;  // consecutive workgroups of an XCD walk 4 row tiles of one column tile

enum PMode { kPlain, kGated, kBack };
struct PParams {
  const bf16_t* X;
  const bf16_t* W;
  const bf16_t* W2;   // kGated, kBack: the up projection (W: the gate)
  const bf16_t* bias;
  bf16_t* Y;
  float* gate_out;    // kGated: [M][d2] each, or null
  float* up_out;
  size_t t_site;      // kGated, kBack: floats to the shrinks of the next site
  // kGated, kBack, 4-bit weights: [site][M of the call] tenant and rank of each row, and the shrinks as two bf16 halves: [site][chunk of 32 ranks][1 + M] lines
  // of 64 values, 32 high halves and 32 low ones; the first line is zero
  const int2* row_lora;
  size_t lora_site;
  const bf16_t* halves;
  size_t half_site, half_chunk;
  float* partial;     // kBack, S > 1: [part][M][d2] sums of the parts of the reduction
  size_t partial_stride;
  int S, steps;       // kBack: parts, and k steps of a part
  int whole, cut, cut_steps;  // (not kPlain on bf16) tiles behind the first `whole` are cut in `cut` parts of so many k steps
  float* cut_sums;            // [tile behind those][part][65536]
  int* cut_cnt;               // [tile behind those][2], zero between launches
  int polls;                  // of the wait for a cut tile's other sums
  const float* t;     // `parts` partial shrinks [part][rows of the whole call][r_max], to be added in part order
  size_t t_stride;    // floats from one part to the next
  int parts;
  const int32_t* row_to_req;
  const int32_t* tenant_id;
  const uint8_t* route;
  AdapterView ad;
  int64_t M;         // rows of this launch
  int64_t row_base;  // index of its first row in the caller's matrix (requests of unmapped rows)
  int d1, d2, site, B;
  int tilesM, tilesN;
};

// Which of the eight 16-byte pieces of its 128-byte LDS line holds k group kg of row r (0..15) of a block:
// kg ^ swz(r).  Eight neighbouring rows get eight different pieces, and rows r and r + 8 (which lie 1 KiB apart, on
// the same banks) differ too, so a 16-byte operand read of 16 rows at one k group touches every bank once.
__device__ __forceinline__ int swz(int r) { return (r & 7) ^ ((r >> 3) & 1); }

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// copy_to_lds16 with four bytes a lane
__device__ __forceinline__ void copy_to_lds4(const void* base, uint32_t voff, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(dst), "v"(voff), "s"(base)
               : "memory");
}

template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0f70);
}

// kGated: the tile's W side is 128 columns of the gate and the same of the up projection, 64 and 64 in each wave's part, so that a
// lane ends up with both for its outputs: Y = silu(g) u, rounded once.
//
// kBack: Y = X [W; W2], the reduction (d1) running over the rows of both row-major weights (each [d1 / 2][d2]): the gradient behind the two
// projections, X = [dg | du].  A k step's W side is 64 rows of 256 columns, copied as they lie, 256 bytes of a row to a half; the transposing
// LDS read (ds_read_b64_tr_b16: four rows x sixteen columns by sixteen lanes) makes operands of them.  A row's sixteen-column pieces are permuted
// so that the four rows of two pieces that half a wave reads at once lie on all banks.  The LoRA steps take t = dz W^B^T against the rows of
// W^A, which are contiguous along the ranks.  Very few tiles: the reduction in S > 4 parts, their fp32 sums added in part order by a launch behind this one.
__device__ __forceinline__ int swz_tr(int k) { return ((k & 3) << 1) | ((k >> 3) & 1); }  // of a row's eight pieces
typedef short s16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bf16x8 read_tr(uint32_t at) {  // rows k .. k + 3 and, 1024 bytes on, k + 4 .. k + 7
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  s16x4 v[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(at + h * 1024));
  return __builtin_bit_cast(bf16x8, v);
}

// Cut tiles (cut_plan; not kPlain on bf16): the tiles of a last turn that would not fill the compute units are dealt to up to four workgroups each.
// What it gains, us of a call with / without (a turn of 4096 inputs 105 us): gated block of 4096 x 11008, 777 rows, 1.3 turns, 217 / 246; 600 rows,
// 1.0, 193 / 324; 4096 rows, 5.4, 702 / 723; 5120 x 13824, 8192 rows, 13.5 turns, 2071 / 2070; 4-bit linear of 5120 x 13824, 1777 rows, 1.5, 237 / 264.
//
// MX: W (and W2) are 4-bit weights; a half's W side is 128 columns x 32 bytes of codes, four copies, and a wave brings four copies of X and one of
// W.  A lane reads the 32 codes of one group of one column at once, so sub-step ks holds the inputs 32 (l / 32) + 8 ks .. + 7 on both sides, and
// turns eight of them into an operand by four conversions between the matrix instructions of the sub-step before.  The scales come sixteen bytes
// of a column at a time, for eight steps, into the ends of ring slots 0 and 1.  (A weight written out in bf16 first costs 20 us per 45 M values.)
// kBack: the codes of a step's 64 rows come as they lie, and each thread turns 64 of them into rows of bf16 in LDS, between the matrix instructions
// of the step before.
constexpr int kScaleAt = 24 * 1024, kScaleBytes = kTN * 16;
template <int MODE, bool MX>
__global__ void __launch_bounds__(kThreadsP, 1) prefill_kernel(PParams p) {
  constexpr bool GATED = MODE == kGated, BACK = MODE == kBack;
  constexpr bool HALVES = MODE != kPlain || MX;  // LoRA terms from prepared halves
  constexpr int kSites = MODE == kPlain ? 1 : 2;
  constexpr int kCopies = MX ? 5 : 8;  // of a half by a wave
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave & 1, wn = wave >> 1;

  // workgroup -> tile: workgroup ids go round-robin over the 8 XCDs; each XCD takes a contiguous run of the
  // tile order, which walks kGroupM row tiles per column tile so that the XCD's L2 serves the re-reads
  // (the 32 workgroups resident on an XCD then cover 4 row tiles x 8 column tiles)
  const int tiles = p.tilesM * p.tilesN;
  const int uncut = HALVES ? p.whole : tiles, total = BACK && p.S > 1 ? tiles * p.S : uncut;
  const int per = (total + 7) / 8;
  int id = (int)(blockIdx.x >> 3), part = 0, cut_tile = -1;
  if (id < per) {
    id += (int)(blockIdx.x & 7) * per;
    if (id >= total) return;
    if (BACK && p.S > 1) {
      part = id / tiles;
      id %= tiles;
    }
  } else {  // parts of the tiles that would fill the compute units for less than a turn; the same part of all of them first
    if (!HALVES) return;
    const int rest = tiles - uncut, units = rest * p.cut;
    id += (int)(blockIdx.x & 7) * ((units + 7) / 8) - per;
    if (id >= units) return;
    part = id / rest;
    cut_tile = id % rest;
    id = uncut + cut_tile;
  }
  const int gspan = kGroupM * p.tilesN;
  const int first = id / gspan * kGroupM;
  const int gsz = p.tilesM - first < kGroupM ? p.tilesM - first : kGroupM;
  const int in_group = id % gspan;
  const int64_t m0 = (int64_t)(first + in_group % gsz) * kTM;
  const int n0 = in_group / gsz * (GATED ? kTN / 2 : kTN);

  const int kt_of = HALVES ? (cut_tile >= 0 ? p.cut_steps : BACK && p.S > 1 ? p.steps : p.d1 / kTK) : p.d1 / kTK;
  const int kt0 = HALVES ? part * kt_of : 0;
  const int KT = HALVES && p.d1 / kTK - kt0 < kt_of ? p.d1 / kTK - kt0 : kt_of;
  const bool last_part = !HALVES || kt0 + KT == p.d1 / kTK;  // adds the LoRA terms
  const uint32_t lds0 = lds_addr(lds);

  // copies.  A k step of 64 is brought in two halves: half 0 = X rows 0..127 and W rows 0..127 of the tile,
  // half 1 = the other rows; a half is 8 + 8 blocks of 16 rows, a block two copy instructions of 8 rows each
  // (8 lanes take the 128-byte line of a row, so every request is for whole cache lines).  Waves 0,1 bring
  // the X blocks of a half (4 each), waves 2,3 the W blocks (GATED: wave 2 the gate's, wave 3 the up projection's).  Which 16 bytes of the line a lane takes is
  // permuted by the row so that the operand reads below spread over all LDS banks.
  const bool is_w = wave >= 2;
  const unsigned char* src = is_w ? (const unsigned char*)(GATED && wave == 3 ? p.W2 : p.W) : (const unsigned char*)p.X;
  const int64_t row0 = is_w ? (int64_t)n0 : m0;
  const int64_t rlim = is_w ? (int64_t)p.d2 : p.M;
  uint32_t voff[2][kCopies];
  if constexpr (MX) {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = wave * 4 + j, rr = lane >> 3;
        int64_t r = m0 + hh * 128 + i * 8 + rr;
        r = r < p.M ? r : p.M - 1;
        voff[hh][j] = (uint32_t)((uint64_t)r * (uint32_t)p.d1 * 2u + (uint32_t)((lane & 7) ^ swz((i & 1) * 8 + rr)) * 16u);
      }
      if constexpr (BACK) {  // 32 inputs of one of the step's 64 rows
        int n = n0 + hh * 128 + (tid & 3) * 32;
        n = n < p.d2 ? n : p.d2 - 32;
        voff[hh][4] = (uint32_t)(tid >> 2) * (uint32_t)(p.d2 >> 1) + (uint32_t)(n >> 1);
      } else {
        int n = GATED ? n0 + hh * 64 + (wave & 1) * 32 + (lane >> 1) : n0 + hh * 128 + wave * 32 + (lane >> 1);
        n = n < p.d2 ? n : p.d2 - 1;
        voff[hh][4] = (uint32_t)n * (uint32_t)(p.d1 >> 1) + (uint32_t)(lane & 1) * 16u;
      }
    }
  } else {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int rr = lane >> 3;
        const int block = GATED && is_w ? hh * 4 + (j >> 1) : hh * 8 + (wave & 1) * 4 + (j >> 1);
        int64_t r = row0 + block * 16 + (j & 1) * 8 + rr;
        r = r < rlim ? r : rlim - 1;
        voff[hh][j] = (uint32_t)((uint64_t)r * (uint32_t)p.d1 * 2u + (uint32_t)((lane & 7) ^ swz((j & 1) * 8 + rr)) * 16u);
        if (BACK && is_w) {  // four rows of 128 columns
          const int k = ((wave & 1) * 8 + j) * 4 + (lane >> 4);
          int n = n0 + hh * 128 + (((lane & 15) >> 1) ^ swz_tr(k)) * 16 + (lane & 1) * 8;
          n = n < p.d2 ? n : p.d2 - 8;  // past the edge: results dropped
          voff[hh][j] = (uint32_t)k * (uint32_t)p.d2 * 2u + (uint32_t)n * 2u;
        }
      }
  }
  // (BACK: the second half of the reduction is the second weight's; of a step's 64 rows wave 2 brings the first 32, wave 3 the others, and the
  // halves meet at a multiple of 32)
  const int second_at = BACK && is_w ? p.d1 / 2 - (wave & 1) * 32 : 0x7fffffff;
  const unsigned char* const src2 = BACK && is_w ? (const unsigned char*)p.W2 - (size_t)(p.d1 / 2) * p.d2 * 2 : src;
  const size_t k_bytes = BACK && is_w ? (size_t)kTK * p.d2 * 2 : kTK * 2;
  const uint32_t dst_in_half = (uint32_t)((is_w ? 8 : 0) + (wave & 1) * 4) * kBlockBytes;
  // half H = 2 * (k step) + hh lives in ring slot H % kHalves
  // copy j (0..7) of a half; a wave's eight copies of a half are spread between its matrix instructions: issued
  // back to back they would hold the wave at the issue of the memory instructions while the matrix cores idle
  const unsigned char* const codes = (const unsigned char*)(GATED && wave >= 2 ? p.W2 : p.W);  // (MX) of this wave's copies
  auto issue_one = [&](int kt, int hh, int slot, int j) __attribute__((always_inline)) {
    if constexpr (MX) {
      const int kk = kt0 + (kt < KT ? kt : KT - 1);
      if (j < 4) copy_to_lds16((const unsigned char*)p.X + (size_t)kk * (kTK * 2), voff[hh][j], lds0 + slot * kHalfBytes + (wave * 4 + j) * 1024);
      else copy_to_lds16(codes + (size_t)kk * 32, voff[hh][4], lds0 + slot * kHalfBytes + (kBlocksM / 2) * kBlockBytes + wave * 1024);
      return;
    }
    const int kk = kt0 + (kt < KT ? kt : KT - 1);  // past the end: re-read the last step into a slot nobody reads
    const unsigned char* b = (BACK && kk * kTK >= second_at ? src2 : src) + (size_t)kk * (BACK ? k_bytes : kTK * 2);
    const uint32_t dst = lds0 + slot * kHalfBytes + dst_in_half;
    copy_to_lds16(b, voff[hh][j], dst + j * 1024);
  };
  // (MX) scales of steps 8 gr .. + 7 of the tile's 256 columns, 64 of them by a wave; the last sixteen bytes of a column where it ends sooner
  const int scale_bytes = p.d1 >> 5;
  auto issue_scales = [&](int gr) __attribute__((always_inline)) {
    const unsigned char* const w = (const unsigned char*)(GATED && (wave & 1) ? p.W2 : p.W) + (size_t)p.d1 * p.d2 / 2;
    int n = GATED ? n0 + (wave >> 1) * 64 + lane : n0 + wave * 64 + lane;
    n = n < p.d2 ? n : p.d2 - 1;
    const int at = gr * 16 < scale_bytes - 16 ? gr * 16 : scale_bytes - 16;
    copy_to_lds16(w + at, (uint32_t)n * (uint32_t)scale_bytes, lds0 + (gr & 1) * kHalfBytes + kScaleAt + wave * 1024);
  };
  auto issue = [&](int kt, int hh, int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kCopies; ++j) issue_one(kt, hh, slot, j);
  };

  // (MX && BACK) the codes of a step as they lie, and their scales: a thread brings, and later turns into operands, 32 inputs of one row in
  // each half; the scales of a wave's 16 rows, four bytes a half, by its first 32 lanes.  A wave's rows lie in one weight (F % 32 == 0).
  constexpr int kRawAt = 4 * kHalfBytes, kRawScaleAt = kRawAt + 16 * 1024;
  const uint32_t sv = (uint32_t)(wave * 16 + ((lane >> 1) & 15)) * (uint32_t)(p.d2 >> 5) + (uint32_t)(n0 >> 5) + (n0 + (lane & 1) * 128 < p.d2 ? (lane & 1) * 4u : 0u);
  auto issue_raw = [&](int kt, int j) __attribute__((always_inline)) {
    const int kk = kt0 + (kt < KT ? kt : KT - 1), F = p.d1 >> 1;
    const bool second = kk * kTK + wave * 16 >= F;
    const unsigned char* const w = (const unsigned char*)(second ? p.W2 : p.W);
    const int64_t row = (int64_t)kk * kTK - (second ? F : 0);
    if (j < 2) copy_to_lds16(w + row * (p.d2 >> 1), voff[j][kCopies - 1], lds0 + kRawAt + (kt & 1) * 8192 + j * 4096 + wave * 1024);
    else copy_to_lds4(w + (size_t)F * p.d2 / 2 + row * (p.d2 >> 5), sv, lds0 + kRawScaleAt + (kt & 1) * 1024 + wave * 256);
  };
  u32x4 raw[2];
  float raw_scale[2];
  auto read_raw = [&](int kt) __attribute__((always_inline)) {
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      raw[hh] = *(const u32x4*)(lds + kRawAt + (kt & 1) * 8192 + hh * 4096 + tid * 16);
      raw_scale[hh] = mx4_scale(lds[kRawScaleAt + (kt & 1) * 1024 + wave * 256 + ((lane >> 2) * 2 + hh) * 4 + (lane & 3)]);
    }
  };
  // eight inputs (of group i = 4 half + u) of row tid / 4 to where a copied row has them; odd rows the other sixteen bytes of a piece first, so that
  // the rows that a cycle writes lie on all banks
  auto put_raw = [&](int kt, int i) __attribute__((always_inline)) {
    const int k = tid >> 2, odd = k & 1, hh = i >> 2, v = (i >> 1) & 1, e = i & 1;
    const uint32_t c = odd ? raw[hh][2 * v + 1 - e] : raw[hh][2 * v + e];
    const int piece = (lane & 3) * 2 + v;
    *(u32x4*)(lds + (2 * (kt & 1) + hh) * kHalfBytes + (kBlocksM / 2) * kBlockBytes + k * 256 + ((piece ^ swz_tr(k)) & 7) * 32 + (e ^ odd) * 16) =
        mx4_bf16(c, raw_scale[hh]);
  };

  int2 lora[kSites];  // (HALVES) of row tid, at the sites
#pragma unroll
  for (int s = 0; s < kSites; ++s) lora[s] = int2{-1, 0};
  if (HALVES && m0 + tid < p.M && last_part)
#pragma unroll
    for (int s = 0; s < kSites; ++s) lora[s] = p.row_lora[s * p.lora_site + p.row_base + m0 + tid];

  // acc[i][j]: rows 32 i .. 32 i + 31 of the wave's X part against rows 32 j .. of its W part
  f32x16 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // operand read: lane l takes row l % 32 of a pair of 16-row blocks and the 16 bytes of k group 2 ks + l / 32
  // (ks = 0..3: the four 16-k sub-steps of a block's 64 k)
  const int rrow = lane & 31;
  int rd[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks)
    rd[ks] = (rrow >> 4) * kBlockBytes + (rrow & 15) * 128 + (((2 * ks + (lane >> 5)) ^ swz(rrow & 15)) << 4);
  const unsigned char* wbase = lds + (kBlocksM / 2) * kBlockBytes;
  uint32_t rd_tr[4];  // (BACK) of the columns 32 j .., rows 8 (l / 32) .. of a sub-step
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int k = (lane >> 5) * 8 + ((lane & 15) >> 2);
    rd_tr[j] = lds0 + (kBlocksM / 2) * kBlockBytes + k * 256 + (((2 * j + ((lane >> 4) & 1)) ^ swz_tr(k)) & 7) * 32 + (lane & 3) * 8;
  }
  // One k step of 64 for the wave's 128 x 128 part: 64 matrix instructions, number q = 16 ks + 4 i + j.  The
  // operand reads come early: the sixteen of the first two sub-steps, then the other sixteen between the matrix
  // instructions of the first sub-step.  `mid` runs after instruction 15, once every wave of the workgroup has
  // its operands in registers: the step's two ring slots are free from there on.  copy(q) runs after instruction q.
  auto mma64 = [&](auto tr, int slot_x, int slot_w, auto mid, auto copy) __attribute__((always_inline)) {
    const unsigned char* sa = lds + slot_x * kHalfBytes;
    const unsigned char* sb = wbase + slot_w * kHalfBytes;
    const uint32_t tb = slot_w * kHalfBytes;
    bf16x8 a[4][4], b[4][4];
    auto read_w = [&](int ks, int j) __attribute__((always_inline)) {
      if constexpr (decltype(tr)::value) return read_tr(rd_tr[j] + tb + ks * 4096);
      else return *(const bf16x8*)(sb + rd[ks] + j * 2 * kBlockBytes);
    };
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[ks][i] = *(const bf16x8*)(sa + rd[ks] + i * 2 * kBlockBytes);
#pragma unroll
      for (int j = 0; j < 4; ++j) b[ks][j] = read_w(ks, j);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      acc[q >> 2][q & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[0][q & 3], a[0][q >> 2], acc[q >> 2][q & 3], 0, 0, 0);
      const int ks = 2 + (q >> 3), e = q & 3;
      if (q & 4) b[ks][e] = read_w(ks, e);
      else a[ks][e] = *(const bf16x8*)(sa + rd[ks] + e * 2 * kBlockBytes);
      copy(q);
      __builtin_amdgcn_sched_barrier(0);
    }
    mid();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 16; q < 64; ++q) {
      acc[(q >> 2) & 3][q & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[q >> 4][q & 3], a[q >> 4][(q >> 2) & 3],
                                                                         acc[(q >> 2) & 3][q & 3], 0, 0, 0);
      copy(q);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // (MX) the same for a step whose W side are codes
  int rdx[4];
  if constexpr (MX)
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
      rdx[ks] = (rrow >> 4) * kBlockBytes + (rrow & 15) * 128 + ((((lane >> 5) * 4 + ks) ^ swz(rrow & 15)) << 4);
  auto mma64_mx = [&](int slot_x, int slot_w, const unsigned char* scales, auto mid, auto copy) __attribute__((always_inline)) {
    const unsigned char* sa = lds + slot_x * kHalfBytes;
    const unsigned char* sb = wbase + slot_w * kHalfBytes + rrow * 32 + (lane >> 5) * 16;
    bf16x8 a[4][4], b[4][4];
    u32x4 c[4];
    float scale[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[j] = *(const u32x4*)(sb + j * 1024);
      scale[j] = mx4_scale(scales[j * 512]);
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 4; ++i) a[ks][i] = *(const bf16x8*)(sa + rdx[ks] + i * 2 * kBlockBytes);
#pragma unroll
    for (int j = 0; j < 4; ++j) b[0][j] = __builtin_bit_cast(bf16x8, mx4_bf16(c[j][0], scale[j]));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 64; ++q) {
      const int ks = q >> 4;
      acc[(q >> 2) & 3][q & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[ks][q & 3], a[ks][(q >> 2) & 3], acc[(q >> 2) & 3][q & 3], 0, 0, 0);
      if (q < 16 && !(q & 1)) a[2 + (q >> 3)][(q >> 1) & 3] = *(const bf16x8*)(sa + rdx[2 + (q >> 3)] + ((q >> 1) & 3) * 2 * kBlockBytes);
      if (ks < 3 && (q & 3) == 1) b[ks + 1][(q >> 2) & 3] = __builtin_bit_cast(bf16x8, mx4_bf16(c[(q >> 2) & 3][ks + 1], scale[(q >> 2) & 3]));
      copy(q);
      __builtin_amdgcn_sched_barrier(0);
      if (q == 15) {
        mid();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  if constexpr (BACK && MX) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int j = 0; j < 3; ++j) issue_raw(kt, j);
#pragma unroll
      for (int j = 0; j < 8; ++j) issue_one(kt, j >> 2, 2 * kt + (j >> 2), j & 3);
    }
    wait_vm<19>();  // codes and scales of the first step
    asm volatile("" ::: "memory");
    read_raw(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) put_raw(0, i);
  } else {
  if constexpr (MX) issue_scales(kt0 >> 3);  // (a part begins with a multiple of eight steps)
  issue(0, 0, 0);
  issue(0, 1, 1);
  issue(1, 0, 2);
  issue(1, 1, 3);
  }
  // 12 of the 16 accumulator tiles in the accumulation registers, 4 in ordinary ones: with all 256 in the
  // accumulation file the compiler has no spare tile there and shuffles tiles between the files in the loop
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (i < kAccTilesRows) asm volatile("" : "+a"(acc[i][j]));
      else asm volatile("" : "+v"(acc[i][j]));
    }
  if constexpr (BACK && MX) {
    // Slots 2 b and 2 b + 1 hold a step of parity b, slot 4 codes and scales of two steps.  In step kt: codes of kt + 2 are asked for before its
    // operands are out; behind that those of kt + 1, asked for a step ago, are turned into its W side, and X of kt + 2 is asked for.  Both waits
    // leave the eleven copies issued since out.
    for (int kt = 0; kt < KT; ++kt) {
      wait_vm<11>();                       // X of this step (behind it: codes of kt + 1, X of kt + 1)
      __builtin_amdgcn_s_waitcnt(0xc07f);  // this wave's part of its W side
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      auto mid = [&]() __attribute__((always_inline)) {
        wait_vm<11>();                       // codes of kt + 1 (behind them: X of kt + 1, codes of kt + 2)
        __builtin_amdgcn_s_waitcnt(0xc07f);  // operand reads have returned
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      };
      auto copy = [&](int q) __attribute__((always_inline)) {
        if (q < 15 && q % 5 == 0) issue_raw(kt + 2, q / 5);
        if (q == 16) read_raw(kt + 1);
        if (q >= 20 && q < 60 && q % 5 == 0) issue_one(kt + 2, (q - 20) / 20, 2 * (kt & 1) + (q - 20) / 20, (q - 20) / 5 % 4);
        if (q >= 22 && q < 62 && q % 5 == 2) put_raw(kt + 1, (q - 22) / 5);
      };
      const int b = 2 * (kt & 1);
      mma64(std::integral_constant<bool, BACK>{}, b + wm, b + wn, mid, copy);
      asm volatile("" ::: "memory");
    }
  } else {
  // The ring: halves 2 kt and 2 kt + 1 (this step) are read, the two of the next step are on their way, the
  // fifth slot takes the first half of the step after next at once and the second half goes into this step's
  // first slot as soon as every wave has taken its operands out: a copy has between one and three quarters and
  // two whole steps of matrix work to arrive.
  int h0 = 0;  // ring slot of half 0 of the current step
  for (int kt = 0; kt < KT; ++kt) {
    const int h1 = h0 + 1 >= kHalves ? h0 + 1 - kHalves : h0 + 1;
    const int h2 = h0 + 2 >= kHalves ? h0 + 2 - kHalves : h0 + 2;
    const int h4 = h0 + 4 >= kHalves ? h0 + 4 - kHalves : h0 + 4;
    wait_vm<2 * kCopies>();         // all but the two halves issued last have landed: both halves of this step
    __builtin_amdgcn_s_barrier();   // for every wave
    asm volatile("" ::: "memory");
    if (MX && (kt & 7) == 0 && kt + 8 < KT) issue_scales(((kt0 + kt) >> 3) + 1);
    auto mid = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): this wave's operand reads have returned
      __builtin_amdgcn_s_barrier();        // and every other wave's
      asm volatile("" ::: "memory");
    };
    // first half of the step after next into the free slot, second half into this step's first slot
    auto copy = [&](int q) __attribute__((always_inline)) {
      if (q < kCopyB0) {
        if (q % kCopyAStride == 0 && q / kCopyAStride < kCopies) issue_one(kt + 2, 0, h4, q / kCopyAStride);
      } else if ((q - kCopyB0) % kCopyBStride == 0 && (q - kCopyB0) / kCopyBStride < kCopies) {
        issue_one(kt + 2, 1, h0, (q - kCopyB0) / kCopyBStride);
      }
    };
    if constexpr (MX) {
      const int gr = (kt0 + kt) >> 3, from = gr * 16 < scale_bytes - 16 ? gr * 16 : scale_bytes - 16;
      mma64_mx(wm ? h1 : h0, wn ? h1 : h0,
               lds + (gr & 1) * kHalfBytes + kScaleAt + (wn * 128 + rrow) * 16 + (kt0 + kt) * 2 + (lane >> 5) - from, mid, copy);
    } else {
      mma64(std::integral_constant<bool, BACK>{}, wm ? h1 : h0, wn ? h1 : h0, mid, copy);
    }
    asm volatile("" ::: "memory");
    h0 = h2;
  }
  }
  wait_vm<0>();
  __syncthreads();

  // ---- LoRA term of the routed rows as one more k step per 32 ranks, two of them filled together ------------
  // t = X W^A (fp32) goes in as bf16 hi + lo: hi in the first k half of a block, lo in the second, against the
  // same 32 rows of the tenant's W^B in both halves; rows of other tenants and unrouted rows enter as zeros.  Bound by the
  // instructions of filling a step: W^B in pieces of 8 ranks x 8 columns, 16-byte loads turned with byte permutes, t four ranks of
  // a row at a time straight into its two halves; and by the round trips to t, about 3 us each (32 loads of two bytes a thread,
  // t by way of LDS, one step at a time: a call of 777 rows on 4096 x 11008 with a tenant of rank 64 131 us, 120 so, 97 without).
  int* ctl = (int*)(lds + 4 * kHalfBytes);  // ring slots 0 .. 3 hold the operand blocks
  int* const row_ten = ctl + 16;            // tenant of each row of the tile, -1: no LoRA term
  if (tid == 0) ctl[1] = 0;  // set: a matrix of some tenant of the tile holds Inf or NaN
  if constexpr (!HALVES) {
  int my_ten = -1;
  {
    const int64_t m = m0 + tid;
    if (m < p.M) {
      const int64_t req = p.row_to_req ? (int64_t)p.row_to_req[m] : p.row_base + m;
      int tenant = 0;
      const int r = (req >= 0 && req < p.B) ? routed_rank(p.ad, p.tenant_id, p.route, (int)req, p.B, p.site, &tenant) : 0;
      if (r) my_ten = tenant;
    }
  }
  row_ten[tid] = my_ten;
  int last = -1;
  for (;;) {
    if (tid == 0) ctl[0] = 0x7fffffff;
    __syncthreads();
    int cand = my_ten > last ? my_ten : 0x7fffffff;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_xor(cand, off, 64);
      cand = o < cand ? o : cand;
    }
    if (lane == 0) atomicMin(&ctl[0], cand);
    __syncthreads();
    const int cur = ctl[0];
    if (cur == 0x7fffffff) break;
    const int r = p.ad.rank[cur];
    gbf16* Bm = in_global(p.ad.B[cur * MILORA_NUM_SITES + p.site]);
    for (int c0 = 0; c0 < r; c0 += 64) {
      int tb = tid;  // opaque: addresses formed from it stay inside the loop instead of being spilled in front of it
      asm volatile("" : "+v"(tb));
      const int steps = r - c0 > 32 ? 2 : 1;
      // W side: ranks c0 + 8 gq .. + 7 of columns 8 pc .. + 7, asked for first, used last
      const int pc = tb & 31, gq = tb >> 5, cw = c0 + gq * 8;
      const bool wput = gq < steps * 4;
      u32x4 a[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = u32x4{0u, 0u, 0u, 0u};
      if (wput && n0 + pc * 8 < p.d2) {
        gbf16* b = Bm + (size_t)cw * p.d2 + n0 + pc * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (cw + i < r) a[i] = *(gu32x4_a2*)(b + (size_t)i * p.d2);  // (whole pieces of 8 columns, d2 % 16 == 0, at any alignment)
      }
      // X side: eight lanes take 32 ranks of a row, the shrink's parts added in part order
      const int rq = tb & 7;
      for (int st = 0; st < steps; ++st) {
        const int cq = c0 + st * 32 + rq * 4;
        const bool vec = (p.ad.r_max & 3) == 0 && cq + 3 < p.ad.r_max;
#pragma unroll 1
        for (int i0 = 0; i0 < 8; i0 += 4) {
          f32x4 v[4];
          const float* q[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int64_t mr = m0 + (tb >> 3) + 32 * (i0 + i);
            q[i] = p.t + (size_t)(mr < p.M ? mr : p.M - 1) * p.ad.r_max + cq;
          }
          if (vec) {
            for (int k0 = 0; k0 < p.parts; k0 += 4) {  // four rows and four parts in flight
              f32x4 x[4][4];
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  x[k][i] = *reinterpret_cast<const f32x4*>(q[i] + (k0 + k < p.parts ? k0 + k : p.parts - 1) * p.t_stride);
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (k0 + k < p.parts)
#pragma unroll
                  for (int i = 0; i < 4; ++i) v[i] += x[k][i];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (cq + e < p.ad.r_max)
                  for (int part = 0; part < p.parts; ++part) v[i][e] += q[i][part * p.t_stride + e];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = (tb >> 3) + 32 * (i0 + i);
            const bool ours = row_ten[row] == cur;
            float tv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) tv[e] = ours && cq + e < r ? v[i][e] : 0.f;
            u32x2 hi, lo;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              hi[h] = pack_bf16x2(tv[2 * h], tv[2 * h + 1]);
              lo[h] = pack_bf16x2(rest_of(tv[2 * h], __uint_as_float(hi[h] << 16)), rest_of(tv[2 * h + 1], __uint_as_float(hi[h] & 0xffff0000u)));
            }
            unsigned char* const x = lds + (2 * st + (row >> 7)) * kHalfBytes + ((row >> 4) & 7) * kBlockBytes + (row & 15) * 128 + (rq & 1) * 8;
            *(u32x2*)(x + (((rq >> 1) ^ swz(row & 15)) << 4)) = hi;
            *(u32x2*)(x + ((((rq >> 1) + 4) ^ swz(row & 15)) << 4)) = lo;
          }
        }
      }
      if (wput) {
        float bad[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) bad[e] = taint(bad[e], a[i][e]);
        if ((bad[0] + bad[1]) + (bad[2] + bad[3]) != 0.f) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) a[i][e] = finite2(a[i][e]);
          ctl[1] = 1;
        }
        u32x4 at[8];
        transpose8(a, at);
        // (columns 8 pc .. + 7: one half of a block of 16)
        unsigned char* const wst = lds + (2 * (gq >> 2) + (pc >> 4)) * kHalfBytes + (kBlocksM / 2 + ((pc >> 1) & 7)) * kBlockBytes;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int n = (pc & 1) * 8 + j;
          *(u32x4*)(wst + n * 128 + (((gq & 3) ^ swz(n)) << 4)) = at[j];
          *(u32x4*)(wst + n * 128 + ((((gq & 3) + 4) ^ swz(n)) << 4)) = at[j];
        }
      }
      __syncthreads();
      for (int st = 0; st < steps; ++st) mma64(std::false_type{}, 2 * st + wm, 2 * st + wn, []() {}, [](int) {});
      __syncthreads();
    }
    last = cur;
  }
  } else {
    // The same for two sites, from the halves prepared in front of the launch: a line of them is a row of a step as it lies, copied straight into
    // LDS, the zero line for rows of other tenants; one round trip for 64 ranks of a tenant (with the shrinks' parts added and split here,
    // 777 rows of 5 requests, three sites each, ranks 8 to 64, gated block of 4096 x 11008: 287 us a call).  32 rows of W^B go in as they lie,
    // [k][column], and are read transposed; kGated: the columns of the other projection are zero.  kBack: eight ranks of a column are eight consecutive
    // values of W^A.
#pragma unroll 1
    for (int s = 0; s < kSites; ++s) {
      const int my_ten = lora[s].y ? lora[s].x : -1;
      const bool later = (lora[s].y & kLaterBit) != 0;
      row_ten[tid] = my_ten;  // (of the site before: read for the last time in front of a barrier)
      int last = -1;
      for (;;) {
        if (tid == 0) ctl[0] = 0x7fffffff;
        __syncthreads();
        if (later) ctl[1] = 1;
        int cand = my_ten > last ? my_ten : 0x7fffffff;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const int o = __shfl_xor(cand, off, 64);
          cand = o < cand ? o : cand;
        }
        if (lane == 0) atomicMin(&ctl[0], cand);
        __syncthreads();
        const int cur = __builtin_amdgcn_readfirstlane(ctl[0]);
        if (cur == 0x7fffffff) break;
        const int r = p.ad.rank[cur];
        gbf16* const Wm = in_global((BACK ? p.ad.A : p.ad.B)[cur * MILORA_NUM_SITES + p.site + s]);
        const bool vec_a = (r & 7) == 0 && ((uintptr_t)Wm & 15) == 0;
        for (int c0 = 0; c0 < r; c0 += 64) {
          int tb = tid;  // opaque: addresses formed from it stay inside the loop instead of being spilled in front of it
          asm volatile("" : "+v"(tb));
          const int steps = r - c0 > 32 ? 2 : 1;
          // X side: eight copies of a step by each wave, eight rows each
          for (int st = 0; st < steps; ++st) {
            const bf16_t* const lines = p.halves + s * p.half_site + (size_t)((c0 >> 5) + st) * p.half_chunk;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int q = wave * 8 + j, i = q & 15, row = (q >> 4) * 128 + i * 8 + ((tb & 63) >> 3);
              const uint32_t line = row_ten[row] == cur ? (uint32_t)(p.row_base + m0 + row + 1) : 0u;
              copy_to_lds16(lines, line * 128u + (uint32_t)((tb & 7) ^ swz(row & 15)) * 16u, lds0 + (2 * st + (q >> 4)) * kHalfBytes + i * 1024);
            }
          }
          // W side
          u32x4 a[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] = u32x4{0u, 0u, 0u, 0u};
          const int pc = tb & 31, gq = tb >> 5;  // kBack: columns 8 pc .. + 7, ranks c0 + 8 gq .. + 7
          if constexpr (BACK) {
            const int cw = c0 + gq * 8;
            if (gq < steps * 4 && n0 + pc * 8 < p.d2 && cw < r)
#pragma unroll
              for (int i = 0; i < 8; ++i) a[i] = load8(Wm + (size_t)(n0 + pc * 8 + i) * r + cw, r - cw, vec_a);
          } else if constexpr (GATED) {  // rank c0 + 32 (i / 2) + .., eight columns of the site: 512 pieces of a step, two a thread
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int e = (i & 1) * 256 + tb, c = c0 + (i >> 1) * 32 + (e >> 4), n = n0 + (e & 15) * 8;
              if ((i >> 1) < steps && c < r && n < p.d2) a[i] = *(gu32x4_a2*)(Wm + (size_t)c * p.d2 + n);
            }
          } else {  // 1024 pieces of a step, four a thread
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int e = (i & 3) * 256 + tb, c = c0 + (i >> 2) * 32 + (e >> 5), n = n0 + (e & 31) * 8;
              if ((i >> 2) < steps && c < r && n < p.d2) a[i] = *(gu32x4_a2*)(Wm + (size_t)c * p.d2 + n);
            }
          }
          float taints[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < (GATED ? 4 : 8); ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) taints[e] = taint(taints[e], a[i][e]);
          if ((taints[0] + taints[1]) + (taints[2] + taints[3]) != 0.f) {
#pragma unroll
            for (int i = 0; i < (GATED ? 4 : 8); ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) a[i][e] = finite2(a[i][e]);
            ctl[1] = 1;
          }
          if constexpr (BACK) {
            if (gq < steps * 4) {
              unsigned char* const wst = lds + (2 * (gq >> 2) + (pc >> 4)) * kHalfBytes + (kBlocksM / 2 + ((pc >> 1) & 7)) * kBlockBytes;
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int n = (pc & 1) * 8 + i;
                *(u32x4*)(wst + n * 128 + (((gq & 3) ^ swz(n)) << 4)) = a[i];
                *(u32x4*)(wst + n * 128 + ((((gq & 3) + 4) ^ swz(n)) << 4)) = a[i];
              }
            }
          } else if constexpr (!GATED) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              if ((i >> 2) >= steps) continue;
              const int e = (i & 3) * 256 + tb, k = e >> 5, cp = e & 31;
              unsigned char* const wst = lds + (2 * (i >> 2) + (cp >> 4)) * kHalfBytes + (kBlocksM / 2) * kBlockBytes + (cp & 1) * 16;
#pragma unroll
              for (int h = 0; h < 2; ++h) *(u32x4*)(wst + (k + 32 * h) * 256 + ((((cp & 15) >> 1) ^ swz_tr(k)) & 7) * 32) = a[i];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if ((i >> 1) >= steps) continue;
              // columns 8 (e % 16) of the site: half (e % 16) / 8, piece of 16 columns there: 4 s + ((e % 16) % 8) / 2
              const int e = (i & 1) * 256 + tb, k = e >> 4, cp = e & 15;
              unsigned char* const wst = lds + (2 * (i >> 1) + (cp >> 3)) * kHalfBytes + (kBlocksM / 2) * kBlockBytes + (cp & 1) * 16;
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                unsigned char* const line = wst + (k + 32 * h) * 256;
                *(u32x4*)(line + (((4 * s + ((cp & 7) >> 1)) ^ swz_tr(k)) & 7) * 32) = a[i];
                *(u32x4*)(line + (((4 * (1 - s) + ((cp & 7) >> 1)) ^ swz_tr(k)) & 7) * 32) = u32x4{0u, 0u, 0u, 0u};
              }
            }
          }
          wait_vm<0>();
          __syncthreads();
          for (int st = 0; st < steps; ++st) mma64(std::integral_constant<bool, !BACK>{}, 2 * st + wm, 2 * st + wn, []() {}, [](int) {});
          __syncthreads();
        }
        last = cur;
      }
    }
  }

  // ---- a cut tile: the workgroup that is done last adds the others' sums to its own, in part order, and goes on; it waits only for workgroups
  // that are already writing theirs, and no longer than milora_set_wait_limit() says (counters that somebody else writes, two calls on one workspace
  // at once): the tile is NaN then ----
  if constexpr (HALVES) {
    if (cut_tile >= 0) {
      int* const cnt = p.cut_cnt + 2 * cut_tile;
      __syncthreads();
      if (tid == 0) ctl[2] = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      typedef unsigned long long two_floats;  // (stores and loads of eight bytes past the caches of an XCD)
      two_floats* const sums = (two_floats*)p.cut_sums + (size_t)cut_tile * p.cut * (kTM * kTN / 2) + tid;
      if (ctl[2] != p.cut - 1) {
        two_floats* const to = sums + (size_t)part * (kTM * kTN / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const f32x2 v = {acc[i][j][2 * e], acc[i][j][2 * e + 1]};
              __hip_atomic_store(to + ((i * 4 + j) * 8 + e) * kThreadsP, __builtin_bit_cast(two_floats, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0) __hip_atomic_fetch_add(cnt + 1, ctl[1] ? 0x10001 : 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return;
      }
      if (tid == 0) {
        int done, polls = p.polls;
        while (((done = __hip_atomic_load(cnt + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) & 0xffff) != p.cut - 1 && --polls > 0) __builtin_amdgcn_s_sleep(2);
        ctl[3] = (done & 0xffff) != p.cut - 1;
        if (done >> 16) ctl[1] = 1;
        __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next launch
        __hip_atomic_store(cnt + 1, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j0 = 0; j0 < 4; j0 += 4) {
          f32x2 sum[32];
          for (int k = 0; k < p.cut; ++k) {
            f32x2 v[32];
            if (k == part) {
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] = f32x2{acc[i][j0 + (e >> 3)][2 * (e & 7)], acc[i][j0 + (e >> 3)][2 * (e & 7) + 1]};
            } else {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                v[e] = __builtin_bit_cast(f32x2, __hip_atomic_load(sums + ((size_t)k * 128 + (i * 4 + j0) * 8 + e) * kThreadsP, __ATOMIC_RELAXED,
                                                                   __HIP_MEMORY_SCOPE_AGENT));
            }
#pragma unroll
            for (int e = 0; e < 32; ++e)
#pragma unroll
              for (int h = 0; h < 2; ++h) sum[e][h] = k ? sum[e][h] + v[e][h] : v[e][h];
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            acc[i][j0 + (e >> 3)][2 * (e & 7)] = sum[e][0];
            acc[i][j0 + (e >> 3)][2 * (e & 7) + 1] = sum[e][1];
          }
        }
      if (__builtin_amdgcn_readfirstlane(ctl[3])) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = __builtin_nanf("");
      }
    }
  }

  // ---- bias, one rounding, store: of a 32 x 32 tile a lane holds row l % 32 and, in registers 4 g .. 4 g + 3, the
  // columns 8 g + 4 (l / 32) .. + 3.  By way of the wave's own LDS, so that a store writes whole lines (256 bytes of four rows instead
  // of 16 bytes of 32 rows, lines that had to be read before they could be written: seven linears of 32768 rows 11.43 -> 10.79 ms), and
  // past the L2's lines of X and W (10.80 -> 10.57 ms).  Also where results are small and read soon: us with all of them past the L2 /
  // those below 64 MB through it / 16 bytes of 32 rows a store, 777 rows of 4096 x 11008: up alone 84.5 / 85.3 / 93.7, up and the down
  // that reads it 182 / 170 / 184, gate, up, their product and down 262 / 263 / 285; the same with every row routed 102.0 / 103.5 /
  // 115.5, 204 / 205 / 223, 316 / 318 / 350; up of 1805 rows of 192 x 7488, every row routed, 30.7 / 33.6 / 45.9.
  const bool bad = ctl[1] != 0;
  __syncthreads();
  unsigned char* const mine = lds + wave * (128 * kOutPitch);
  if constexpr (GATED) {
    // What the stages could not take (products of the tenant's own Inf and NaN) has to be in g and u before the activation: formed
    // row by row in the wave's LDS, 64 columns at a time, and added.
    if (bad) {
#pragma unroll 1
      for (int s = 0; s < 2; ++s) {
        for (int row = lane; row < 128; row += 64) {
          float* const more = (float*)(mine + row * kOutPitch);
          for (int n = 0; n < 64; ++n) more[n] = 0.f;
          const int64_t m = m0 + wm * 128 + row;
          if (m >= p.M) continue;
          const int64_t req = p.row_to_req ? (int64_t)p.row_to_req[m] : p.row_base + m;
          int tenant = 0;
          const int r = (req >= 0 && req < p.B) ? routed_rank(p.ad, p.tenant_id, p.route, (int)req, p.B, p.site + s, &tenant) : 0;
          for (int c = 0; c < r; ++c) {
            gbf16* b = in_global(p.ad.B[tenant * MILORA_NUM_SITES + p.site + s]) + (size_t)c * p.d2;
            float t = 0.f;
            for (int k = 0; k < p.parts; ++k) t += p.t[s * p.t_site + k * p.t_stride + (size_t)m * p.ad.r_max + c];
            for (int q = 0; q < 64; ++q) {
              const int n = n0 + wn * 64 + q;
              if (n < p.d2 && ((b[n] & 0x7f80u) == 0x7f80u || !finite_f32(t))) more[q] += t * bf16_to_f32(b[n]);
            }
          }
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if ((j >> 1) == s)
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const f32x4 v = *(const f32x4*)(mine + (i * 32 + (lane & 31)) * kOutPitch + ((j & 1) * 32 + g * 8 + (lane >> 5) * 4) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] += v[e];
              }
        __builtin_amdgcn_s_waitcnt(0xc07f);
        asm volatile("" ::: "memory");
      }
    }
  }
  if constexpr (MODE != kPlain) {
    // 64 columns of the wave's sums in fp32, whole lines of four rows a store
    auto save = [&](int s, float* to, int col0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *(f32x4*)(mine + (i * 32 + (lane & 31)) * kOutPitch + (j * 32 + g * 8 + (lane >> 5) * 4) * 4) =
                f32x4{acc[i][2 * s + j][4 * g], acc[i][2 * s + j][4 * g + 1], acc[i][2 * s + j][4 * g + 2], acc[i][2 * s + j][4 * g + 3]};
      __builtin_amdgcn_s_waitcnt(0xc07f);
      asm volatile("" ::: "memory");
      const int n = col0 + (lane & 15) * 4;
      const int64_t mw = m0 + wm * 128 + (lane >> 4);
      const unsigned char* q = mine + (lane >> 4) * kOutPitch + (lane & 15) * 16;
      if (n < p.d2)
#pragma unroll 4
        for (int it = 0; it < 32; ++it)
          if (mw + it * 4 < p.M)
            __builtin_nontemporal_store(*(const f32x4*)(q + it * 4 * kOutPitch), (f32x4_a4*)(to + (size_t)(mw + it * 4) * p.d2 + n));
      __builtin_amdgcn_s_waitcnt(0xc07f);
      asm volatile("" ::: "memory");
    };
    if constexpr (BACK) {
      if (p.S > 1) {
        float* const mine_out = p.partial + part * p.partial_stride;
        save(0, mine_out, n0 + wn * 128);
        save(1, mine_out, n0 + wn * 128 + 64);
      }
    } else {
      if (p.gate_out) save(0, p.gate_out, n0 + wn * 64);  // g and u as they are, for a backward pass
      if (p.up_out) save(1, p.up_out, n0 + wn * 64);
    }
  }
  if constexpr (GATED) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x2 v;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            v[h] = pack_bf16x2(silu(acc[i][j][4 * g + 2 * h]) * acc[i][j + 2][4 * g + 2 * h],
                               silu(acc[i][j][4 * g + 2 * h + 1]) * acc[i][j + 2][4 * g + 2 * h + 1]);
          *(u32x2*)(mine + (i * 32 + (lane & 31)) * kOutPitch + (j * 32 + g * 8 + (lane >> 5) * 4) * 2) = v;
        }
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
    const int n = n0 + wn * 64 + (lane & 7) * 8;
    const int64_t mw = m0 + wm * 128 + (lane >> 3);
    bf16_t* y = p.Y + (size_t)mw * p.d2 + n;
    const unsigned char* q = mine + (lane >> 3) * kOutPitch + (lane & 7) * 16;
    if (n < p.d2)
#pragma unroll 4
      for (int it = 0; it < 16; ++it)
        if (mw + it * 8 < p.M) {
          const u32x4_a8 v = *(const u32x4*)(q + it * 8 * kOutPitch);
          __builtin_nontemporal_store(v, (u32x4_a8*)(y + (size_t)(it * 8) * p.d2));
        }
    return;
  }
  const bool whole = !BACK || p.S == 1;  // the sums are the result
  if (whole) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = j * 32 + g * 8 + (lane >> 5) * 4, n = n0 + wn * 128 + c;
      float bv[4] = {0.f, 0.f, 0.f, 0.f};
      if (p.bias && n < p.d2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bv[e] = bf16_to_f32(p.bias[n + e]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u32x2 v;
        v[0] = pack_bf16x2(acc[i][j][4 * g] + bv[0], acc[i][j][4 * g + 1] + bv[1]);
        v[1] = pack_bf16x2(acc[i][j][4 * g + 2] + bv[2], acc[i][j][4 * g + 3] + bv[3]);
        *(u32x2*)(mine + (i * 32 + (lane & 31)) * kOutPitch + c * 2) = v;
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0xc07f);  // the wave's own writes, read by its other lanes
  asm volatile("" ::: "memory");
  {
    const int n = n0 + wn * 128 + (lane & 15) * 8;
    const int64_t mw = m0 + wm * 128 + (lane >> 4);
    bf16_t* y = p.Y + (size_t)mw * p.d2 + n;
    const unsigned char* q = mine + (lane >> 4) * kOutPitch + (lane & 15) * 16;
    if (n < p.d2)
#pragma unroll 4
      for (int it = 0; it < 32; ++it) {
        if (mw + it * 4 < p.M) {
          const u32x4_a8 v = *(const u32x4*)(q + it * 4 * kOutPitch);
          __builtin_nontemporal_store(v, (u32x4_a8*)(y + (size_t)(it * 4) * p.d2));
        }
      }
  }
  }

  // ---- what the stages could not take: products with the tenant's own Inf and NaN, onto the stored results (no finite part of
  // them matters any more)
  if (bad) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int i = 0; i < 4; ++i) {
      const int64_t m = m0 + wm * 128 + i * 32 + (lane & 31);
      if (m >= p.M) continue;
      const int64_t req = p.row_to_req ? (int64_t)p.row_to_req[m] : p.row_base + m;
      for (int s = 0; s < kSites; ++s) {
      int tenant = 0;
      const int r = (req >= 0 && req < p.B) ? routed_rank(p.ad, p.tenant_id, p.route, (int)req, p.B, p.site + s, &tenant) : 0;
      for (int c = 0; c < r; ++c) {
        gbf16* b = in_global((BACK ? p.ad.A : p.ad.B)[tenant * MILORA_NUM_SITES + p.site + s]) + (BACK ? (size_t)c : (size_t)c * p.d2);
        float t = 0.f;
        for (int k = 0; k < p.parts; ++k) t += p.t[(kSites > 1 ? s * p.t_site : 0) + k * p.t_stride + (size_t)m * p.ad.r_max + c];
        for (int q = 0; q < 64; ++q) {  // this lane's columns
          const int n = n0 + wn * 128 + (q >> 4) * 32 + ((q >> 2) & 3) * 8 + (lane >> 5) * 4 + (q & 3);
          if (n >= p.d2) continue;
          const bf16_t bv = b[BACK ? (size_t)n * r : (size_t)n];
          // (MX forward: Inf and NaN of t are left for here too; a high half by itself otherwise)
          if ((bv & 0x7f80u) != 0x7f80u && !(HALVES && !BACK && !finite_f32(t))) continue;
          if (whole) {
            bf16_t* const y = p.Y + (size_t)m * p.d2 + n;
            *y = f32_to_bf16(bf16_to_f32(*y) + t * bf16_to_f32(bv));
          } else {
            p.partial[part * p.partial_stride + (size_t)m * p.d2 + n] += t * bf16_to_f32(bv);
          }
        }
      }
      }
    }
  }
}

// SITES: several sites in one launch, blockIdx.z = site x shares + share.
template <int RT, bool INFO, bool SITES, bool TRANS>
__global__ void __launch_bounds__(512, 4) shrink_tiles_kernel(const ShrinkArgs g) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[8 * kShrinkWaveBytes];
  __shared__ int row_ten[RT * 16 * (INFO ? 2 : 1)];
  auto store = [](float* p, float v) { *p = v; };
  if constexpr (SITES) {
    const int shares = gridDim.z / g.sites, s = blockIdx.z / shares;
    ShrinkArgs one = g;
    one.site += s;
    one.X += s * g.x_site;
    one.t += s * g.t_site;
    if (one.row_lora) one.row_lora += s * g.lora_site;
    shrink_block<RT, 8, INFO, TRANS>(one, blockIdx.x, blockIdx.y, gridDim.y, blockIdx.z % shares, shares, smem, row_ten, store);
  } else {
    shrink_block<RT, 8, INFO, TRANS>(g, blockIdx.x, blockIdx.y, gridDim.y, blockIdx.z, gridDim.z, smem, row_ten, store);
  }
  static_assert(kShrinkClear == 512, "one word per thread");
  if (INFO && g.clear && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) g.clear[threadIdx.x] = 0;
}

template <int RT>
void launch_shrink_block(const ShrinkArgs& g, dim3 grid, bool trans, hipStream_t st) {
  const bool info = g.row_lora || g.clear;
  if (!trans) {
    if (info) hipLaunchKernelGGL((shrink_tiles_kernel<RT, true, true, false>), grid, dim3(512), 0, st, g);
    else hipLaunchKernelGGL((shrink_tiles_kernel<RT, false, true, false>), grid, dim3(512), 0, st, g);
  } else if (g.sites > 1) {
    if (info) hipLaunchKernelGGL((shrink_tiles_kernel<RT, true, true, true>), grid, dim3(512), 0, st, g);
    else hipLaunchKernelGGL((shrink_tiles_kernel<RT, false, true, true>), grid, dim3(512), 0, st, g);
  } else {
    if (info) hipLaunchKernelGGL((shrink_tiles_kernel<RT, true, false, true>), grid, dim3(512), 0, st, g);
    else hipLaunchKernelGGL((shrink_tiles_kernel<RT, false, false, true>), grid, dim3(512), 0, st, g);
  }
}

}  // namespace

bool prefill_supported(int64_t M, int d1, int d2, const void* X, const void* W, const void* Y) {
  if (M < 64 || d1 % kTK != 0 || d2 % 16 != 0) return false;
  if ((((uintptr_t)X | (uintptr_t)W) & 15) != 0 || ((uintptr_t)Y & 7) != 0) return false;
  return (uint64_t)d2 * (uint64_t)d1 * 2u < (1ull << 32);  // 32-bit byte offsets inside W (X is cut into row slices)
}

template <int MODE, bool MX>
static int launch_prefill(PParams p, int64_t M, int64_t row_base, hipStream_t stream) {
  static thread_local int lds_set_for = -1;
  int dev = 0;
  MILORA_HIP(hipGetDevice(&dev));
  if (lds_set_for != dev) {
    MILORA_HIP(hipFuncSetAttribute((const void*)prefill_kernel<MODE, MX>, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsBytesP));
    lds_set_for = dev;
  }
  // rows are independent: slices whose byte offsets inside X fit 32 bits and whose tile count fits a launch
  p.polls = wait_limit();
  const PParams all = p;
  int64_t slice = (int64_t)(((1ull << 32) - 1) / ((uint64_t)p.d1 * 2u)) / kTM * kTM;
  constexpr int kCols = MODE == kGated ? kTN / 2 : kTN;
  const int tilesN = (p.d2 + kCols - 1) / kCols;
  const int64_t by_grid = (int64_t)((1 << 24) / tilesN) * kTM;
  if (slice > by_grid) slice = by_grid;
  if (slice < kTM) return MILORA_EUNSUPPORTED;
  for (int64_t r0 = 0; r0 < M; r0 += slice) {
    p.M = M - r0 < slice ? M - r0 : slice;
    p.X = all.X + (size_t)r0 * p.d1;
    p.Y = all.Y + (size_t)r0 * p.d2;
    if (all.gate_out) p.gate_out = all.gate_out + (size_t)r0 * p.d2;
    if (all.up_out) p.up_out = all.up_out + (size_t)r0 * p.d2;
    if (all.partial) p.partial = all.partial + (size_t)r0 * p.d2;
    p.t = all.t + (size_t)r0 * p.ad.r_max;
    p.row_to_req = all.row_to_req ? all.row_to_req + r0 : nullptr;
    p.row_base = row_base + r0;
    p.tilesM = (int)((p.M + kTM - 1) / kTM);
    p.tilesN = tilesN;
    const int64_t tiles = (int64_t)p.tilesM * p.tilesN;
    int64_t total = tiles * (MODE == kBack && p.S > 1 ? p.S : 1), units = 0;
    if ((MODE != kPlain || MX) && total == tiles) {
      const CutPlan cut = cut_plan(tiles, p.d1 / kTK, MX && MODE != kBack);
      p.whole = (int)cut.whole; p.cut = cut.parts; p.cut_steps = cut.steps;
      total = cut.whole;
      units = (tiles - cut.whole) * cut.parts;
    }
    hipLaunchKernelGGL((prefill_kernel<MODE, MX>), dim3((unsigned)(8 * ((total + 7) / 8 + (units + 7) / 8))), dim3(kThreadsP), kLdsBytesP, stream, p);
    const int rc = check_launch();
    if (rc) return rc;
  }
  return MILORA_OK;
}

int routed_linear_prefill(const bf16_t* X, int64_t M, int d1, int d2, const int32_t* row_to_req, const bf16_t* W,
                          const bf16_t* bias, const AdapterView& ad, int site, const int32_t* tenant_id,
                          const uint8_t* route, int B, const float* t, bf16_t* Y, hipStream_t stream) {
  PParams p{};
  p.X = X; p.W = W; p.bias = bias; p.Y = Y; p.t = t;
  p.t_stride = (size_t)M * ad.r_max;
  p.parts = shrink_parts(M, d1);
  p.row_to_req = row_to_req; p.tenant_id = tenant_id; p.route = route; p.ad = ad;
  p.d1 = d1; p.d2 = d2; p.site = site; p.B = B;
  return launch_prefill<kPlain, false>(p, M, 0, stream);
}

int gated_prefill(const GatedTileArgs& g, hipStream_t stream) {
  PParams p{};
  p.X = g.X; p.W = g.Wg; p.W2 = g.Wu; p.Y = g.Y; p.gate_out = g.gate_out; p.up_out = g.up_out;
  p.t = g.t; p.t_stride = g.t_stride; p.t_site = g.t_site; p.parts = g.parts;
  p.row_to_req = g.row_to_req; p.tenant_id = g.tenant_id; p.route = g.route; p.ad = g.ad;
  p.row_lora = g.row_lora; p.lora_site = g.lora_site; p.halves = g.halves.at; p.half_site = g.halves.site; p.half_chunk = g.halves.chunk;
  p.cut_sums = g.partial; p.cut_cnt = g.cnt;
  p.d1 = g.d; p.d2 = g.F; p.site = 4; p.B = g.B;
  return g.mx4 ? launch_prefill<kGated, true>(p, g.M, g.row_base, stream) : launch_prefill<kGated, false>(p, g.M, g.row_base, stream);
}

// The same tiles on 4-bit weights (p.W in their place): LoRA terms from the halves of one site.
int linear_prefill_mx4(const GatedTileArgs& g, const bf16_t* bias, int site, hipStream_t stream) {
  PParams p{};
  p.X = g.X; p.W = g.Wg; p.bias = bias; p.Y = g.Y;
  p.t = g.t; p.t_stride = g.t_stride; p.t_site = g.t_site; p.parts = g.parts;
  p.row_to_req = g.row_to_req; p.tenant_id = g.tenant_id; p.route = g.route; p.ad = g.ad;
  p.row_lora = g.row_lora; p.lora_site = g.lora_site; p.halves = g.halves.at; p.half_site = g.halves.site; p.half_chunk = g.halves.chunk;
  p.cut_sums = g.partial; p.cut_cnt = g.cnt;
  p.d1 = g.d; p.d2 = g.F; p.site = site; p.B = g.B;
  return launch_prefill<kPlain, true>(p, g.M, g.row_base, stream);
}

// (scales are copied sixteen bytes at a time, from addresses that are multiples of four, the last ones from the end of a column's)
bool mx4_prefill_supported(int64_t M, int d1, int d2) {
  return M >= 64 && M <= kHalvesRows && d1 % 128 == 0 && d1 >= 512 && d2 % 16 == 0 && (uint64_t)d1 * 2u * kTM < (1ull << 32) &&
         (uint64_t)d2 * d1 / 2 < (1ull << 32);
}

// Parts of the reduction: as many as make the tiles fill the compute units once, whole k steps each, eight at least.
static int back_parts(int64_t M, int d, int F, int* steps) {
  const int64_t tiles = ((M + kTM - 1) / kTM) * ((d + kTN - 1) / kTN);
  const int KT = 2 * F / kTK;
  int64_t S = 256 / tiles;
  if (S > KT / 8) S = KT / 8;
  if (S <= kCutParts) S = 1;  // (a cut of all tiles does without the launch behind)
  *steps = (int)((KT + S - 1) / S);
  return (KT + *steps - 1) / *steps;
}

// What the sums of a call with several parts take, at most: 256 workgroups share its reduction, eight k steps at least each.  Never
// less for a larger call, so that a workspace for the largest serves all.
size_t back_partial_floats(int64_t M, int d, int F) {
  const size_t by_grid = (size_t)256 * kTM * kTN, by_steps = (size_t)(F / 256 + 1) * (size_t)M * d;
  const size_t all = by_steps < by_grid ? by_steps : by_grid, cut = cut_bytes_bound(M, d) / sizeof(float);
  return all > cut ? all : cut;
}

bool back_supported(int64_t M, int d, int F, const void* dz, const void* Wg, const void* Wu, const void* dX) {
  if (F % (kTK / 2) != 0 || d % 16 != 0 || M < 1 || M > kHalvesRows) return false;
  if ((((uintptr_t)dz | (uintptr_t)Wg | (uintptr_t)Wu) & 15) != 0 || ((uintptr_t)dX & 7) != 0) return false;
  return (uint64_t)d * kTK * 2u < (1ull << 31) && (uint64_t)F * 4u * kTM < (1ull << 32) && (int64_t)((d + kTN - 1) / kTN) <= 1 << 16;
}

static __global__ void __launch_bounds__(256) add_parts_kernel(const float* __restrict__ partial, int S, size_t stride, int64_t fours, bf16_t* __restrict__ y) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= fours) return;
  const float* const q = partial + i * 4;
  f32x4 v = *(const f32x4*)q;
  int s = 1;
  for (; s + 4 <= S; s += 4) {
    f32x4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = *(const f32x4*)(q + (s + u) * stride);
#pragma unroll
    for (int u = 0; u < 4; ++u) v += x[u];
  }
  for (; s < S; ++s) v += *(const f32x4*)(q + s * stride);
  u32x2 o;
  o[0] = pack_bf16x2(v[0], v[1]);
  o[1] = pack_bf16x2(v[2], v[3]);
  *(u32x2*)(y + i * 4) = o;
}

int gated_dx_tiles(const GatedBackArgs& g, hipStream_t stream) {
  PParams p{};
  p.X = g.dz; p.W = g.Wg; p.W2 = g.Wu; p.Y = g.dX; p.t = g.low; p.t_stride = g.low_stride; p.t_site = g.low_site; p.parts = g.parts;
  p.row_to_req = g.row_to_req; p.tenant_id = g.tenant_id; p.route = g.route; p.ad = g.ad;
  p.row_lora = g.row_lora; p.lora_site = g.lora_site; p.halves = g.halves.at; p.half_site = g.halves.site; p.half_chunk = g.halves.chunk;
  p.d1 = 2 * g.F; p.d2 = g.d; p.site = 4; p.B = g.B;
  p.S = back_parts(g.M, g.d, g.F, &p.steps);
  p.partial = p.S > 1 ? g.partial : nullptr;
  p.cut_sums = g.partial; p.cut_cnt = g.cnt;
  p.partial_stride = (size_t)g.M * g.d;
  const int rc = g.mx4 ? launch_prefill<kBack, true>(p, g.M, 0, stream) : launch_prefill<kBack, false>(p, g.M, 0, stream);
  if (rc || p.S == 1) return rc;
  const int64_t fours = g.M * g.d / 4;
  hipLaunchKernelGGL(add_parts_kernel, dim3((unsigned)((fours + 255) / 256)), dim3(256), 0, stream, g.partial, p.S, p.partial_stride, fours, g.dX);
  return check_launch();
}

static int launch_shrinks(ShrinkArgs g, bool trans, hipStream_t stream) {
  const ShrinkArgs all = g;
  const int64_t M = g.M;
  const int parts = shrink_parts(M, g.d1, g.sites);
  const int64_t slice = (int64_t)1 << 28;  // rows per launch: 512 threads for 64 rows, a grid has to stay below 2^32 threads
  for (int64_t r0 = 0; r0 < M; r0 += slice) {
    g.X = all.X + (size_t)r0 * g.ldx;
    g.M = M - r0 < slice ? M - r0 : slice;
    g.row_base = r0;
    g.row_to_req = all.row_to_req ? all.row_to_req + r0 : nullptr;
    g.t = all.t + (size_t)r0 * g.ad.r_max;
    g.row_lora = all.row_lora ? all.row_lora + r0 : nullptr;
    if (M <= kTileMaxRows) {
      const int64_t blocks = (g.M + 15) / 16;
      const int shares = shrink_shares(blocks, parts, g.sites, g.B, g.ad);
      launch_shrink_block<1>(g, dim3((unsigned)blocks, parts, shares * g.sites), trans, stream);
    }
    else
      launch_shrink_block<4>(g, dim3((unsigned)((g.M + 63) / 64), parts, g.sites), trans, stream);
    const int rc = check_launch();
    if (rc) return rc;
  }
  return MILORA_OK;
}

// LoRA shrink of the rows the tile kernel serves (same conditions as prefill_supported) at `sites` consecutive sites: t receives
// shrink_parts(M, d1, sites) partial results [site][part][M][r_max], to be added in part order, row_lora (or null) [site][M] what the
// look-ups found of each row; `clear` (or null) is zeroed.
int launch_shrink_sites(const bf16_t* X, int64_t ldx, int64_t M, int d1, const int32_t* row_to_req, const AdapterView& ad, int site, int sites,
                        const int32_t* tenant_id, const uint8_t* route, int B, float* t, int2* row_lora, int* clear, hipStream_t stream) {
  const size_t t_stride = (size_t)M * ad.r_max;
  return launch_shrinks(ShrinkArgs{X, ldx, M, 0, d1, site, B, row_to_req, tenant_id, route, ad, t, t_stride, row_lora, clear, sites,
                                   t_stride * shrink_parts(M, d1, sites), (size_t)M, 0}, true, stream);
}

// low[site][part][m][0..r) = dz[m] (of the site) . (W^B)^T for the rows routed to the gate (site 4) and the up projection; dz [M][2 F],
// F % 32 == 0, shrink_parts(M, F, 2) parts.
int launch_low_sites(const bf16_t* dz, int64_t M, int F, const int32_t* row_to_req, const AdapterView& ad, const int32_t* tenant_id,
                     const uint8_t* route, int B, float* low, hipStream_t stream) {
  const size_t stride = (size_t)M * ad.r_max;
  return launch_shrinks(ShrinkArgs{dz, 2 * (int64_t)F, M, 0, F, 4, B, row_to_req, tenant_id, route, ad, low, stride, nullptr, nullptr, 2,
                                   stride * shrink_parts(M, F, 2), (size_t)M, F}, false, stream);
}

int launch_shrink_tiles(const bf16_t* X, int64_t M, int d1, const int32_t* row_to_req, const AdapterView& ad, int site,
                        const int32_t* tenant_id, const uint8_t* route, int B, float* t, int2* row_lora, int* clear, hipStream_t stream) {
  return launch_shrink_sites(X, d1, M, d1, row_to_req, ad, site, 1, tenant_id, route, B, t, row_lora, clear, stream);
}

}  // namespace milora

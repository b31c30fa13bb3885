// Interface of the matrix-core tile kernel for few to some thousand rows (tiles.hip).
#pragma once
#include "common.h"

namespace milora {

// Tiles and parts of the reduction of one launch; a function of the sizes alone, shared by the launch and the sizing of
// the workspace.
enum TileShape { kTiles64 = 0, kTiles128 = 1, kTiles256 = 2 };
struct TilePlan {
  int shape;  // TileShape: 64 x 64 and 128 x 128 (tiles.hip), 256 x 256 (prefill.hip)
  int tilesM, tilesN;
  int S, steps;          // parts of the reduction, stages of 64 k per part
  size_t partial_bytes;  // fp32 partial tiles in the workspace (0 when S == 1)
  int64_t time;          // what the choice reckons, in 10 ns
};
// What writing a 4-bit weight out in bf16 takes, in 10 ns (4096 x 11008: 20 us).
inline int64_t write_out_time(int d1, int d2) { return 300 + (int64_t)d1 * d2 / 26000; }
constexpr int kStreamRows = 32;      // rows up to which a packed linear takes the weight-streaming kernel (decode.hip)
constexpr int kMaxSplitUnits = 512;  // tiles x parts of a launch that cuts its reduction
constexpr int kMaxParts = 8;         // of one reduction
// 256 x 256 tiles run one a compute unit, whole turns of 256.  Those of a last turn that is not full are cut along the reduction where that is
// faster: `parts` workgroups a tile, of `steps` k steps of 64 (a multiple of eight for 4-bit weights, whose scales come for eight), whose sums meet in
// memory (prefill.hip).  A turn's step takes 1.6 us, the exchange some 15 us.
struct CutPlan {
  int64_t whole;  // tiles that are not cut, in front of the others
  int parts, steps;
};
constexpr int kCutParts = 4, kCutCost = 1500;  // (10 ns)
inline CutPlan cut_plan(int64_t tiles, int KT, bool mx4) {
  const CutPlan none{tiles, 1, KT};
  const int rest = (int)(tiles % 256);
  if (rest == 0 || rest > 128) return none;
  int parts = 256 / rest < kCutParts ? 256 / rest : kCutParts;
  if (parts > KT / 8) parts = KT / 8;
  if (parts < 2) return none;
  int steps = (KT + parts - 1) / parts;
  if (mx4) steps = (steps + 7) / 8 * 8;
  parts = (KT + steps - 1) / steps;
  if (parts < 2 || (KT - steps) * 163 <= kCutCost) return none;
  return CutPlan{tiles - rest, parts, steps};
}
// What the sums of cut tiles take, at most; never less for larger sizes.  (columns: gate and up together)
inline size_t cut_bytes_bound(int64_t M, int64_t columns) {
  const int64_t tiles = ((M + 255) / 256) * ((columns + 255) / 256);
  return (size_t)(tiles < 256 / kCutParts ? tiles * kCutParts : 256) * 65536 * sizeof(float);
}

// The first bytes of a routed linear's workspace belong to control words: those of the stream kernels (decode.hip), then the
// part counters of the tile kernel, zeroed by the shrink launch in front of it.  Both keep their data behind them, so calls of
// any sizes and any layout can follow one another on one workspace (those of 4-bit weights leave all of it alone), and the status word can be asked for after either.
constexpr int kStreamCtrlBytes = 16384;
constexpr int kTileCtrlBytes = kMaxSplitUnits * (int)sizeof(int);
constexpr int kTileCtrlOffset = kStreamCtrlBytes - kTileCtrlBytes;

// `small`: the tiles of tiles.hip are a choice up to kTileMaxRows rows (tiles_supported); `large`: the 256 x 256 kernel is one
// (row-major weights, 64 rows or more).  At least one of them.
// kCut: the 256 x 256 kernel cuts its last tiles, kCutMx4: and reads 4-bit weights.
enum TileCut { kNoCut, kCut, kCutMx4 };
TilePlan plan_tiles(int64_t M, int d1, int d2, bool small, bool large, bool gated = false, TileCut cut = kNoCut);
// The most partial_bytes over the plans of all calls of up to these sizes; never less for a larger size.
size_t partial_bytes_bound(int64_t M, int d1, int d2);
bool tiles_supported(int64_t M, int d1, int d2, bool packed, const void* X, const void* W, const void* Y);
// `row_lora` (always there for packed weights): the LoRA term in fp32 row by row.  Null: by the matrix cores, from the look-ups of
// the other arguments; the rows are then all of the call's.
int routed_linear_tiles(const bf16_t* X, int64_t M, int d1, int d2, const int32_t* row_to_req, const bf16_t* W, bool packed,
                        const int2* row_lora, const bf16_t* bias, const AdapterView& ad, int site, const int32_t* tenant_id, const uint8_t* route,
                        int B, const float* t, size_t t_stride, int parts, const TilePlan& pl, int* cnt, float* partial, bf16_t* Y, hipStream_t st);

// The gated block Y = silu(X Wg + its term) * (X Wu + its term): gate and up columns side by side in a tile (plan_tiles and
// tiles_supported with 2 F columns).  kTiles256: gated_prefill.
// Shrinks of the two sites as bf16 halves (gated.hip): [site][chunk of 32 ranks][1 + M] lines of 64 values, 32 high and 32 low, the first line zero.
struct Halves {
  bf16_t* at;
  size_t site, chunk;  // elements from one's to the next's
};
constexpr int64_t kHalvesRows = (int64_t)1 << 24;  // (32-bit byte offsets of the lines)
inline Halves halves_of(bf16_t* at, int64_t M, int r_max) {
  const size_t chunk = (size_t)(M + 1) * 64;
  return Halves{at, chunk * ((r_max + 31) / 32), chunk};
}

struct GatedTileArgs {
  const bf16_t* X;
  int64_t M, row_base;  // rows of the launch, index of the first in the caller's matrix (requests of unmapped rows)
  int d, F;
  const int32_t* row_to_req;
  const bf16_t *Wg, *Wu;
  bool packed;
  bool mx4;              // (kTiles256) Wg and Wu are 4-bit weights
  const int2* row_lora;  // [2][lora_site]; kTiles64, kTiles128: or null, the terms by the matrix cores
  size_t lora_site;
  Halves halves;         // kTiles256
  AdapterView ad;
  const int32_t* tenant_id;
  const uint8_t* route;
  int B;
  const float* t;  // [2][part][t_stride]
  size_t t_stride, t_site;
  int parts;
  int* cnt;
  float* partial;
  bf16_t* Y;
  float *gate_out, *up_out;
};
int gated_tiles(const GatedTileArgs& g, const TilePlan& pl, hipStream_t st);
int gated_prefill(const GatedTileArgs& g, hipStream_t st);
bool mx4_prefill_supported(int64_t M, int d1, int d2);
// A linear on 4-bit weights (g.Wg, g.d inputs, g.F columns), [1][..] shrinks, look-ups and halves.
int linear_prefill_mx4(const GatedTileArgs& g, const bf16_t* bias, int site, hipStream_t st);
// (gated.hip) v [site][part][M][r_max] to `sites` sites' halves.  Inf and NaN become zeros there and set kLaterBit of the row's rank.
constexpr int kLaterBit = 1 << 16;
int launch_halves(const float* v, int parts, int64_t M, int r_max, int2* row_lora, int sites, const Halves& out, hipStream_t st);

// dX = [dg | du] [W_gate; W_up] + sum over the two sites of low A^T on 256 x 256 tiles (prefill.hip).
struct GatedBackArgs {
  const bf16_t* dz;  // [M][2 F]
  int64_t M;
  int d, F;
  const int32_t* row_to_req;
  const bf16_t *Wg, *Wu;  // row-major [F][d]
  bool mx4;               // 4-bit weights in their place, d % 128 == 0
  AdapterView ad;
  const int32_t* tenant_id;
  const uint8_t* route;
  int B;
  const int2* row_lora;  // [2][lora_site]
  size_t lora_site;
  Halves halves;     // of low
  const float* low;  // [2][part][M][r_max] = dz W^B^T, to be added in part order
  size_t low_stride, low_site;
  int parts;
  float* partial;  // back_partial_floats(M, d, F)
  int* cnt;        // kShrinkClear words, zero
  bf16_t* dX;
};
bool back_supported(int64_t M, int d, int F, const void* dz, const void* Wg, const void* Wu, const void* dX);
size_t back_partial_floats(int64_t M, int d, int F);
int gated_dx_tiles(const GatedBackArgs& g, hipStream_t st);

}  // namespace milora

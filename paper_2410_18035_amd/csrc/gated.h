// Interface of the gated block and its backward pass (gated.hip).
#pragma once
#include "common.h"

namespace milora {

// A call whose arguments have been accepted.  Base weights row-major in `dtype`, or (mx4) 4-bit ones.
struct GatedCall {
  const void* X;
  int64_t M;
  int d, F, dtype;
  bool mx4;
  const int32_t* row_to_req;
  const void *Wg, *Wu;
  AdapterView ad;
  const int32_t* tenant_id;
  const uint8_t* route;
  int B;
};

size_t gated_workspace_bytes(int64_t M, int d, int F, int dtype, bool mx4, int r_max);
int run_gated(const GatedCall& g, void* Y, float* gate_out, float* up_out, void* workspace, hipStream_t st);

size_t gated_backward_workspace_bytes(int64_t M, int d, int F, int dtype, bool mx4, int r_max);
// dA, dB: device tables [T * 7] of gradients' addresses (null entries: not wanted), or null.
int run_gated_backward(const GatedCall& g, const void* dY, const float* gate, const float* up, void* dX, void* const* dA, void* const* dB,
                       void* workspace, hipStream_t st);

}  // namespace milora

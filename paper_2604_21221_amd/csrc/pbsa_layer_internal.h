// Internal launcher interface between the C-ABI shim of pbsa_layer.h (pbsa_layer_api.hip) and the kernel files.
// Every launcher only enqueues on `stream` and returns the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pbsa_layer.h"

namespace pbsa {

int report(hipError_t e);   // pbsa_api.hip: PBSA_OK, or PBSA_EHIP with its text kept for pbsa_strerror

enum class RotaryOp { rotate, norm, norm_grad };

// What the three calls on a pbsa_rotary pass on: index 0 the queries, 1 the keys.
struct RotaryTensors {
  const void* x[2];         // inputs of the forward call
  const void* dy[2];        // norm_grad: gradients that come in
  void* y[2];               // what is written
  const float* w[2];
  float* dw[2];
  const int64_t* pos;
  const double* freq;
  float sign;               // of the angles
};
size_t rotary_workspace_bytes(const pbsa_rotary& p);
hipError_t launch_rotary(const pbsa_rotary& p, RotaryOp op, const RotaryTensors& t, void* ws, hipStream_t stream);

bool cross_fits(const pbsa_cross& p, bool masked);   // into a launch
size_t cross_workspace_bytes(const pbsa_cross& p, bool masked);
// The attended states of each sequence under a mask, in order: counts [n] in the first attended_first(n) places of the scratch,
// the list [n][Nk] behind them (pbsa_cross_list.hip).
inline size_t attended_first(int n) { return ((size_t)n + 63) & ~(size_t)63; }
inline size_t attended_bytes(int n, int Nk) { return (attended_first(n) + (size_t)n * Nk) * sizeof(int32_t); }
hipError_t launch_attended(const int32_t* k_len, const uint8_t* k_mask, int64_t mask_stride_b, int n, int Nk, int32_t* list, int32_t* counts,
                           hipStream_t stream);
hipError_t launch_cross(const pbsa_cross& p, const void* Q, const void* K, const void* V, const int32_t* k_len, const uint8_t* k_mask,
                        void* O, float* lse, void* ws, hipStream_t stream);
size_t cross_bwd_workspace_bytes(const pbsa_cross& p);
hipError_t launch_cross_bwd(const pbsa_cross& p, const void* Q, const void* K, const void* V, const int32_t* k_len, const uint8_t* k_mask,
                            const void* O, const void* dO, const float* lse, void* dQ, void* dK, void* dV, void* ws,
                            hipStream_t stream);

}  // namespace pbsa

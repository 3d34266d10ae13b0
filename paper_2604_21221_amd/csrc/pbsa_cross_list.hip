// The states of each sequence that a mask leaves, in order, for the cross attention kernels that many rows share: they walk the
// list instead of the states, so that a masked state costs nothing but its byte.
//
// One workgroup to a sequence: 16 bytes of the mask to a thread, the threads' counts summed up across the workgroup, round
// after round.  Bound by its rounds' latency: a round takes 16384 states.
#include "pbsa_layer_internal.h"

namespace pbsa {
namespace {

constexpr int kThreads = 1024, kEach = 16;

constexpr int kMostGroups = 1 << 21;

__device__ void list_sequence(const int32_t* k_len, const uint8_t* k_mask, int64_t mask_stride_b, int Nk, int32_t* list, int32_t* counts,
                              int64_t b, int* wave_sum) {
  const uint8_t* const mask = k_mask + b * mask_stride_b;
  int32_t* const to = list + b * Nk;
  const int len = k_len ? min(max(k_len[b], 0), Nk) : Nk;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int before = 0;                    // states listed in earlier rounds
  for (int k0 = 0; k0 < len; k0 += kThreads * kEach) {
    const int k = k0 + threadIdx.x * kEach;
    uint32_t on = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (k + j < len && mask[k + j] != 0) on |= 1u << j;
    const int mine = __popc(on);
    int upto = mine;                 // of this wave's lanes up to this one
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int v = __shfl_up(upto, s);
      if (lane >= s) upto += v;
    }
    __syncthreads();                 // the last round's sums have been read
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int at = before + upto - mine, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      const int v = wave_sum[w];
      at += w < wave ? v : 0;
      all += v;
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (on >> j & 1) to[at++] = k + j;
    before += all;
  }
  if (threadIdx.x == 0) counts[b] = before;
}
__global__ void __launch_bounds__(kThreads) attended_kernel(const int32_t* k_len, const uint8_t* k_mask, int64_t mask_stride_b, int n, int Nk,
                                                            int32_t* list, int32_t* counts) {
  __shared__ int wave_sum[kThreads / 64];
  for (int64_t b = blockIdx.x; b < n; b += gridDim.x) list_sequence(k_len, k_mask, mask_stride_b, Nk, list, counts, b, wave_sum);
}

}  // namespace

hipError_t launch_attended(const int32_t* k_len, const uint8_t* k_mask, int64_t mask_stride_b, int n, int Nk, int32_t* list, int32_t* counts,
                           hipStream_t stream) {
  hipLaunchKernelGGL(attended_kernel, dim3((unsigned)(n < kMostGroups ? n : kMostGroups)), dim3(kThreads), 0, stream, k_len, k_mask, mask_stride_b,
                     n, Nk, list, counts);
  return hipGetLastError();
}

}  // namespace pbsa

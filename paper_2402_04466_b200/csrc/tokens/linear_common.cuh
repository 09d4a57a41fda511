// What the kernels of tt_linear_attention share.
#pragma once

#include "tokens.h"

namespace tt {
namespace tok {

template <typename T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }
template <>
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

// Slot of entry b, or -1: it is passed over, because its slot is out of range or an earlier entry's.  All of the block's threads call it.
__device__ __forceinline__ int slot_of(const int32_t* slots, int num_slots, int b) {
  if (!slots) return b < num_slots ? b : -1;
  const int mine = slots[b];
  bool taken = false;
  for (int i = threadIdx.x; i < b; i += blockDim.x) taken |= slots[i] == mine;
  return __syncthreads_or(taken) || mine < 0 || mine >= num_slots ? -1 : mine;
}

// exp(log_decay * n), formed in 64 bits: a state that fades over thousands of tokens multiplies many of these.
__device__ __forceinline__ float decay_power(float log_decay, int n) { return n == 0 ? 1.f : (float)exp((double)log_decay * n); }

}  // namespace tok
}  // namespace tt

// Element types and row helpers of the row operators (k_embed.hip,
// k_rows.hip): loads and stores of fp32, fp16 and bf16 rows that start at any
// element, and fixed-order reductions over a workgroup.
#pragma once

#include "ifvs_internal.h"

namespace ifvs {

template <typename T>
__device__ __forceinline__ float elem_load(const T* p) {
  return static_cast<float>(*p);
}

// One rounding, to nearest even (past the range of fp16: infinity).
template <typename T>
__device__ __forceinline__ T elem_round(float v) {
  return static_cast<T>(v);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Sum / maximum over the workgroup, the same value in every thread; `s` holds
// one entry per wavefront and may be reused right after the call.
template <int kWaves>
__device__ __forceinline__ double block_add(double v, double* s) {
  v = wave_add(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v += s[w];
  __syncthreads();
  return v;
}

template <int kWaves>
__device__ __forceinline__ float block_max(float v, double* s) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  v = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) v = fmaxf(v, static_cast<float>(s[w]));
  __syncthreads();
  return v;
}

}  // namespace ifvs

// Device helpers of the row operators: element access, sums and maxima over a
// workgroup, and the treatment of values that are no number.
#pragma once

#include "ctcbeam_lane.h"
#include "ctcbeam_rows.h"

namespace ctcbeam {
namespace rows {

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLargest = 3.402823466e38f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct F16 { uint16_t u; };
struct BF16 { uint16_t u; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(F16 v) { return static_cast<float>(__builtin_bit_cast(_Float16, v.u)); }
__device__ __forceinline__ float to_float(BF16 v) { return __uint_as_float(static_cast<uint32_t>(v.u) << 16); }
__device__ __forceinline__ void from_float(float v, float* o) { *o = v; }
__device__ __forceinline__ void from_float(float v, F16* o) { o->u = __builtin_bit_cast(uint16_t, static_cast<_Float16>(v)); }
__device__ __forceinline__ void from_float(float v, BF16* o) { o->u = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }

// NaN counts as -inf, +inf as the largest number
__device__ __forceinline__ float clean(float v) { return v != v ? kNegInf : fminf(v, kLargest); }

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

template <int N>
__device__ __forceinline__ float block_max(float v, float* lds) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = lds[0];
  for (int i = 1; i < N / 64; ++i) r = fmaxf(r, lds[i]);
  return r;
}
template <int N>
__device__ __forceinline__ float block_sum(float v, float* lds) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = lds[0];
  for (int i = 1; i < N / 64; ++i) r += lds[i];
  return r;
}

__device__ __forceinline__ int length_of(const RowsView& v, int b) {
  if (!v.lengths) return v.T;
  const int l = v.lengths[b];
  return l < 0 ? 0 : (l > v.T ? v.T : l);
}

}  // namespace rows
}  // namespace ctcbeam

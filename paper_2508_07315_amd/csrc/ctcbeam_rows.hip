// Row operators, the simple forms: one workgroup per row, the row read from
// memory for each pass over it.
#include "ctcbeam_rows_lane.h"

namespace ctcbeam {
namespace rows {

constexpr int kN = 256;

template <int N>
__device__ __forceinline__ float block_max(float v, float* lds) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = lds[0];
  for (int i = 1; i < N / 64; ++i) r = fmaxf(r, lds[i]);
  return r;
}
template <int N>
__device__ __forceinline__ float block_sum(float v, float* lds) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = lds[0];
  for (int i = 1; i < N / 64; ++i) r += lds[i];
  return r;
}

template <typename T>
__global__ void __launch_bounds__(kN) distill_kernel(const DistillParams p) {
  __shared__ uint32_t listed[kMaxLabels / 32];
  __shared__ int32_t ids[kMaxTop];
  __shared__ float prob[kMaxTop];
  __shared__ float red[kN / 64];
  const int W = p.in.W, tid = threadIdx.x, k = p.k;
  const int b = blockIdx.x / p.in.T, t = blockIdx.x % p.in.T;
  const int64_t row = static_cast<int64_t>(b) * p.in.T + t;
  const T* x = static_cast<const T*>(p.in.data) + b * p.in.stride_b + t * p.in.stride_t;
  T* grad = p.grad ? static_cast<T*>(p.grad) + b * p.grad_stride_b + t * p.grad_stride_t : nullptr;
  bool there = t < length_of(p.in, b);
  float u = kNegInf, rest = kNegInf, m = kNegInf, mr = kNegInf, Z = 0.0f;
  if (there) {
    // the teacher's list: P_c = e^u_c / Z, equal labels summed into their first entry
    int32_t id = -1;
    if (tid < k) {
      id = p.ids[row * k + tid];
      u = clean(p.values[row * k + tid]);
      u = fminf(u * p.scale, kLargest);
      if (id < 0 || id >= W || !(u > kNegInf)) {
        id = -1;
        u = kNegInf;
      }
    }
    if (p.tail) rest = clean(p.tail[row]);
    for (int i = tid; i < (W + 31) / 32; i += kN) listed[i] = 0;
    const float mt = fmaxf(block_max<kN>(u, red), rest);
    if (mt > kNegInf) {
      const float e = u > kNegInf ? exp2_((u - mt) * kLog2e) : 0.0f;
      Z = block_sum<kN>(e, red) + (rest > kNegInf ? exp2_((rest - mt) * kLog2e) : 0.0f);
      if (tid < k) {
        ids[tid] = id;
        prob[tid] = e / Z;
      }
      if (id >= 0) atomicOr(&listed[id >> 5], 1u << (id & 31));
    } else {
      there = false;
    }
    __syncthreads();
    if (there) {
      for (int c = tid; c < W; c += kN) {
        const float v = to_float(x[c]) * p.scale;
        m = fmaxf(m, v);
        if (!((listed[c >> 5] >> (c & 31)) & 1u)) mr = fmaxf(mr, v);
      }
      m = block_max<kN>(m, red);
      mr = block_max<kN>(mr, red);
      float nan = 0.0f;  // a NaN score makes the row's loss and gradient NaN
      for (int c = tid; c < W; c += kN) {
        const float v = to_float(x[c]);
        if (v != v) nan = 1.0f;
      }
      nan = block_max<kN>(nan, red);
      if (nan != 0.0f) m = __builtin_nanf("");
      if (m == kNegInf) there = false;
    }
    if (there) {
      float s = 0.0f, sr = 0.0f;
      for (int c = tid; c < W; c += kN) {
        const float v = to_float(x[c]) * p.scale;
        s += exp2_((v - m) * kLog2e);
        if (v > kNegInf && !((listed[c >> 5] >> (c & 31)) & 1u)) sr += exp2_((v - mr) * kLog2e);
      }
      s = block_sum<kN>(s, red);
      sr = block_sum<kN>(sr, red);
      const float lse = m + logf(s);
      const float pr = rest > kNegInf ? exp2_((rest - mt) * kLog2e) / Z : 0.0f;
      float term = 0.0f, P = 0.0f;
      if (id >= 0) {
        bool first = true;
        for (int i = 0; i < k; ++i)
          if (ids[i] == id) {
            if (i < tid) first = false;
            P += prob[i];
          }
        if (!first) id = -1;
      }
      const float w = (p.weights ? p.weights[b * p.weight_stride_b + t * p.weight_stride_t] : p.weight) * p.scale;
      if (id >= 0) {
        const float v = to_float(x[id]) * p.scale;
        if (P > 0.0f) term = P * (logf(P) - (v - lse));
        if (grad) from_float((exp2_((v - m) * kLog2e) / s - P) * w, &grad[id]);
      }
      if (tid == 0 && pr > 0.0f) term += pr * (rest - mt - logf(Z) - (sr > 0.0f ? mr + logf(sr) - lse : kNegInf));
      term = block_sum<kN>(term, red);
      if (p.loss && tid == 0) p.loss[row] = term;
      if (grad) {
        const float a = 1.0f / s, c1 = sr > 0.0f ? pr / sr : 0.0f;
        for (int c = tid; c < W; c += kN) {
          if ((listed[c >> 5] >> (c & 31)) & 1u) continue;
          const float v = to_float(x[c]) * p.scale;
          float g = exp2_((v - m) * kLog2e) * a;
          if (v > kNegInf) g -= exp2_((v - mr) * kLog2e) * c1;
          from_float(g * w, &grad[c]);
        }
      }
      return;
    }
  }
  if (p.loss && tid == 0) p.loss[row] = 0.0f;
  if (grad)
    for (int c = tid; c < W; c += kN) from_float(0.0f, &grad[c]);
}

template <typename P, typename F>
hipError_t by_type(const P& p, F f) {
  if (p.in.type == kTypeF32) f(float());
  else if (p.in.type == kTypeF16) f(F16());
  else f(BF16());
  return hipGetLastError();
}

}  // namespace rows

hipError_t launch_distill(const DistillParams& p, hipStream_t stream) {
  return rows::by_type(p, [&](auto t) {
    rows::distill_kernel<decltype(t)><<<p.in.B * p.in.T, rows::kN, 0, stream>>>(p);
  });
}
}  // namespace ctcbeam

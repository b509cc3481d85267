// Device side of the row operators: a row held in registers, sums and maxima
// over the threads of a row, and the treatment of values that are no number.
#pragma once

#include <type_traits>

#include "ctcbeam_lane.h"
#include "ctcbeam_rows.h"
#include "ctcbeam_rows_plan.h"

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
// one rounding, to nearest even
__device__ __forceinline__ void from_float(float v, float* o) { *o = v; }
__device__ __forceinline__ void from_float(float v, F16* o) { o->u = __builtin_bit_cast(uint16_t, static_cast<_Float16>(v)); }
__device__ __forceinline__ void from_float(float v, BF16* o) { o->u = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }

// NaN counts as -inf, +inf as the largest number
__device__ __forceinline__ float clean(float v) { return fminf(fmaxf(v, kNegInf), kLargest); }

__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint16_t bits_of(F16 v) { return v.u; }
__device__ __forceinline__ uint16_t bits_of(BF16 v) { return v.u; }
__device__ __forceinline__ float from_bits(uint32_t u, float) { return __uint_as_float(u); }
template <typename T>
__device__ __forceinline__ T from_bits(uint16_t u, T) { return T{u}; }

// The hardware's 2^x, logarithm and reciprocal: one step of fp32 each, for the
// numbers they are asked for here (sums from 1 on, exponents from 0 down).
__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float log_(float v) { return __builtin_amdgcn_logf(v) * kLn2; }
__device__ __forceinline__ float rcp_(float v) { return __builtin_amdgcn_rcpf(v); }

// The larger of three (of two); where one is NaN, any of them.
__device__ __forceinline__ float max3_any(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// 16 bytes at any address: rows of an odd number of labels start anywhere.
struct __attribute__((packed, aligned(2))) Bytes16 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) Floats4 { float f[4]; };

template <typename T>
struct Packed {
  static constexpr int kVec = 16 / static_cast<int>(sizeof(T));
};
__device__ __forceinline__ void unpack(const Bytes16& b, float* o, float) {
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(b.w[i]);
}
__device__ __forceinline__ void unpack(const Bytes16& b, float* o, F16) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = to_float(F16{static_cast<uint16_t>(b.w[i])});
    o[2 * i + 1] = to_float(F16{static_cast<uint16_t>(b.w[i] >> 16)});
  }
}
__device__ __forceinline__ void unpack(const Bytes16& b, float* o, BF16) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = __uint_as_float(b.w[i] << 16);
    o[2 * i + 1] = __uint_as_float(b.w[i] & 0xFFFF0000u);
  }
}

// 16 bytes of values, each rounded once
__device__ __forceinline__ uint4 pack(const float* v, float) {
  return {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float* v, T) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    T lo, hi;
    from_float(v[2 * i], &lo);
    from_float(v[2 * i + 1], &hi);
    w[i] = static_cast<uint32_t>(lo.u) | (static_cast<uint32_t>(hi.u) << 16);
  }
  return {w[0], w[1], w[2], w[3]};
}

// Which of a workgroup's rows a thread is at: the same for its whole wave,
// which keeps the row's addresses in scalar registers.
template <int N>
__device__ __forceinline__ int team_of() {
  if constexpr (N >= kThreads) return 0;
  else return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / N);
}

// ---- over a wave: every lane gets the result, and the same bits of it ----
template <typename Op>
__device__ __forceinline__ float wave_join(float v, Op op) {
  const auto dpp = [](float x, auto ctrl) {
    return __uint_as_float(detail::dpp_full<decltype(ctrl)::value>(__float_as_uint(x)));
  };
  v = op(v, dpp(v, std::integral_constant<int, detail::kDppQuadXor1>{}));
  v = op(v, dpp(v, std::integral_constant<int, detail::kDppQuadXor2>{}));
  v = op(v, dpp(v, std::integral_constant<int, 0x141>{}));  // mirrored within 8 lanes
  v = op(v, dpp(v, std::integral_constant<int, 0x140>{}));  // mirrored within 16
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
__device__ __forceinline__ float wave_max(float v) { return wave_join(v, Max()); }
__device__ __forceinline__ float wave_sum(float v) { return wave_join(v, Sum()); }

// ---- over the N threads of a row: a wave, or the whole workgroup ----
// Consecutive calls use the two halves of `lds` in turn, so one barrier a call
// is enough.
template <int N>
struct Team {
  float (*lds)[N / 64];  // [4]
  int turn = 0;
  __device__ __forceinline__ explicit Team(float (*l)[N / 64]) : lds(l) {}
  // two values by the same operation
  template <typename Op>
  __device__ __forceinline__ void join2(float& a, float& b, Op op) {
    a = wave_join(a, op);
    b = wave_join(b, op);
    if constexpr (N > 64) {
      if ((threadIdx.x & 63) == 0) {
        lds[turn][threadIdx.x >> 6] = a;
        lds[turn + 1][threadIdx.x >> 6] = b;
      }
      __syncthreads();
      a = lds[turn][0];
      b = lds[turn + 1][0];
#pragma unroll
      for (int i = 1; i < N / 64; ++i) {
        a = op(a, lds[turn][i]);
        b = op(b, lds[turn + 1][i]);
      }
      turn ^= 2;
    }
  }
  template <typename Op>
  __device__ __forceinline__ float join(float v, Op op) {
    v = wave_join(v, op);
    if constexpr (N > 64) {
      if ((threadIdx.x & 63) == 0) lds[turn][threadIdx.x >> 6] = v;
      __syncthreads();
      v = lds[turn][0];
#pragma unroll
      for (int i = 1; i < N / 64; ++i) v = op(v, lds[turn][i]);
      turn ^= 2;
    }
    return v;
  }
  __device__ __forceinline__ float max(float v) { return join(v, Max()); }
  __device__ __forceinline__ float sum(float v) { return join(v, Sum()); }
  // between what one thread of the row writes to LDS and another reads
  __device__ __forceinline__ void sync() {
    if constexpr (N > 64) __syncthreads();
    else wave_order();
  }
  // the same within a wave, whose LDS accesses complete in order: nothing is
  // to be reordered by the compiler
  __device__ __forceinline__ void wave_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
};

// The labels of a row (or of a span of it), spread over N threads: first whole
// vectors of 16 bytes a thread, i-th vector at label (i*N + tid)*kVec, then
// what is left label by label, j-th at base + j*N + tid.  An odd number of
// labels costs one load more, not a half-empty vector.
template <typename T, int N, int F>
struct Layout {
  static constexpr int kVec = Packed<T>::kVec, kVecs = F / kVec;
  int W, tid, vecs, base, left;
  __device__ __forceinline__ Layout(int w, int t) : W(w), tid(t) {
    vecs = w / (N * kVec);
    base = vecs * N * kVec;
    left = (w - base + N - 1) / N;
  }
  __device__ __forceinline__ int vec_label(int i) const { return (i * N + tid) * kVec; }
  __device__ __forceinline__ int left_label(int j) const { return base + j * N + tid; }
  // f(e, label, value index) for every label of this thread
  template <typename Fn>
  __device__ __forceinline__ void each(Fn f) const {
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (i < vecs) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) f(i * kVec + e, vec_label(i) + e);
      }
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      if (j >= left) break;
      if (left_label(j) < W) f(F + j, left_label(j));
    }
  }
};

// A row as it was read; each pass over it unpacks it again.
template <typename T, int N, int F>
struct RawRow {
  using L = Layout<T, N, F>;
  Bytes16 raw[L::kVecs] = {};
  T one[L::kVec] = {};
  RawRow() = default;
  __device__ __forceinline__ RawRow(const L& lay, const T* row) { load(lay, row); }
  __device__ __forceinline__ void load(const L& lay, const T* row) {
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i)
      if (i < lay.vecs) raw[i] = *reinterpret_cast<const Bytes16*>(row + lay.vec_label(i));
#pragma unroll
    for (int j = 0; j < L::kVec; ++j) {
      if (j >= lay.left) break;
      if (lay.left_label(j) < lay.W) one[j] = row[lay.left_label(j)];
    }
  }
  // f(value, label, there) for the labels of this thread, by all threads alike:
  // `there` is false behind the last label
  template <typename Fn>
  __device__ __forceinline__ void every(const L& lay, Fn f) {
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i)
      if (i < lay.vecs) {
        forget(i);
        float v[L::kVec];
        unpack(raw[i], v, T());
        int label = lay.vec_label(i);
        asm volatile("" : "+v"(label));  // (nor are all the labels kept)
#pragma unroll
        for (int e = 0; e < L::kVec; ++e) f(v[e], label + e, true);
      }
#pragma unroll
    for (int j = 0; j < L::kVec; ++j)
      if (j < lay.left) f(to_float(one[j]), lay.left_label(j), lay.left_label(j) < lay.W);
  }
  template <typename Fn>
  __device__ __forceinline__ void each(const L& lay, Fn f) {
    every(lay, [&](float v, int label, bool there) {
      if (there) f(v, label);
    });
  }
  // x[0 .. F+kVec): the values as fp32, as Layout::each counts them
  __device__ __forceinline__ void values(const L& lay, float* x) const {
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i)
      if (i < lay.vecs) unpack(raw[i], x + i * L::kVec, T());
#pragma unroll
    for (int j = 0; j < L::kVec; ++j) {
      if (j >= lay.left) break;
      x[L::kVecs * L::kVec + j] = to_float(one[j]);
    }
  }
  // the largest value, where no value is NaN
  __device__ __forceinline__ float largest(const L& lay) const {
    float m = kNegInf;
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i)
      if (i < lay.vecs) {
        float v[L::kVec];
        unpack(raw[i], v, T());
#pragma unroll
        for (int e = 0; e < L::kVec; e += 2) m = max3_any(m, v[e], v[e + 1]);
      }
#pragma unroll
    for (int j = 0; j < L::kVec; ++j) {
      if (j >= lay.left) break;
      if (lay.left_label(j) < lay.W) m = fmaxf(m, to_float(one[j]));
    }
    return m;
  }
  // the i-th value as Layout::each counts them, i known when unrolled
  __device__ __forceinline__ float value(int i) const {
    if (i >= F) return to_float(one[i - F]);
    float v[L::kVec];
    unpack(raw[i / L::kVec], v, T());
    return v[i % L::kVec];
  }
  // What follows unpacks the row anew, instead of keeping unpacked (or
  // otherwise derived) values of all labels in registers from before.
  __device__ __forceinline__ void forget() {
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i) forget(i);
  }
  // The same for one vector, in the order of the program: its values are not
  // unpacked while others are still worked on.
  __device__ __forceinline__ void forget(int i) {
#pragma unroll
    for (int w = 0; w < 4; ++w) asm volatile("" : "+v"(raw[i].w[w]));
  }
};

// kVec fp32 values at an address of 4-byte alignment
template <int V>
__device__ __forceinline__ void load_floats(const float* p, float* o) {
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    const Floats4 f = reinterpret_cast<const Floats4*>(p)[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[4 * i + e] = f.f[e];
  }
}
template <int V>
__device__ __forceinline__ void store_floats(float* p, const float* v) {
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    Floats4 f;
#pragma unroll
    for (int e = 0; e < 4; ++e) f.f[e] = v[4 * i + e];
    reinterpret_cast<Floats4*>(p)[i] = f;
  }
}

__device__ __forceinline__ int length_of(const RowsView& v, int b) {
  if (!v.lengths) return v.T;
  const int l = v.lengths[b];
  return l < 0 ? 0 : (l > v.T ? v.T : l);
}

__device__ __forceinline__ Part join_parts(const Part* parts, int n) {
  const int lane = threadIdx.x & 63;
  float m = kNegInf, s = 0.0f;
  for (int i = lane; i < n; i += 64) m = fmaxf(m, parts[i].m);
  m = wave_max(m);
  for (int i = lane; i < n; i += 64) {
    const Part p = parts[i];
    if (p.m > kNegInf) s += p.s * exp2_((p.m - m) * kLog2e);
  }
  return {m, wave_sum(s)};
}

}  // namespace rows
}  // namespace ctcbeam

// Distillation from a teacher's top logits: the divergence of each frame and
// its gradient, in one pass over the student's row.
//
//   Z = sum_i exp(u_i) + exp(tail), P_c = sum_(i of c) exp(u_i) / Z, P_r = exp(tail) / Z
//   r, m: the largest score of the labels that are not listed, and of all
//   R = sum over the labels that are not listed of e_c, e_c = exp(s (x_c - r))
//   S = R exp(s (r - m)) + sum over the listed labels of exp(s (x_c - m))
//   loss = sum_c P_c (log P_c - s (x_c - m) + log S) + P_r (log P_r - s (r - m) - log R + log S)
//   grad_c = w s (exp(s (x_c - m)) / S - P_c) where listed,
//            w s (exp(s (r - m)) / S - P_r / R) e_c elsewhere
//
// The listed labels are taken out of the row (set to -inf) as soon as it is
// there, and come back as they are written.  So the passes over the row know
// nothing of the list, R is a sum of its own at its own scale, never S less the
// listed labels, and neither the loss nor the gradient cancels.
//
// What bounds it is memory, the row in and the gradient out, and for 16-bit rows
// nearly as much the exponentials and conversions: 19200 of 25600 rows of 1025
// bf16 labels, k = 16, take 24 us for 92 MB, 3.8 TB/s (a table of the list's
// probabilities beside the row, read in both passes, took 34 us); fp32 rows of
// that length 4.5 TB/s, a copy 5.2.
//
// A wave takes rows of fewer than 2304 labels where there are many, a workgroup of
// 256 rows of fewer than 9216, through a copy of the row in LDS in which the
// list is taken out and put back.  Longer rows are held by a workgroup of 256 to
// 1024, in packed registers, with a bit per label in LDS; or, where they are few
// or longer than that, cut into spans whose sums a second launch joins.  2048
// rows of 131072 bf16 labels, k = 64: 276 us for 1.07 GB, 3.9 TB/s; in spans
// 345 us.
//
// Scores, sums and probabilities are fp32; a gradient is rounded once, to the
// student's type.
#pragma once

#include "ctcbeam_rows_lane.h"
#include "ctcbeam_rows_plan.h"

namespace ctcbeam {
namespace rows {

enum DistillPhase { kOneLaunch = 0, kSpanSums = 1, kSpanGrads = 2 };

// The teacher's list of a row, two entries a lane.
struct List {
  int id[2];  // label within the span, -1: no entry of this span
  float prob[2], log_prob[2], score[2];
  float rest_p, log_rest_p;
  bool any, two;  // more than 64 entries: the lanes' second ones

  List() = default;
  __device__ __forceinline__ List(const DistillParams& p, int64_t row, int c0, int W) {
    const int lane = threadIdx.x & 63;
    two = p.k > 64;
    float u[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = lane + 64 * e;
      u[e] = kNegInf;
      id[e] = -1;
      prob[e] = log_prob[e] = score[e] = 0.0f;
      if (e == 1 && !two) break;
      if (i < p.k) {
        const int at = p.ids[row * p.k + i];
        const float v = clean(p.values[row * p.k + i]);
        if (at >= 0 && at < p.in.W && v > kNegInf) {
          id[e] = at - c0;
          u[e] = fminf(v * p.scale, kLargest);
        }
      }
      if (id[e] >= W) id[e] = -1;
    }
    const float rest = p.tail ? clean(p.tail[row]) : kNegInf;
    const float mt = fmaxf(wave_max(fmaxf(u[0], u[1])), rest);
    any = mt > kNegInf;
    const float m0 = any ? mt : 0.0f;
    each([&](int e) { prob[e] = exp2_((u[e] - m0) * kLog2e); });
    const float rest_e = exp2_((rest - m0) * kLog2e), Z = wave_sum(prob[0] + prob[1]) + rest_e;
    const float log_z = log_(Z), per_z = rcp_(Z);
    rest_p = rest_e * per_z;
    log_rest_p = (rest - m0) - log_z;
    each([&](int e) {
      prob[e] *= per_z;
      log_prob[e] = (u[e] - m0) - log_z;
    });
  }

  template <typename Fn>
  __device__ __forceinline__ void each(Fn f) const {
    f(0);
    if (two) f(1);
  }

  // Labels listed more than once: their first entry takes the sum, in the
  // list's order, the others are no entries.
  __device__ __forceinline__ void sum_equal_labels(int k) {
    const int lane = threadIdx.x & 63;
    float sum[2] = {0.0f, 0.0f};
    int first[2] = {kMaxTop, kMaxTop};
#pragma unroll
    for (int h = 0; h < 2; ++h)
      for (int i = 0; i < k - 64 * h && i < 64; ++i) {
        const int other = detail::rdlane(id[h], i);
        const float more = detail::rdlane(prob[h], i);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool equal = other == id[e];
          sum[e] += equal ? more : 0.0f;
          first[e] = min(first[e], equal ? i + 64 * h : kMaxTop);
        }
      }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (id[e] < 0) continue;
      prob[e] = sum[e];
      log_prob[e] = logf(sum[e]);
      if (first[e] != lane + 64 * e) id[e] = -1;
    }
  }

  __device__ __forceinline__ float largest() const {
    return fmaxf(id[0] >= 0 ? score[0] : kNegInf, id[1] >= 0 ? score[1] : kNegInf);
  }
  // the listed labels' sum relative to m
  __device__ __forceinline__ float sum(float m, float c) const {
    float s = 0.0f;
    each([&](int e) {
      if (id[e] >= 0) s += exp2_((score[e] - m) * c);
    });
    return s;
  }
  // their part of the loss but for log S
  __device__ __forceinline__ float terms(float m, float scale) const {
    float t = 0.0f;
    each([&](int e) {
      if (id[e] >= 0 && prob[e] > 0.0f) t += prob[e] * (log_prob[e] - (score[e] - m) * scale);
    });
    return t;
  }
  __device__ __forceinline__ float listed() const {
    return (id[0] >= 0 ? prob[0] : 0.0f) + (id[1] >= 0 ? prob[1] : 0.0f);
  }
};

// What the sums of a row make: its loss, from the listed labels' part of it,
// and the factors of the gradient.
struct RowSums {
  float m, r, R, S;
  __device__ __forceinline__ RowSums(float m_, float r_, float R_, float listed_sum, float c) : m(m_), r(r_), R(R_) {
    // (with nothing above -inf, R is 0, or NaN where a score is)
    S = (r > kNegInf ? R * exp2_((r - m) * c) : R) + listed_sum;
  }
  // the part of the loss of the labels that are not listed
  __device__ __forceinline__ float rest_loss(const List& list, float scale) const {
    if (!(list.rest_p > 0.0f)) return 0.0f;
    const float log_q = R > 0.0f ? (r - m) * scale + log_(R) - log_(S) : S != S ? S : kNegInf;
    return list.rest_p * (list.log_rest_p - log_q);
  }
  __device__ __forceinline__ float listed_factor(float w) const { return w * rcp_(S); }
  __device__ __forceinline__ float rest_factor(float w, float c, float rest_p) const {
    return (r > kNegInf ? exp2_((r - m) * c) : 0.0f) * (w * rcp_(S)) - (R > 0.0f ? w * rest_p * rcp_(R) : 0.0f);
  }
};

__device__ __forceinline__ float row_weight(const DistillParams& p, int b, int t) {
  return (p.weights ? p.weights[b * p.weight_stride_b + t * p.weight_stride_t] : p.weight) * p.scale;
}

// Loss 0 and gradient 0.
template <typename T, int N, int F>
__device__ __forceinline__ void store_nothing(const Layout<T, N, F>& lay, T* grad, float* loss) {
  if (loss && lay.tid == 0) *loss = 0.0f;
  if (grad) {
#pragma unroll
    for (int i = 0; i < Layout<T, N, F>::kVecs; ++i)
      if (i < lay.vecs) *reinterpret_cast<Bytes16*>(grad + lay.vec_label(i)) = Bytes16{};
#pragma unroll
    for (int j = 0; j < Layout<T, N, F>::kVec; ++j) {
      if (j >= lay.left) break;
      if (lay.left_label(j) < lay.W) grad[lay.left_label(j)] = T{};
    }
  }
}

__device__ __forceinline__ float reference(float m) { return m > kNegInf ? m : 0.0f; }

template <typename T, int N, int F, int PHASE>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(F > 16 ? 4 : 8)))
distill_kernel(const DistillParams p, const DistillPlan plan, SpanSums* sums) {
  using L = Layout<T, N, F>;
  constexpr int V = L::kVec, kTeams = kThreads / N;
  extern __shared__ __align__(16) char stages[];
  __shared__ float red_all[kTeams][4][N / 64];
  const int tid = threadIdx.x % N, team = team_of<N>(), lane = threadIdx.x & 63;
  const bool first_wave = tid < 64;
  Team<N> tm(red_all[team]);
  const uint32_t at = blockIdx.x * kTeams + team, T_ = p.in.T;
  if (at >= p.in.B * T_) return;  // (a wave's row: no barrier is passed below)
  const int b = at / T_, t = at % T_;
  const int64_t row = at;
  const int span = PHASE == kOneLaunch ? 0 : blockIdx.y, c0 = PHASE == kOneLaunch ? 0 : span * plan.span;
  const L lay(PHASE == kOneLaunch ? p.in.W : min(p.in.W - c0, plan.span), tid);
  T* grad = p.grad && PHASE != kSpanSums ? static_cast<T*>(p.grad) + b * p.grad_stride_b + t * p.grad_stride_t + c0 : nullptr;
  float* loss = p.loss && PHASE != kSpanSums && span == 0 ? p.loss + row : nullptr;
  if (t >= length_of(p.in, b)) return store_nothing(lay, grad, loss);
  RawRow<T, N, F> x(lay, static_cast<const T*>(p.in.data) + b * p.in.stride_b + t * p.in.stride_t + c0);
  List list(p, row, c0, lay.W);
  if (!list.any) return store_nothing(lay, grad, loss);

  // the list out of the row
  T* stage = reinterpret_cast<T*>(stages) + team * ((lay.W + V - 1) / V * V);
#pragma unroll
  for (int i = 0; i < L::kVecs; ++i)
    if (i < lay.vecs) *reinterpret_cast<uint4*>(stage + lay.vec_label(i)) = __builtin_bit_cast(uint4, x.raw[i]);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (j >= lay.left) break;
    if (lay.left_label(j) < lay.W) stage[lay.left_label(j)] = x.one[j];
  }
  tm.sync();
  if (first_wave) {
    using Mark = decltype(bits_of(T{}));
    volatile Mark* mark = reinterpret_cast<volatile Mark*>(stage);
    bool again = false;
    list.each([&](int d) {
      if (list.id[d] >= 0) list.score[d] = to_float(from_bits(mark[list.id[d]], T{}));
    });
    list.each([&](int d) {
      if (list.id[d] >= 0) mark[list.id[d]] = static_cast<Mark>(lane + 64 * d);
    });
    tm.wave_order();
    list.each([&](int d) {
      if (list.id[d] >= 0) again |= mark[list.id[d]] != static_cast<Mark>(lane + 64 * d);
    });
    if (__ballot(again)) list.sum_equal_labels(p.k);
    tm.wave_order();
    T none;
    from_float(kNegInf, &none);
    list.each([&](int d) {
      if (list.id[d] >= 0) mark[list.id[d]] = bits_of(none);
    });
  }
  tm.sync();
#pragma unroll
  for (int i = 0; i < L::kVecs; ++i)
    if (i < lay.vecs) x.raw[i] = __builtin_bit_cast(Bytes16, *reinterpret_cast<const uint4*>(stage + lay.vec_label(i)));
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (j >= lay.left) break;
    if (lay.left_label(j) < lay.W) x.one[j] = stage[lay.left_label(j)];
  }

  const float c = p.scale * kLog2e;
  float m, r, R, listed_sum, terms, listed;
  if (PHASE == kSpanGrads) {
    const SpanSums* all = sums + row * plan.spans;
    m = r = kNegInf;
    for (int i = lane; i < plan.spans; i += 64) {
      m = fmaxf(m, all[i].m);
      if (all[i].R > 0.0f) r = fmaxf(r, all[i].r);
    }
    m = wave_max(m);
    r = wave_max(r);
    R = listed_sum = terms = listed = 0.0f;
    for (int i = lane; i < plan.spans; i += 64) {
      const SpanSums a = all[i];
      R += a.R > 0.0f ? a.R * exp2_((a.r - r) * c) : a.R;
      if (a.listed_sum != 0.0f) listed_sum += a.listed_sum * exp2_((reference(a.m) - reference(m)) * c);
      if (a.listed > 0.0f) terms += a.terms + a.listed * ((reference(m) - reference(a.m)) * p.scale);
      listed += a.listed;
    }
    R = wave_sum(R);
    listed_sum = wave_sum(listed_sum);
  } else {
    r = x.largest(lay);
    m = first_wave ? fmaxf(r, list.largest()) : r;
    tm.join2(r, m, Max());
    R = 0.0f;
  }
  float e[F + V];
  if (PHASE != kSpanGrads || grad) {
    const float ref = reference(r);
    lay.each([&](int i, int) {
      e[i] = exp2_((x.value(i) - ref) * c);
      if (PHASE != kSpanGrads) R += e[i];
    });
  }
  if (PHASE != kSpanGrads) {
    listed_sum = first_wave ? list.sum(reference(m), c) : 0.0f;
    tm.join2(R, listed_sum, Sum());
    terms = list.terms(reference(m), p.scale);
    listed = list.listed();
  }
  if (PHASE == kSpanSums) {
    if (first_wave) {
      terms = wave_sum(terms);
      listed = wave_sum(listed);
      if (tid == 0) sums[row * plan.spans + span] = {m, listed_sum, r, R, terms, listed};
    }
    return;
  }
  const RowSums of(reference(m), r, R, listed_sum, c);
  if (of.S == 0.0f) return store_nothing(lay, grad, loss);  // a row of -inf
  if (loss && first_wave) {
    // (of spans, each lane has sums of other spans)
    const float l = wave_sum(terms + (listed > 0.0f ? listed * log_(of.S) : 0.0f)) + of.rest_loss(list, p.scale);
    if (tid == 0) *loss = l;
  }
  if (!grad) return;

  // the gradient, and the list back into it
  const float w = row_weight(p, b, t), rest = of.rest_factor(w, c, list.rest_p);
#pragma unroll
  for (int i = 0; i < L::kVecs; ++i)
    if (i < lay.vecs) {
      float o[V];
#pragma unroll
      for (int d = 0; d < V; ++d) o[d] = e[i * V + d] * rest;
      *reinterpret_cast<uint4*>(stage + lay.vec_label(i)) = pack(o, T{});
    }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (j >= lay.left) break;
    if (lay.left_label(j) < lay.W) from_float(e[F + j] * rest, &stage[lay.left_label(j)]);
  }
  tm.sync();
  if (first_wave) {
    const float a = of.listed_factor(w);
    list.each([&](int d) {
      if (list.id[d] >= 0) from_float(exp2_((list.score[d] - of.m) * c) * a - list.prob[d] * w, &stage[list.id[d]]);
    });
  }
  tm.sync();
#pragma unroll
  for (int i = 0; i < L::kVecs; ++i)
    if (i < lay.vecs)
      *reinterpret_cast<Bytes16*>(grad + lay.vec_label(i)) =
          __builtin_bit_cast(Bytes16, *reinterpret_cast<const uint4*>(stage + lay.vec_label(i)));
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (j >= lay.left) break;
    if (lay.left_label(j) < lay.W) grad[lay.left_label(j)] = stage[lay.left_label(j)];
  }
}

// Rows that a workgroup holds in packed registers (up to 124, none spilled).  A bit per
// label in LDS says which are listed; few vectors of a wave hold one, and only
// those look their gradient up, in a table of four places an entry, each
// label at the first free one from its own on.  One workgroup fills a compute unit, so reading,
// computing and writing overlap between units, not within one.
constexpr int kPlaces = 4 * kMaxTop;
static_assert(kPlaces == 512, "nine bits of the product");
// a label's own place: labels at even distances do not meet in one
__device__ __forceinline__ int place_of(int label) { return static_cast<int>(static_cast<uint32_t>(label) * 0x9E3779B1u >> 23); }

template <typename T, int N, int VECS>
__global__ void __launch_bounds__(N) distill_wide_kernel(const DistillParams p) {
  using L = Layout<T, N, VECS * Packed<T>::kVec>;
  constexpr int V = L::kVec, kWords = N * (VECS + 1) * V / 32;
  __shared__ __align__(16) uint32_t bits[kWords];
  __shared__ float red[4][N / 64];
  __shared__ int place_label[kPlaces];
  __shared__ float place_grad[kPlaces];
  __shared__ int any;
  __shared__ float rest_p;
  const int tid = threadIdx.x, lane = tid & 63;
  const bool first_wave = tid < 64;
  Team<N> tm(red);
  const uint32_t row = blockIdx.x, T_ = p.in.T;
  const int b = row / T_, t = row % T_;
  const L lay(p.in.W, tid);
  const T* in = static_cast<const T*>(p.in.data) + b * p.in.stride_b + t * p.in.stride_t;
  T* grad = p.grad ? static_cast<T*>(p.grad) + b * p.grad_stride_b + t * p.grad_stride_t : nullptr;
  float* loss = p.loss ? p.loss + row : nullptr;
  if (t >= length_of(p.in, b)) return store_nothing(lay, grad, loss);
  RawRow<T, N, L::kVecs * V> x(lay, in);
  List list;
  int place[2];
  for (int i = tid; i < (lay.W + 31) / 32; i += N) bits[i] = 0;
  for (int i = tid; i < kPlaces; i += N) place_label[i] = -1;
  if (first_wave) {
    list = List(p, row, 0, lay.W);
    list.each([&](int d) {
      if (list.id[d] >= 0) list.score[d] = to_float(in[list.id[d]]);
    });
    if (lane == 0) {
      any = list.any;
      rest_p = list.rest_p;
    }
  }
  __syncthreads();
  if (!any) return store_nothing(lay, grad, loss);
  if (first_wave) {
    bool again = false;
    list.each([&](int d) {
      const uint32_t bit = 1u << (list.id[d] & 31);
      if (list.id[d] >= 0) again |= (atomicOr(&bits[list.id[d] >> 5], bit) & bit) != 0;
    });
    if (__ballot(again)) list.sum_equal_labels(p.k);
    list.each([&](int d) {
      if (list.id[d] < 0) return;
      int at = place_of(list.id[d]);  // (at most kMaxTop labels: there is a free place)
      while (atomicCAS(&place_label[at], -1, list.id[d]) != -1) at = (at + 1) % kPlaces;
      place[d] = at;
    });
  }
  __syncthreads();

  // the list out of the row
  const uint8_t* bytes = reinterpret_cast<const uint8_t*>(bits);
  const auto flags_of = [&](int i) -> uint32_t {
    const int at = i * N + tid;
    if constexpr (V == 8) return bytes[at];
    else return (bytes[at >> 1] >> (at & 1) * 4) & 15u;
  };
  const auto is_listed = [&](int label) { return ((bits[label >> 5] >> (label & 31)) & 1u) != 0; };
  T none;
  from_float(kNegInf, &none);
  const uint32_t none_bits = bits_of(none);
#pragma unroll
  for (int i = 0; i < VECS; ++i)
    if (i < lay.vecs) {
      const uint32_t f = flags_of(i);
      if (__ballot(f != 0)) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t& u = x.raw[i].w[w];
          if constexpr (V == 8) {
            if ((f >> (2 * w)) & 1u) u = (u & 0xFFFF0000u) | none_bits;
            if ((f >> (2 * w)) & 2u) u = (u & 0x0000FFFFu) | (none_bits << 16);
          } else {
            if ((f >> w) & 1u) u = none_bits;
          }
        }
      }
    }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (j >= lay.left) break;
    if (lay.left_label(j) < lay.W && is_listed(lay.left_label(j))) x.one[j] = none;
  }

  const float c = p.scale * kLog2e;
  float r = x.largest(lay), m = first_wave ? fmaxf(r, list.largest()) : r;
  tm.join2(r, m, Max());
  const float ref = reference(r);
  float R = 0.0f, listed_sum = first_wave ? list.sum(reference(m), c) : 0.0f;
  x.forget();
  x.each(lay, [&](float v, int) { R += exp2_((v - ref) * c); });
  tm.join2(R, listed_sum, Sum());
  const RowSums of(reference(m), r, R, listed_sum, c);
  if (of.S == 0.0f) return store_nothing(lay, grad, loss);  // a row of -inf
  const float w = row_weight(p, b, t);
  if (first_wave) {
    if (loss) {
      const float listed = list.listed();
      const float l = wave_sum(list.terms(of.m, p.scale) + (listed > 0.0f ? listed * log_(of.S) : 0.0f));
      if (lane == 0) *loss = l + of.rest_loss(list, p.scale);
    }
    const float a = of.listed_factor(w);
    list.each([&](int d) {
      const float g = exp2_((list.score[d] - of.m) * c) * a - list.prob[d] * w;
      if (list.id[d] >= 0) place_grad[place[d]] = g;
    });
  }
  if (!grad) return;
  __syncthreads();
  const float rest = of.rest_factor(w, c, rest_p);
  x.forget();
  const auto gradient_of = [&](int label) {
    int at = place_of(label);  // (a listed label: it has a place)
    while (place_label[at] != label) at = (at + 1) % kPlaces;
    return place_grad[at];
  };
#pragma unroll
  for (int i = 0; i < VECS; ++i)
    if (i < lay.vecs) {
      float v[V], o[V];
      unpack(x.raw[i], v, T());
#pragma unroll
      for (int d = 0; d < V; ++d) o[d] = exp2_((v[d] - ref) * c) * rest;
      uint32_t f = flags_of(i);
      while (f) {
        const int at = __ffs(f) - 1;
        const float g = gradient_of(lay.vec_label(i) + at);
#pragma unroll
        for (int d = 0; d < V; ++d) o[d] = d == at ? g : o[d];
        f &= f - 1;
      }
      *reinterpret_cast<Bytes16*>(grad + lay.vec_label(i)) = __builtin_bit_cast(Bytes16, pack(o, T{}));
    }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if (j >= lay.left) break;
    const int label = lay.left_label(j);
    if (label < lay.W)
      from_float(is_listed(label) ? gradient_of(label) : exp2_((to_float(x.one[j]) - ref) * c) * rest, &grad[label]);
  }
}

template <typename T, int N, int F>
static void run_distill(const DistillParams& p, const DistillPlan& q, SpanSums* sums, hipStream_t stream) {
  constexpr int teams = kThreads / N;
  const int64_t rows = static_cast<int64_t>(p.in.B) * p.in.T;
  const size_t lds = static_cast<size_t>(teams) * ((std::min(q.span, p.in.W) * sizeof(T) + 15) / 16 * 16);
  const uint32_t groups = static_cast<uint32_t>((rows + teams - 1) / teams);
  if constexpr (N > 64) {
    if (q.spans > 1) {
      distill_kernel<T, N, F, kSpanSums><<<dim3(groups, q.spans), kThreads, lds, stream>>>(p, q, sums);
      distill_kernel<T, N, F, kSpanGrads><<<dim3(groups, p.grad ? q.spans : 1), kThreads, lds, stream>>>(p, q, sums);
      return;
    }
  }
  distill_kernel<T, N, F, kOneLaunch><<<groups, kThreads, lds, stream>>>(p, q, nullptr);
}

template <typename T>
static hipError_t launch_distill_impl(const DistillParams& p, void* workspace, hipStream_t stream) {
  SpanSums* sums = static_cast<SpanSums*>(workspace);
  const DistillPlan q = plan_distill(p.in.type, p.in.B, p.in.T, p.in.W);
  const uint32_t rows = static_cast<uint32_t>(p.in.B) * p.in.T;
  if (q.spans == 0) {
    const int vecs = q.f / Packed<T>::kVec;
    if (q.n == 1024 && vecs == 4) distill_wide_kernel<T, 1024, 4><<<rows, 1024, 0, stream>>>(p);
    else if (q.n == 1024 && vecs == 8) distill_wide_kernel<T, 1024, 8><<<rows, 1024, 0, stream>>>(p);
    else if (q.n == 1024) distill_wide_kernel<T, 1024, 16><<<rows, 1024, 0, stream>>>(p);
    else if (q.n == 512) distill_wide_kernel<T, 512, 16><<<rows, 512, 0, stream>>>(p);
    else if (vecs == 16) distill_wide_kernel<T, 256, 16><<<rows, 256, 0, stream>>>(p);
    // (8 vectors of fp32 hold rows of fewer than kRowOfGroup labels, which come through LDS)
    else if constexpr (Packed<T>::kVec == 8) distill_wide_kernel<T, 256, 8><<<rows, 256, 0, stream>>>(p);
  } else if (q.n == 64) q.f == 16 ? run_distill<T, 64, 16>(p, q, sums, stream) : run_distill<T, 64, 32>(p, q, sums, stream);
  else if (q.f == 8) run_distill<T, 256, 8>(p, q, sums, stream);
  else if (q.f == 16) run_distill<T, 256, 16>(p, q, sums, stream);
  else run_distill<T, 256, 32>(p, q, sums, stream);
  return hipGetLastError();
}

}  // namespace rows
}  // namespace ctcbeam

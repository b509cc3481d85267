// Distillation from a teacher's top logits: the divergence of each frame and
// its gradient, in one pass over the student's row.
//
//   Z = sum_i exp(u_i) + exp(tail), P_c = sum_(i of c) exp(u_i) / Z, P_r = exp(tail) / Z
//   e_c = exp(s (x_c - m)), S = sum e_c, R = sum of e_c over the labels that are not listed
//   loss = sum_c P_c (log P_c - log e_c + log S) + P_r (log P_r - log R + log S)
//   grad_c = w s (e_c / S - P_c) where listed, w s e_c (1 / S - P_r / R) elsewhere
//
// R is a sum of its own, never S less the listed labels, and where it is too
// small for fp32 beside m it is taken again relative to its own maximum, so
// neither the loss nor the gradient cancels.
//
// The row is read once into registers.  The teacher's probabilities are
// scattered to a table in LDS with a place for every label of the span, which
// both passes over the registers read beside them: whether a label is listed,
// and what to take from its gradient.  Labels listed twice are found by the
// scatter itself and summed in the order of the list.
//
// What bounds it is memory: the row in and the gradient out.  A wave takes
// rows of fewer than 2304 labels where there are many, a workgroup rows of
// fewer than 9216; longer ones are cut into spans whose sums a second launch
// joins, reading the row again for the gradient.
#include <algorithm>

#include "ctcbeam_rows_lane.h"

namespace ctcbeam {
namespace rows {

enum DistillPhase { kOneLaunch = 0, kSpanSums = 1, kSpanGrads = 2 };

struct DistillPlan {
  int n, f;   // threads of a row (of a span), labels of a thread
  int spans;  // per row
  int span;   // labels of a span (the last one may hold fewer)
};

// What a span leaves for the second launch: m and S; R relative to r; the
// listed labels' part of the loss but for log S, and their probability.
struct SpanSums {
  float m, S, r, R, terms, listed;
};

constexpr float kSmallRest = 0x1p-80f;      // R below this is taken again relative to its own maximum
constexpr float kListed = 1.17549435e-38f;  // least table entry of a listed label

__device__ __forceinline__ void store_vec(float* p, const float* v) { store_floats<4>(p, v); }
template <typename T>
__device__ __forceinline__ void store_vec(T* p, const float* v) {
  Bytes16 b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    T lo, hi;
    from_float(v[2 * i], &lo);
    from_float(v[2 * i + 1], &hi);
    b.w[i] = static_cast<uint32_t>(lo.u) | (static_cast<uint32_t>(hi.u) << 16);
  }
  *reinterpret_cast<Bytes16*>(p) = b;
}

template <typename T, int N, int F, int PHASE>
__global__ void __launch_bounds__(kThreads) distill_kernel(const DistillParams p, const DistillPlan plan, SpanSums* sums) {
  using L = Layout<T, N, F>;
  constexpr int V = L::kVec, kTeams = kThreads / N;
  extern __shared__ __align__(16) float tables[];
  __shared__ float red_all[kTeams][2][N / 64];
  const int tid = threadIdx.x % N, team = threadIdx.x / N, lane = threadIdx.x & 63;
  const bool first_wave = tid < 64;
  Team<N> tm(red_all[team]);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kTeams + team;
  if (row >= static_cast<int64_t>(p.in.B) * p.in.T) return;  // (a wave's row: no barrier is passed below)
  const int b = static_cast<int>(row / p.in.T), t = static_cast<int>(row % p.in.T);
  const int span = PHASE == kOneLaunch ? 0 : blockIdx.y, c0 = PHASE == kOneLaunch ? 0 : span * plan.span;
  const L lay(PHASE == kOneLaunch ? p.in.W : min(p.in.W - c0, plan.span), tid);
  const T* in = static_cast<const T*>(p.in.data) + b * p.in.stride_b + t * p.in.stride_t + c0;
  T* grad = p.grad && PHASE != kSpanSums ? static_cast<T*>(p.grad) + b * p.grad_stride_b + t * p.grad_stride_t + c0 : nullptr;
  const bool writes_loss = p.loss && PHASE != kSpanSums && span == 0 && first_wave;
  const auto nothing = [&]() {
    if (writes_loss && lane == 0) p.loss[row] = 0.0f;
    if (grad) {
#pragma unroll
      for (int i = 0; i < L::kVecs; ++i)
        if (i < lay.vecs) *reinterpret_cast<Bytes16*>(grad + lay.vec_label(i)) = Bytes16{};
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < lay.left && lay.left_label(j) < lay.W) grad[lay.left_label(j)] = T{};
    }
  };
  if (t >= length_of(p.in, b)) return nothing();

  // the teacher's list, two entries a lane, by every wave alike
  float u[2], prob[2], log_prob[2];
  int id[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int i = lane + 64 * e;
    u[e] = kNegInf;
    id[e] = -1;
    if (i < p.k) {
      const int at = p.ids[row * p.k + i];
      const float v = clean(p.values[row * p.k + i]);
      if (at >= 0 && at < p.in.W && v > kNegInf) {
        id[e] = at - c0;  // within this span or not
        u[e] = fminf(v * p.scale, kLargest);
      }
    }
    if (id[e] >= lay.W) id[e] = -1;
  }
  const float rest = p.tail ? clean(p.tail[row]) : kNegInf;
  const bool with_rest = rest > kNegInf;
  RawRow<T, N, F> x(lay, in);
  float at_id[2];  // the student's scores of the listed labels
#pragma unroll
  for (int e = 0; e < 2; ++e) at_id[e] = id[e] >= 0 && first_wave ? to_float(in[id[e]]) : 0.0f;

  const float mt = fmaxf(wave_max(fmaxf(u[0], u[1])), rest);
  if (!(mt > kNegInf)) return nothing();
#pragma unroll
  for (int e = 0; e < 2; ++e) prob[e] = exp2_((u[e] - mt) * kLog2e);
  const float rest_e = exp2_((rest - mt) * kLog2e), Z = wave_sum(prob[0] + prob[1]) + rest_e;
  const float log_z = logf(Z), rest_p = rest_e / Z;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    prob[e] /= Z;
    log_prob[e] = (u[e] - mt) - log_z;
  }

  // their table
  const int places = (lay.W + 3) / 4 * 4;
  float* table = tables + team * places;
  for (int i = tid; i < places / 4; i += N) reinterpret_cast<float4*>(table)[i] = float4{0.0f, 0.0f, 0.0f, 0.0f};
  tm.sync();
  if (first_wave) {
    bool again = false;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (id[e] >= 0) again |= atomicExch(&table[id[e]], fmaxf(prob[e], kListed)) != 0.0f;
    if (__ballot(again)) {
      // labels listed more than once: their first entry takes the sum, in the list's order
      float sum[2] = {0.0f, 0.0f};
      bool first[2] = {true, true};
      for (int i = 0; i < p.k; ++i) {
        const int other = i < 64 ? __shfl(id[0], i) : __shfl(id[1], i - 64);
        const float more = i < 64 ? __shfl(prob[0], i) : __shfl(prob[1], i - 64);
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (id[e] >= 0 && other == id[e]) {
            sum[e] += more;
            if (i < lane + 64 * e) first[e] = false;
          }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (id[e] >= 0) {
          if (first[e]) table[id[e]] = fmaxf(sum[e], kListed);
          prob[e] = first[e] ? sum[e] : 0.0f;
          log_prob[e] = logf(sum[e]);
        }
    }
  }
  tm.sync();

  // m, S, and R relative to r
  const float c = p.scale * kLog2e;
  float m, S, r, R;
  // f(values, table entries, first label) of each vector, then of each label left
  const auto with_table = [&](auto vec, auto one) {
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i)
      if (i < lay.vecs) {
        float v[V];
        unpack(x.raw[i], v, T());
        float q[V];
#pragma unroll
        for (int d = 0; d < V / 4; ++d) {
          const float4 f = *reinterpret_cast<const float4*>(&table[lay.vec_label(i) + 4 * d]);
          q[4 * d] = f.x;
          q[4 * d + 1] = f.y;
          q[4 * d + 2] = f.z;
          q[4 * d + 3] = f.w;
        }
        vec(v, q, lay.vec_label(i));
      }
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j < lay.left && lay.left_label(j) < lay.W) one(to_float(x.one[j]), table[lay.left_label(j)], lay.left_label(j));
  };
  const auto each_with_table = [&](auto f) {
    with_table(
        [&](const float* v, const float* q, int) {
#pragma unroll
          for (int e = 0; e < V; ++e) f(v[e], q[e]);
        },
        [&](float v, float q, int) { f(v, q); });
  };
  if (PHASE != kSpanGrads) {
    m = kNegInf;
    x.each(lay, [&](float v, int) { m = fmaxf(m, v); });
    m = tm.max(m);
    if (m == kNegInf) {
      // nothing but -inf, or NaN among it, which is to be seen
      float nan = 0.0f;
      x.each(lay, [&](float v, int) { nan = v != v ? 1.0f : nan; });
      if (tm.max(nan) != 0.0f) m = 0.0f;
      else if (PHASE == kOneLaunch) return nothing();
    }
    const float m0 = m == kNegInf ? 0.0f : m;
    S = R = 0.0f;
    r = m;
    x.forget();
    if (with_rest) {
      each_with_table([&](float v, float q) {
        const float e = exp2_((v - m0) * c);
        S += e;
        R += q != 0.0f ? 0.0f : e;
      });
      S = tm.sum(S);
      R = tm.sum(R);
      if (R < kSmallRest) {
        x.forget();
        r = kNegInf;
        each_with_table([&](float v, float q) { r = fmaxf(r, q != 0.0f ? kNegInf : v); });
        r = tm.max(r);
        R = 0.0f;
        if (r > kNegInf) {
          each_with_table([&](float v, float q) { R += q != 0.0f ? 0.0f : exp2_((v - r) * c); });
          R = tm.sum(R);
        }
      }
    } else {
      x.each(lay, [&](float v, int) { S += exp2_((v - m0) * c); });
      S = tm.sum(S);
    }
  }
  if (PHASE == kSpanSums) {
    float terms = 0.0f, listed = 0.0f;
    if (first_wave) {
      const float m0 = m == kNegInf ? 0.0f : m;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (id[e] >= 0 && prob[e] > 0.0f) {
          terms += prob[e] * (log_prob[e] - (at_id[e] - m0) * p.scale);
          listed += prob[e];
        }
      terms = wave_sum(terms);
      listed = wave_sum(listed);
      if (lane == 0) sums[row * plan.spans + span] = {m, S, r, R, terms, listed};
    }
    return;
  }
  float term = 0.0f;  // of the loss, but for the rest's
  if (PHASE == kSpanGrads) {
    const SpanSums* all = sums + row * plan.spans;
    m = r = kNegInf;
    for (int i = lane; i < plan.spans; i += 64) {
      m = fmaxf(m, all[i].m);
      if (all[i].R > 0.0f) r = fmaxf(r, all[i].r);
    }
    m = wave_max(m);
    r = wave_max(r);
    if (m == kNegInf) return nothing();
    S = R = 0.0f;
    float listed = 0.0f;
    for (int i = lane; i < plan.spans; i += 64) {
      const SpanSums a = all[i];
      if (a.m != kNegInf) S += a.S * exp2_((a.m - m) * c);
      if (a.R > 0.0f) R += a.R * exp2_((a.r - r) * c);
      if (a.listed > 0.0f) term += a.terms + a.listed * ((m - (a.m == kNegInf ? 0.0f : a.m)) * p.scale);
      listed += a.listed;
    }
    S = wave_sum(S);
    R = wave_sum(R);
    const float beside = R * exp2_((r - m) * c);
    if (beside >= kSmallRest) {
      R = beside;
      r = m;
    }
    term = wave_sum(term) + wave_sum(listed) * logf(S);
  } else {
    const float log_s = logf(S);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (id[e] >= 0 && prob[e] > 0.0f) term += prob[e] * (log_prob[e] - ((at_id[e] - m) * p.scale - log_s));
    if (writes_loss) term = wave_sum(term);
  }
  if (writes_loss && lane == 0) {
    if (rest_p > 0.0f) {
      const float log_q = R > 0.0f ? (r - m) * p.scale + logf(R) - logf(S) : S != S ? S : kNegInf;
      term += rest_p * ((rest - mt) - log_z - log_q);
    }
    p.loss[row] = term;
  }
  if (!grad) return;

  const float w = (p.weights ? p.weights[b * p.weight_stride_b + t * p.weight_stride_t] : p.weight) * p.scale;
  const float a = w / S, per_rest = R > 0.0f ? w * rest_p / R : 0.0f;
  x.forget();
  const auto store = [&](auto g) {
    with_table(
        [&](const float* v, const float* q, int label) {
          float o[V];
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = g(v[e], q[e]);
          store_vec(grad + label, o);
        },
        [&](float v, float q, int label) { from_float(g(v, q), &grad[label]); });
  };
  if (r == m || !(per_rest != 0.0f)) {
    const float a_rest = a - per_rest;
    store([&](float v, float q) { return exp2_((v - m) * c) * (q != 0.0f ? a : a_rest) - q * w; });
  } else {
    store([&](float v, float q) {
      const float e = exp2_((v - m) * c) * a;
      return q != 0.0f ? e - q * w : e - exp2_((v - r) * c) * per_rest;
    });
  }
}

static DistillPlan plan_distill(int B, int T, int W) {
  const int64_t rows = static_cast<int64_t>(B) * T;
  if (W < 64 * 36 && rows >= 1024) return {64, W < 64 * 20 ? 16 : 32, 1, W};
  if (W < 256 * 36) return {256, W < 256 * 12 ? 8 : W < 256 * 20 ? 16 : 32, 1, W};
  int span = 8192;
  while (span > 2048 && rows * ((W + span - 1) / span) < 512) span >>= 1;
  return {256, span / 256, (W + span - 1) / span, span};
}

template <typename T, int N, int F>
static void run_distill(const DistillParams& p, const DistillPlan& q, SpanSums* sums, hipStream_t stream) {
  constexpr int teams = kThreads / N;
  const int64_t rows = static_cast<int64_t>(p.in.B) * p.in.T;
  const size_t lds = sizeof(float) * teams * ((std::min(q.span, p.in.W) + 3) / 4 * 4);
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
static hipError_t choose_distill(const DistillParams& p, SpanSums* sums, hipStream_t stream) {
  const DistillPlan q = plan_distill(p.in.B, p.in.T, p.in.W);
  if (q.n == 64) q.f == 16 ? run_distill<T, 64, 16>(p, q, sums, stream) : run_distill<T, 64, 32>(p, q, sums, stream);
  else if (q.f == 8) run_distill<T, 256, 8>(p, q, sums, stream);
  else if (q.f == 16) run_distill<T, 256, 16>(p, q, sums, stream);
  else run_distill<T, 256, 32>(p, q, sums, stream);
  return hipGetLastError();
}

}  // namespace rows

size_t distill_workspace(int B, int T, int W) {
  const rows::DistillPlan q = rows::plan_distill(B, T, W);
  return q.spans == 1 ? 0 : static_cast<size_t>(B) * T * q.spans * sizeof(rows::SpanSums);
}

hipError_t launch_distill(const DistillParams& p, void* workspace, hipStream_t stream) {
  rows::SpanSums* sums = static_cast<rows::SpanSums*>(workspace);
  if (p.in.type == kTypeF32) return rows::choose_distill<float>(p, sums, stream);
  if (p.in.type == kTypeF16) return rows::choose_distill<rows::F16>(p, sums, stream);
  return rows::choose_distill<rows::BF16>(p, sums, stream);
}

}  // namespace ctcbeam

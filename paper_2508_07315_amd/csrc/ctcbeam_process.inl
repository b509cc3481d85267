// Penalties for repeated tokens, biases and grammar masks on logits, and the
// log-softmax that makes the decoders' input of them.
//
// A row is read once into registers (as fp32), changed there, and written.
// What bounds it is memory, W*(sizeof(T) + 4) bytes a row: without history,
// bias and mask 25600 fp32 rows of 1025 labels take 42 us, 5.0 TB/s, what a
// copy reaches; a bias, a mask and a history add 2 to 5 us each (their loads and
// selects), all of them 12.  Rows need not be aligned: 1024, 1025 and 1032
// labels run at the same rate.
//
// Rows of fewer than kRowOfWave labels belong to a wave, four rows of an
// utterance to a workgroup (several rows in turn by each wave, with the next one
// loaded ahead, measured slower: 50 us against 45); longer ones to a
// workgroup; rows beyond that, and rows too few to fill the card, are cut into
// spans of a workgroup each.  With a log-softmax the spans leave (max, sum) in
// the workspace, and a second launch reads them and the scores again, which are
// still in the caches: 64 rows of 131072 bf16 labels with a history of 2048 and
// a mask take 14.5 + 16.4 us for 50 MB.  Spans of 4096 and 2048 labels
// measured 16 + 18 and 18 + 21 us: each counts the whole history.
//
// The counts of the labels emitted before live in LDS, for the span that the
// workgroup holds, and serve all its frames.  Scores are fp32 from the load to
// the store; a sum's terms are added by lane, then across lanes.
#pragma once

#include "ctcbeam_rows_lane.h"
#include "ctcbeam_rows_plan.h"

namespace ctcbeam {
namespace rows {

enum Phase { kWhole = 0, kStats = 1, kFinish = 2 };

// (four waves a SIMD for 32 labels a thread: 16.4 us against 21 for the second
// launch above, though at 128 registers the second launch and the whole-row form
// spill 12 to 16 of them for 16-bit rows, 6 for fp32, 28 to 60 bytes a lane.  The forms
// of fewer labels spill none, and would under a bound: 57 us against 45)
template <typename T, int N, int F, int PHASE>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(F == 32 ? 4 : 1)))
process_kernel(const ProcessParams p, const ProcessPlan plan, Part* parts) {
  using L = Layout<T, N, F>;
  constexpr int V = L::kVec;
  extern __shared__ __align__(16) uint32_t count[];
  __shared__ float red[4][N / 64];
  const int tid = threadIdx.x % N, team = team_of<N>(), teams = kThreads / N;
  const int span = blockIdx.y, b = blockIdx.x / plan.groups;
  const int t0 = (blockIdx.x % plan.groups) * plan.frames;
  const int T1 = min(length_of(p.in, b), t0 + plan.frames);
  if (t0 >= T1) return;
  const int c0 = span * plan.span;
  const L lay(min(p.in.W - c0, plan.span), tid);
  Team<N> tm(red);

  // the first row is on its way while the history is counted
  const auto row_at = [&](int t) {
    return static_cast<const T*>(p.in.data) + b * p.in.stride_b + t * p.in.stride_t + c0;
  };
  RawRow<T, N, F> raw;
  if (t0 + team < T1) raw.load(lay, row_at(t0 + team));

  int H = p.H;
  float rep = 1.0f, pre = 0.0f, fre = 0.0f;
  if (H) {
    if (p.history_lengths) H = max(0, min(H, p.history_lengths[b]));
    rep = p.penalties ? p.penalties[3 * b] : p.repetition;
    pre = p.penalties ? p.penalties[3 * b + 1] : p.presence;
    fre = p.penalties ? p.penalties[3 * b + 2] : p.frequency;
  }
  const float per_rep = 1.0f / rep;  // (a quotient by way of it is off by a step and a half at most)
  if (H) {
    const int32_t* hist = p.history + b * p.history_stride;
    for (int i = threadIdx.x * 4; i < lay.W; i += kThreads * 4) *reinterpret_cast<uint4*>(&count[i]) = uint4{0, 0, 0, 0};
    __syncthreads();
    // four labels on their way at a time
    for (int i = threadIdx.x; i < H; i += 4 * kThreads) {
      uint32_t c[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        c[q] = i + q * kThreads < H ? static_cast<uint32_t>(hist[i + q * kThreads]) - static_cast<uint32_t>(c0) : ~0u;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (c[q] < static_cast<uint32_t>(lay.W)) atomicAdd(&count[c[q]], 1u);
    }
    __syncthreads();
  }
  const float* bias = p.bias ? p.bias + b * p.bias_stride + c0 : nullptr;

  for (int t = t0 + team; t < T1; t += teams) {
    const int64_t row = static_cast<int64_t>(b) * p.in.T + t;
    const uint32_t* mask = p.mask ? p.mask + b * p.mask_stride_b + t * p.mask_stride_t + (c0 >> 5) : nullptr;
    if (t >= t0 + teams) raw.load(lay, row_at(t));
    float x[F + V];
    raw.values(lay, x);
    const auto seen = [&](float v, uint32_t n) {
      const float w = clean((v * (v > 0.0f ? per_rep : rep) - fre * static_cast<float>(n)) - pre);
      return n ? w : v;
    };
    float m = kNegInf;
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i)
      if (i < lay.vecs) {
        const int c = lay.vec_label(i);
        float* y = x + i * V;
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = clean(y[e]);
        if (H) {
#pragma unroll
          for (int q = 0; q < V / 4; ++q) {
            const uint4 n = *reinterpret_cast<const uint4*>(&count[c + 4 * q]);
            if (n.x | n.y | n.z | n.w) {
              y[4 * q] = seen(y[4 * q], n.x);
              y[4 * q + 1] = seen(y[4 * q + 1], n.y);
              y[4 * q + 2] = seen(y[4 * q + 2], n.z);
              y[4 * q + 3] = seen(y[4 * q + 3], n.w);
            }
          }
        }
        if (bias) {
          float a[V];
          load_floats<V>(bias + c, a);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] = clean(y[e] + a[e]);
        }
        if (mask) {
          const uint32_t bits = mask[c >> 5] >> (c & 31);
#pragma unroll
          for (int e = 0; e < V; ++e) y[e] = (bits >> e) & 1u ? y[e] : kNegInf;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) m = fmaxf(m, y[e]);
      }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (j >= lay.left) break;
      if (lay.left_label(j) < lay.W) {
        const int c = lay.left_label(j);
        float v = clean(x[F + j]);
        if (H) v = seen(v, count[c]);
        if (bias) v = clean(v + bias[c]);
        if (mask && !((mask[c >> 5] >> (c & 31)) & 1u)) v = kNegInf;
        x[F + j] = v;
        m = fmaxf(m, v);
      }
    }

    float total = 0.0f;
    if (PHASE == kStats || (PHASE == kWhole && p.normalize)) {
      m = tm.max(m);
      float s = 0.0f;
      if (m > kNegInf) {
        lay.each([&](int e, int) { s += exp2_((x[e] - m) * kLog2e); });
        s = tm.sum(s);
        total = m + logf(s);
      }
      if (PHASE == kStats) {
        if (tid == 0) parts[row * plan.spans + span] = {m, s};
        continue;
      }
    }
    if (PHASE == kFinish) {
      const Part all = join_parts(parts + row * plan.spans, plan.spans);
      if (all.m > kNegInf) total = all.m + logf(all.s);
    }
    float* out = p.out + row * p.in.W + c0;
#pragma unroll
    for (int i = 0; i < L::kVecs; ++i)
      if (i < lay.vecs) {
        float y[V];
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = x[i * V + e] - total;
        store_floats<V>(out + lay.vec_label(i), y);
      }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (j >= lay.left) break;
      if (lay.left_label(j) < lay.W) out[lay.left_label(j)] = x[F + j] - total;
    }
  }
}

template <typename T, int N, int F>
static hipError_t run_process(const ProcessParams& p, const ProcessPlan& q, Part* parts, hipStream_t stream) {
  const size_t lds = p.H ? sizeof(uint32_t) * ((std::min(q.span, p.in.W) + 3) / 4 * 4) : 0;
  const dim3 grid(static_cast<uint32_t>(p.in.B) * q.groups, q.spans);
  if constexpr (N > 64) {
    if (q.spans > 1 && p.normalize) {
      process_kernel<T, N, F, kStats><<<grid, kThreads, lds, stream>>>(p, q, parts);
      process_kernel<T, N, F, kFinish><<<grid, kThreads, lds, stream>>>(p, q, parts);
      return hipGetLastError();
    }
  }
  process_kernel<T, N, F, kWhole><<<grid, kThreads, lds, stream>>>(p, q, nullptr);
  return hipGetLastError();
}

template <typename T>
static hipError_t choose_process(const ProcessParams& p, const ProcessPlan& q, int n, int f, Part* parts, hipStream_t stream) {
  if (n == 64) return f == 16 ? run_process<T, 64, 16>(p, q, parts, stream) : run_process<T, 64, 32>(p, q, parts, stream);
  if (f == 8) return run_process<T, 256, 8>(p, q, parts, stream);
  if (f == 16) return run_process<T, 256, 16>(p, q, parts, stream);
  return run_process<T, 256, 32>(p, q, parts, stream);
}

template <typename T>
static hipError_t launch_process_impl(const ProcessParams& p, void* workspace, hipStream_t stream) {
  int n, f;
  const ProcessPlan q = plan_process(p.in.B, p.in.T, p.in.W, p.H, p.normalize != 0, &n, &f);
  return choose_process<T>(p, q, n, f, static_cast<Part*>(workspace), stream);
}

}  // namespace rows
}  // namespace ctcbeam

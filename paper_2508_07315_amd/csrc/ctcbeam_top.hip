// The k largest logits of every row, and the log-sum of the others.
//
// A row is read once and stays in registers as it was read.  The k-th largest
// of the threads' own maxima bounds the k-th largest label from below (each
// of the k threads above it holds at least one label above it), and few
// labels lie above that bound: they go to LDS, where each counts the larger
// ones, which is its place in the list.  The labels below the bound are summed
// in the same pass that finds the others.  Where more labels than LDS has
// room for lie above the bound (rows of equal values), the k-th label is found
// exactly, bit by bit.
//
// What bounds it is reading the row.  A wave takes rows of fewer than 2304
// labels (lists of up to 32), a workgroup longer ones; rows beyond a workgroup
// are cut into spans whose lists and sums a second launch joins.
#include <algorithm>

#include "ctcbeam_rows_lane.h"

namespace ctcbeam {
namespace rows {

struct TopPlan {
  int n, f;   // threads of a row (of a span), labels of a thread
  int spans;  // per row
  int span;   // labels of a span (the last one may hold fewer)
};

// what a span leaves for the second launch: k keys, descending (0: none), and
// the sum over the labels that are not among them
__device__ __forceinline__ uint64_t* span_keys(void* ws, int64_t row, int spans, int span, int k) {
  return static_cast<uint64_t*>(ws) + (row * spans + span) * (k + 1);
}

__device__ __forceinline__ uint32_t order32(float v) { return static_cast<uint32_t>(detail::order_key(v, 0) >> 32); }
__device__ __forceinline__ float from_order32(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u);
}
__device__ __forceinline__ float key_value(uint64_t key) { return from_order32(static_cast<uint32_t>(key >> 32)); }
__device__ __forceinline__ int key_label(uint64_t key) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(key)); }

constexpr uint32_t kOrderNegInf = 0x007FFFFFu;  // order32(-inf)
constexpr float kTooSmall = 0x1p-80f;           // a sum that its reference may have pushed below fp32

// Places above the largest bound of 16 leading bits that at least k of n keys
// reach; 4 keys a lane (of all zeros where there is none).
template <int PER>
__device__ __forceinline__ uint32_t bound_of(const uint32_t* keys, int k) {
  uint32_t bound = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t t = bound | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += __popcll(__ballot(keys[i] >= t));
    if (n >= k) bound = t;
  }
  return bound;
}

template <typename T, int N, int F, bool PART>
__global__ void __launch_bounds__(N > kThreads ? N : kThreads) top_kernel(const TopParams p, const TopPlan plan, void* ws) {
  using L = Layout<T, N, F>;
  constexpr int kTeams = N > kThreads ? 1 : kThreads / N;
  constexpr int kMaxima = N == 64 ? 64 : 256;  // groups whose maxima give the bound
  constexpr int kRoom = 4 * N, kOwn = kRoom / N;
  __shared__ float red_all[kTeams][4][N / 64];
  __shared__ __align__(16) uint64_t room_all[kTeams][kRoom + 2];
  __shared__ uint32_t maxima[N == 64 ? 1 : kMaxima];
  __shared__ int found_lds;
  __shared__ uint64_t last_all[kTeams];
  const int tid = threadIdx.x % N, team = team_of<N>(), lane = threadIdx.x & 63;
  Team<N> tm(red_all[team]);
  uint64_t* room = room_all[team];
  const uint32_t at = blockIdx.x * kTeams + team, T_ = p.in.T;
  if (at >= p.in.B * T_) return;  // (a wave's row: no barrier is passed below)
  const int b = at / T_, t = at % T_;
  const int64_t row = at;
  if (t >= length_of(p.in, b)) {
    if (!PART) {
      for (int i = tid; i < p.k; i += N) {
        p.values[row * p.k + i] = kNegInf;
        p.ids[row * p.k + i] = -1;
      }
      if (tid == 0) p.tail[row] = kNegInf;
    }
    return;
  }
  const int span = PART ? blockIdx.y : 0, c0 = PART ? span * plan.span : 0;
  const L lay(PART ? min(p.in.W - c0, plan.span) : p.in.W, tid);
  const int k = PART ? min(p.k, lay.W) : p.k;
  RawRow<T, N, F> x(lay, static_cast<const T*>(p.in.data) + b * p.in.stride_b + t * p.in.stride_t + c0);

  // the bound
  float mx = kNegInf;
  x.each(lay, [&](float v, int) { mx = fmaxf(mx, v); });
  mx = clean(mx);
  uint32_t bound;
  if constexpr (N == 64) {
    const uint32_t key = order32(mx);
    bound = bound_of<1>(&key, k);
  } else {
    if constexpr (N > 256) {
      mx = fmaxf(mx, __uint_as_float(detail::dpp_full<detail::kDppQuadXor1>(__float_as_uint(mx))));
      if constexpr (N > 512) mx = fmaxf(mx, __uint_as_float(detail::dpp_full<detail::kDppQuadXor2>(__float_as_uint(mx))));
    }
    constexpr int per = N / kMaxima;
    if (tid % per == 0) maxima[tid / per] = order32(mx);
    if (tid == 0) found_lds = 0;
    __syncthreads();
    uint32_t keys[kMaxima / 64];
#pragma unroll
    for (int i = 0; i < kMaxima / 64; ++i) keys[i] = maxima[lane + 64 * i];
    bound = bound_of<kMaxima / 64>(keys, k);
  }
  float t0 = bound <= kOrderNegInf ? kNegInf : from_order32(bound);

  // labels from the bound on go to LDS, the others into the sum
  const float c = p.scale * kLog2e;
  float low = 0.0f;
  int n = 0;
  const auto put = [&](bool take, float v, int label) {
    if constexpr (N == 64) {
      const uint64_t who = __ballot(take);
      if (who) {
        const int at = n + __popcll(who & detail::lanemask_lt());
        if (take && at < kRoom) room[at] = detail::order_key(clean(v), c0 + label);
        n += __popcll(who);
      }
    } else if (take) {
      const int at = atomicAdd(&found_lds, 1);
      if (at < kRoom) room[at] = detail::order_key(clean(v), c0 + label);
    }
  };
  const auto found = [&]() {
    if constexpr (N > 64) {
      __syncthreads();
      n = found_lds;
    }
    return n;
  };
  x.forget();
  x.every(lay, [&](float v, int label, bool there) {
    v = fmaxf(v, kNegInf);
    const bool take = there && v >= t0;
    put(take, v, label);
    low += take || !there ? 0.0f : exp2_((v - t0) * c);
  });
  if (found() > kRoom) {
    const auto count = [&](auto which) {
      float mine = 0.0f;  // whole numbers below 2^24: exact
      x.forget();
      x.each(lay, [&](float v, int label) { mine += which(order32(clean(v)), label) ? 1.0f : 0.0f; });
      return static_cast<int>(tm.sum(mine));
    };
    uint32_t kth = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = kth | (1u << bit);
      if (count([&](uint32_t u, int) { return u >= t; }) >= k) kth = t;
    }
    const int ties = k - count([&](uint32_t u, int) { return u > kth; });
    int last = 0;  // the label of the last tie that is listed
    for (int bit = 17; bit >= 0; --bit) {
      const int t = last | (1 << bit);
      if (count([&](uint32_t u, int label) { return u == kth && label < t; }) < ties) last = t;
    }
    if constexpr (N > 64) {
      if (tid == 0) found_lds = 0;
      __syncthreads();
    }
    n = 0;
    low = 0.0f;
    t0 = from_order32(kth);
    x.forget();
    x.every(lay, [&](float v, int label, bool there) {
      v = clean(v);
      const uint32_t u = order32(v);
      const bool take = there && (u > kth || (u == kth && label <= last));
      put(take, v, label);
      low += take || !there || !(v > kNegInf) ? 0.0f : exp2_((v - t0) * c);
    });
    found();
  }

  // each label's place is the number of larger keys
  if (tid < 2) room[n + tid] = 0;
  tm.sync();
  float beside[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    beside[i] = kNegInf;
    const int at = tid + i * N;
    if (at < n) {
      const uint64_t key = room[at];
      int place = 0;
      for (int j = 0; j < n; j += 2) {
        const uint64_t a = room[j], d = room[j + 1];
        place += (a > key) + (d > key);
      }
      if (place == k - 1) last_all[team] = key;
      if (place >= k) {
        beside[i] = key_value(key);
      } else if (PART) {
        span_keys(ws, row, plan.spans, span, p.k)[place] = key;
      } else {
        p.values[row * p.k + place] = key_value(key);
        p.ids[row * p.k + place] = key_label(key);
      }
    }
  }
  tm.sync();
  const uint64_t last = last_all[team];
  float ref = key_value(last), s = 0.0f;
  if (ref > kNegInf) {
    s = low > 0.0f ? low * exp2_((t0 - ref) * c) : 0.0f;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) s += exp2_((beside[i] - ref) * c);
    s = tm.sum(s);
    if (s < kTooSmall && k < lay.W) {
      // what is left lies far below the list: relative to its own maximum
      float m = kNegInf;
      x.forget();
      x.each(lay, [&](float v, int label) {
        v = clean(v);
        if (detail::order_key(v, c0 + label) < last) m = fmaxf(m, v);
      });
      ref = tm.max(m);
      s = 0.0f;
      if (ref > kNegInf) {
        x.forget();
        x.each(lay, [&](float v, int label) {
          v = clean(v);
          if (detail::order_key(v, c0 + label) < last) s += exp2_((v - ref) * c);
        });
        s = tm.sum(s);
      }
    }
  }
  if (PART) {
    uint64_t* keys = span_keys(ws, row, plan.spans, span, p.k);
    for (int i = k + tid; i < p.k; i += N) keys[i] = 0;
    if (tid == 0) *reinterpret_cast<Part*>(keys + p.k) = {s > 0.0f ? ref : kNegInf, s};
  } else if (tid == 0) {
    p.tail[row] = s > 0.0f ? ref * p.scale + logf(s) : kNegInf;
  }
}

// The lists and sums of a row's spans, joined: a key's place is its place in
// its own list plus the larger keys of the others, which are in order.
__global__ void __launch_bounds__(kThreads) join_top_kernel(const TopParams p, const TopPlan plan, const void* ws) {
  extern __shared__ uint64_t lists[];  // [spans][k]
  __shared__ float red[4][kThreads / 64];
  const int tid = threadIdx.x, k = p.k, n = plan.spans * k;
  const int64_t row = blockIdx.x;
  const uint32_t T_ = p.in.T;
  const int b = blockIdx.x / T_, t = blockIdx.x % T_;
  if (t >= length_of(p.in, b)) {
    for (int i = tid; i < k; i += kThreads) {
      p.values[row * k + i] = kNegInf;
      p.ids[row * k + i] = -1;
    }
    if (tid == 0) p.tail[row] = kNegInf;
    return;
  }
  const uint64_t* from = static_cast<const uint64_t*>(ws) + row * plan.spans * (k + 1);
  for (int i = tid; i < n; i += kThreads) lists[i] = from[i / k * (k + 1) + i % k];
  __syncthreads();
  Team<kThreads> tm(red);
  const auto place_of = [&](int i) {
    const uint64_t key = lists[i];
    int place = i % k;
    for (int s = 0; s < plan.spans; ++s) {
      if (s == i / k) continue;
      int lo = 0, hi = k;  // the first place of list s whose key is smaller
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (lists[s * k + mid] > key) lo = mid + 1;
        else hi = mid;
      }
      place += lo;
    }
    return place;
  };
  const Part* parts = reinterpret_cast<const Part*>(from + k);
  const float c = p.scale * kLog2e;
  float m = kNegInf;
  for (int i = tid; i < n; i += kThreads) {
    const uint64_t key = lists[i];
    if (!key) continue;
    const int place = place_of(i);
    if (place < k) {
      p.values[row * k + place] = key_value(key);
      p.ids[row * k + place] = key_label(key);
    } else {
      m = fmaxf(m, key_value(key));
    }
  }
  for (int i = tid; i < plan.spans; i += kThreads) m = fmaxf(m, parts[i * (k + 1)].m);
  m = tm.max(m);
  float s = 0.0f;
  if (m > kNegInf) {
    for (int i = tid; i < n; i += kThreads)
      if (lists[i] && place_of(i) >= k) s += exp2_((key_value(lists[i]) - m) * c);
    for (int i = tid; i < plan.spans; i += kThreads) {
      const Part q = parts[i * (k + 1)];
      if (q.m > kNegInf) s += q.s * exp2_((q.m - m) * c);
    }
    s = tm.sum(s);
  }
  if (tid == 0) p.tail[row] = s > 0.0f ? m * p.scale + logf(s) : kNegInf;
}

static TopPlan plan_top(int B, int T, int W, int k) {
  const int64_t rows = static_cast<int64_t>(B) * T;
  if (W < 64 * 36 && k <= 32 && rows >= 1024) return {64, W < 64 * 20 ? 16 : 32, 1, W};
  if (W < 256 * 36) return {256, W < 256 * 12 ? 8 : W < 256 * 20 ? 16 : 32, 1, W};
  // equal spans of what a workgroup of 1024 holds
  const int most = 1024 * 36 - 1, spans = (W + most - 1) / most;
  const int span = ((W + spans - 1) / spans + 63) / 64 * 64;
  return {1024, 32, spans, std::min(span, W)};
}

template <typename T, int N, int F>
static void run_top(const TopParams& p, const TopPlan& q, void* ws, hipStream_t stream) {
  constexpr int threads = N > kThreads ? N : kThreads;
  const int64_t rows = static_cast<int64_t>(p.in.B) * p.in.T;
  if constexpr (N == 1024) {
    if (q.spans > 1) {
      top_kernel<T, N, F, true><<<dim3(static_cast<uint32_t>(rows), q.spans), threads, 0, stream>>>(p, q, ws);
      join_top_kernel<<<static_cast<uint32_t>(rows), kThreads, sizeof(uint64_t) * q.spans * p.k, stream>>>(p, q, ws);
      return;
    }
  }
  const int64_t per = threads / N;
  top_kernel<T, N, F, false><<<static_cast<uint32_t>((rows + per - 1) / per), threads, 0, stream>>>(p, q, ws);
}

template <typename T>
static hipError_t choose_top(const TopParams& p, void* ws, hipStream_t stream) {
  const TopPlan q = plan_top(p.in.B, p.in.T, p.in.W, p.k);
  if (q.n == 64) q.f == 16 ? run_top<T, 64, 16>(p, q, ws, stream) : run_top<T, 64, 32>(p, q, ws, stream);
  else if (q.n == 1024) run_top<T, 1024, 32>(p, q, ws, stream);
  else if (q.f == 8) run_top<T, 256, 8>(p, q, ws, stream);
  else if (q.f == 16) run_top<T, 256, 16>(p, q, ws, stream);
  else run_top<T, 256, 32>(p, q, ws, stream);
  return hipGetLastError();
}

}  // namespace rows

size_t top_workspace(int B, int T, int W, int k) {
  const rows::TopPlan q = rows::plan_top(B, T, W, k);
  return q.spans == 1 ? 0 : static_cast<size_t>(B) * T * q.spans * (k + 1) * sizeof(uint64_t);
}

hipError_t launch_top(const TopParams& p, void* workspace, hipStream_t stream) {
  if (p.in.type == kTypeF32) return rows::choose_top<float>(p, workspace, stream);
  if (p.in.type == kTypeF16) return rows::choose_top<rows::F16>(p, workspace, stream);
  return rows::choose_top<rows::BF16>(p, workspace, stream);
}

}  // namespace ctcbeam

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
// What bounds it: for long rows the reading and what follows it in the same
// workgroup (2048 rows of 65537 labels, k = 64: bf16 268 MB in 83 us, 3.2 TB/s, fp32
// 537 MB in 148 us, 3.6 TB/s, where a copy moves 4.96 TB/s), as a vector of which
// no wave holds a label above the bound costs a conversion, a comparison and an
// exponential a label, and those wait for the bound, so for the whole row.  For
// shorter rows the chain after the reading: 19200 rows of 1025 bf16 labels, k = 16,
// take 20 us, 2048 rows of 9300, k = 64, 22 us, twice and three times the time to
// read them, for the bound's 16 dependent steps, the places (each taken label
// against all) and the sums.  Loading the taken labels again from memory or from
// a copy of the row in LDS takes the same time.
//
// A wave takes rows of fewer than 2304 labels (lists of up to 32), a workgroup of
// 256 to 1024 threads longer ones; rows beyond a workgroup are cut into spans
// whose lists and sums a second launch joins.
#pragma once

#include "ctcbeam_rows_lane.h"
#include "ctcbeam_rows_plan.h"

namespace ctcbeam {
namespace rows {

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

// The largest bound of 16 leading bits that at least k of the keys reach, PER
// keys a lane.
template <int PER>
__device__ __forceinline__ uint32_t bound_of(const uint32_t* keys, int k) {
  uint32_t own[PER], bound = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) own[i] = keys[i * 64];
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t t = bound | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += __popcll(__ballot(own[i] >= t));
    if (n >= k) bound = t;
  }
  return bound;
}

template <int CTRL>
__device__ __forceinline__ float max_dpp(float v) {
  return fmaxf(v, __uint_as_float(detail::dpp_full<CTRL>(__float_as_uint(v))));
}
// the maximum of each `group` lanes (a power of two up to 16), in all of them
__device__ __forceinline__ float group_max(float v, int group) {
  if (group > 1) v = max_dpp<detail::kDppQuadXor1>(v);
  if (group > 2) v = max_dpp<detail::kDppQuadXor2>(v);
  if (group > 4) v = max_dpp<0x141>(v);
  if (group > 8) v = max_dpp<0x140>(v);
  return v;
}

// (four waves a SIMD for 16 vectors a thread: two workgroups of 512 a compute
// unit, 87 us against 139 for 2048 rows of 65537; at 128 registers the 16-bit forms
// spill 10 of them at 256 and 512 threads, 24 bytes a lane, and 19 to 36 at 1024, 48
// bytes; the fp32 forms none)
template <typename T, int N, int VECS, bool PART>
__global__ void __launch_bounds__(N > kThreads ? N : kThreads) __attribute__((amdgpu_waves_per_eu(VECS == 16 ? 4 : 1)))
top_kernel(const TopParams p, const TopPlan plan, void* ws) {
  using L = Layout<T, N, VECS * Packed<T>::kVec>;
  constexpr int V = L::kVec, kTeams = N > kThreads ? 1 : kThreads / N;
  constexpr int kRoom = N == 64 ? 256 : 1024;
  static_assert(N > 64 || (VECS + 1) * V <= 64, "a lane's labels as bits");
  __shared__ float red_all[kTeams][4][N / 64];
  __shared__ __align__(16) uint64_t room_all[kTeams][kRoom + 2];
  __shared__ float beside[N == 64 ? 1 : kRoom];  // exponentials of the labels behind the list, by place
  __shared__ uint32_t maxima[N == 64 ? 1 : 256];
  __shared__ int found_lds;
  __shared__ uint32_t bound_lds;
  __shared__ uint64_t last_all[kTeams];
  const int tid = threadIdx.x % N, team = team_of<N>(), lane = threadIdx.x & 63;
  Team<N> tm(red_all[team]);
  uint64_t* room = room_all[team];
  const uint32_t at_row = blockIdx.x * kTeams + team, T_ = p.in.T;
  if (at_row >= p.in.B * T_) return;  // (a wave's row: no barrier is passed below)
  const int b = at_row / T_, t = at_row % T_;
  const int64_t row = at_row;
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
  const T* in = static_cast<const T*>(p.in.data) + b * p.in.stride_b + t * p.in.stride_t + c0;
  RawRow<T, N, VECS * V> x(lay, in);

  // the bound (a maximum that a signalling NaN has spoilt only makes it lower)
  const float mx = clean(x.largest(lay));
  uint32_t bound;
  if constexpr (N == 64) {
    const uint32_t key = order32(mx);
    bound = bound_of<1>(&key, k);
  } else {
    // twice as many groups as places in the list, or 256; those of short rows
    // are single threads, so that k of them have a label
    const int groups = lay.vecs == 0 || k > 64 ? 256 : k > 32 ? 128 : 64, per = N / groups;
    const float g = group_max(mx, per);
    if (tid % per == 0) maxima[tid / per] = order32(g);
    if (tid == 0) found_lds = 0;
    __syncthreads();
    if (tid < 64) {
      const uint32_t* keys = maxima + lane;
      bound = groups == 64 ? bound_of<1>(keys, k) : groups == 128 ? bound_of<2>(keys, k) : bound_of<4>(keys, k);
      if (tid == 0) bound_lds = bound;
    }
    __syncthreads();
    bound = bound_lds;
  }
  float t0 = bound <= kOrderNegInf ? kNegInf : from_order32(bound);

  // labels from the bound on go to LDS, the others into the sum
  const float c = p.scale * kLog2e;
  float low = 0.0f;
  int n = 0;
  const auto put = [&](float v, int label) {
    const int at = atomicAdd(&found_lds, 1);
    if (at < kRoom) room[at] = detail::order_key(clean(v), c0 + label);
  };
  const auto found = [&]() {
    if constexpr (N > 64) {
      __syncthreads();
      n = found_lds;
    }
  };
  {
    const float shift = t0 * c;  // (one rounding, the same for all: within that of the result)
    x.forget();
    if constexpr (N == 64) {
      // a lane's taken labels as bits; places by a sum over the lanes before
      uint64_t taken = 0;
#pragma unroll
      for (int i = 0; i < VECS; ++i)
        if (i < lay.vecs) {
          x.forget(i);
          float v[V];
          unpack(x.raw[i], v, T());
          uint32_t m = 0;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const bool take = v[e] >= t0;
            m |= take ? 1u << e : 0u;
            low += exp2_(take ? kNegInf : __builtin_fmaf(v[e], c, -shift));
          }
          taken |= static_cast<uint64_t>(m) << (i * V);
        }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (j >= lay.left) break;
        const float v = lay.left_label(j) < lay.W ? to_float(x.one[j]) : __builtin_nanf("");
        const bool take = v >= t0;
        taken |= take ? 1ull << (VECS * V + j) : 0ull;
        if (lay.left_label(j) < lay.W) low += exp2_(take ? kNegInf : __builtin_fmaf(v, c, -shift));
      }
      const int mine = __popcll(taken);
      int at = detail::wave_incl_scan(mine, lane);
      n = __builtin_amdgcn_readlane(at, 63);
      at -= mine;
      if (n <= kRoom) {
        while (taken) {
          const int bit = __ffsll(static_cast<unsigned long long>(taken)) - 1;
          const int label = bit < VECS * V ? lay.vec_label(bit / V) + bit % V : lay.left_label(bit - VECS * V);
          room[at++] = detail::order_key(clean(to_float(in[label])), label);
          taken &= taken - 1;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < VECS; ++i)
        if (i < lay.vecs) {
          x.forget(i);
          float v[V];
          unpack(x.raw[i], v, T());
          bool any = false;
#pragma unroll
          for (int e = 0; e < V; ++e) any |= v[e] >= t0;
          if (__ballot(any)) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              if (v[e] >= t0) put(v[e], lay.vec_label(i) + e);
              else low += exp2_(__builtin_fmaf(v[e], c, -shift));
            }
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) low += exp2_(__builtin_fmaf(v[e], c, -shift));
          }
        }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (j >= lay.left) break;
        if (lay.left_label(j) < lay.W) {
          const float v = to_float(x.one[j]);
          if (v >= t0) put(v, lay.left_label(j));
          else low += exp2_(__builtin_fmaf(v, c, -shift));
        }
      }
      found();
    }
  }
  // More labels than there is room for, or (where threads have none, or NaN)
  // no bound, or fewer than k above it: the k-th is found exactly.
  if (n > kRoom || n < k || t0 == kNegInf) {
    const auto count = [&](auto which) {
      float mine = 0.0f;  // whole numbers below 2^24: exact
      x.forget();
      x.each(lay, [&](float v, int label) { mine += which(order32(clean(v)), label) ? 1.0f : 0.0f; });
      return static_cast<int>(tm.sum(mine));
    };
    uint32_t kth = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t u = kth | (1u << bit);
      if (count([&](uint32_t o, int) { return o >= u; }) >= k) kth = u;
    }
    const int ties = k - count([&](uint32_t o, int) { return o > kth; });
    int last = 0;  // the label of the last tie that is listed
    for (int bit = 17; bit >= 0; --bit) {
      const int l = last | (1 << bit);
      if (count([&](uint32_t o, int label) { return o == kth && label < l; }) < ties) last = l;
    }
    tm.sync();
    if (tid == 0) found_lds = 0;
    tm.sync();
    low = 0.0f;
    t0 = from_order32(kth);
    x.forget();
    int at = 0;  // (a wave's places: counted by all lanes alike)
    x.every(lay, [&](float v, int label, bool there) {
      v = clean(v);
      const uint32_t o = order32(v);
      const bool take = there && (o > kth || (o == kth && label <= last));
      if constexpr (N == 64) {
        const uint64_t who = __ballot(take);
        if (take) room[at + __popcll(who & detail::lanemask_lt())] = detail::order_key(v, label);
        at += __popcll(who);
      } else {
        if (take) put(v, label);
      }
      low += take || !there || !(v > kNegInf) ? 0.0f : exp2_((v - t0) * c);
    });
    n = k;
    found();
  }

  // each label's place is the number of larger keys; those behind the list
  // belong to the sum
  if (tid < 2) room[n + tid] = 0;
  tm.sync();
#pragma unroll 1
  for (int at = tid; at < n; at += N) {
    const uint64_t key = room[at];
    int place = 0;
    for (int j = 0; j < n; j += 2) {
      const uint64_t a = room[j], d = room[j + 1];
      place += (a > key) + (d > key);
    }
    if (place == k - 1) last_all[team] = key;
    if (place >= k) {
      // (the places in `room` of a workgroup's labels depend on its waves' order,
      // those in the list do not: the sum is to be the same every time)
      const float e = exp2_((key_value(key) - t0) * c);
      if constexpr (N == 64) low += e;
      else beside[place] = e;
    } else if (PART) {
      span_keys(ws, row, plan.spans, span, p.k)[place] = key;
    } else {
      p.values[row * p.k + place] = key_value(key);
      p.ids[row * p.k + place] = key_label(key);
    }
  }
  if constexpr (N > 64) {
    __syncthreads();
    for (int at = k + tid; at < n; at += N) low += beside[at];
  }
  float ref = t0, s = tm.sum(low);
  if (!(s >= kTooSmall && s < kLargest) && k < lay.W) {
    // what is left lies far from the bound, or there is NaN among it: relative to its own maximum
    tm.sync();
    const uint64_t last = last_all[team];
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
  const bool some = k < lay.W && s > 0.0f;
  if (PART) {
    uint64_t* keys = span_keys(ws, row, plan.spans, span, p.k);
    for (int i = k + tid; i < p.k; i += N) keys[i] = 0;
    if (tid == 0) *reinterpret_cast<Part*>(keys + p.k) = {some ? ref : kNegInf, some ? s : 0.0f};
  } else if (tid == 0) {
    p.tail[row] = some ? ref * p.scale + logf(s) : kNegInf;
  }
}

// The lists and sums of a row's spans, joined: a key's place is its place in
// its own list plus the larger keys of the others, which are in order.
static __global__ void __launch_bounds__(kThreads) join_top_kernel(const TopParams p, const TopPlan plan, const void* ws) {
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

template <typename T, int N, int VECS>
static void run_top(const TopParams& p, const TopPlan& q, void* ws, hipStream_t stream) {
  constexpr int threads = N > kThreads ? N : kThreads;
  const uint32_t rows = static_cast<uint32_t>(p.in.B) * p.in.T;
  if constexpr (N == 1024 && VECS == 16) {
    if (q.spans > 1) {
      top_kernel<T, N, VECS, true><<<dim3(rows, q.spans), threads, 0, stream>>>(p, q, ws);
      join_top_kernel<<<rows, kThreads, sizeof(uint64_t) * q.spans * p.k, stream>>>(p, q, ws);
      return;
    }
  }
  constexpr uint32_t per = threads / N;
  top_kernel<T, N, VECS, false><<<(rows + per - 1) / per, threads, 0, stream>>>(p, q, ws);
}

template <typename T>
static hipError_t launch_top_impl(const TopParams& p, void* ws, hipStream_t stream) {
  constexpr int V = Packed<T>::kVec;
  const TopPlan q = plan_top(p.in.type, p.in.B, p.in.T, p.in.W, p.k);
  if (q.n == 64) q.vecs == 16 / V ? run_top<T, 64, 16 / V>(p, q, ws, stream) : run_top<T, 64, 32 / V>(p, q, ws, stream);
  else if (q.n == 512) run_top<T, 512, 16>(p, q, ws, stream);
  else if (q.n == 1024) {
    if (q.vecs == 4) run_top<T, 1024, 4>(p, q, ws, stream);
    else if (q.vecs == 8) run_top<T, 1024, 8>(p, q, ws, stream);
    else run_top<T, 1024, 16>(p, q, ws, stream);
  } else {
    if (q.vecs == 1) run_top<T, 256, 1>(p, q, ws, stream);
    else if (q.vecs == 2) run_top<T, 256, 2>(p, q, ws, stream);
    else if (q.vecs == 4) run_top<T, 256, 4>(p, q, ws, stream);
    else if (q.vecs == 8) run_top<T, 256, 8>(p, q, ws, stream);
    else run_top<T, 256, 16>(p, q, ws, stream);
  }
  return hipGetLastError();
}

}  // namespace rows
}  // namespace ctcbeam

// C entry points of the operators on rows of scores: argument checks and the
// launches.  Every check comes before the first HIP call, so that a refused
// call needs no device.
#include <cmath>
#include <exception>
#include <initializer_list>
#include <limits>

#include "../../include/ctcbeam.h"
#include "ctcbeam_internal.h"
#include "ctcbeam_rows.h"
#include "ctcbeam_rows_plan.h"

static_assert(CTCBEAM_TYPE_F32 == ctcbeam::kTypeF32 && CTCBEAM_TYPE_F16 == ctcbeam::kTypeF16 &&
                  CTCBEAM_TYPE_BF16 == ctcbeam::kTypeBF16,
              "type codes");
static_assert(CTCBEAM_MAX_LABELS == ctcbeam::kMaxLabels, "label limit");
static_assert(CTCBEAM_MAX_TOP == ctcbeam::kMaxTop, "list limit");

namespace {

using Wide = __int128;

// fails with a message; nothing may be thrown through a C entry point
int refuse(int code, const char* msg) noexcept {
  try {
    return ctcbeam::set_last_error(code, msg);
  } catch (...) {
    return code;
  }
}

int launched(hipError_t e) noexcept {
  return e == hipSuccess ? 0 : refuse(e == hipErrorOutOfMemory ? 3 : 4, hipGetErrorString(e));
}

// the bytes [lo, hi) that an argument covers
struct Span {
  Wide lo = 0, hi = 0;
};

Span span(const void* p, Wide elements, int size) {
  Span s;
  if (p && elements > 0) {
    s.lo = static_cast<Wide>(reinterpret_cast<uintptr_t>(p));
    s.hi = s.lo + elements * size;
  }
  return s;
}

Wide extent(int64_t B, int64_t T, int64_t W, int64_t sb, int64_t st) {
  return static_cast<Wide>(B - 1) * sb + static_cast<Wide>(T - 1) * st + W;
}

bool meet(const Span& a, const Span& b) { return a.lo < b.hi && b.lo < a.hi; }

template <typename Spans>
bool meet_any(const Span& a, const Spans& others) {
  for (const Span& o : others)
    if (meet(a, o)) return true;
  return false;
}
bool meet_any(const Span& a, std::initializer_list<Span> others) {
  return meet_any<std::initializer_list<Span>>(a, others);
}

int element_size(int type) { return type == CTCBEAM_TYPE_F32 ? 4 : 2; }

bool misaligned(const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }

constexpr Wide kMaxExtent = static_cast<Wide>(1) << 60;

// 0, or the code of a refusal; *empty: no row at all
int check_rows(const ctcbeam_rows* r, bool* empty) {
  *empty = false;
  if (!r) return refuse(1, "null rows");
  if (r->type != CTCBEAM_TYPE_F32 && r->type != CTCBEAM_TYPE_F16 && r->type != CTCBEAM_TYPE_BF16)
    return refuse(1, "unknown element type");
  if (r->B < 0 || r->T < 0) return refuse(1, "B and T must be >= 0");
  if (r->W < 1) return refuse(1, "W must be >= 1");
  if (r->W > CTCBEAM_MAX_LABELS) return refuse(2, "W above CTCBEAM_MAX_LABELS");
  if (static_cast<Wide>(r->B) * r->T > CTCBEAM_MAX_ROWS) return refuse(2, "more than CTCBEAM_MAX_ROWS rows");
  if (r->stride_b < 0 || r->stride_t < 0) return refuse(1, "strides must be >= 0");
  if (r->B == 0 || r->T == 0) {
    *empty = true;
    return 0;
  }
  if (!r->data) return refuse(1, "null device pointer");
  if (misaligned(r->data, element_size(r->type))) return refuse(1, "rows are not aligned to their type");
  if (misaligned(r->lengths, 4)) return refuse(1, "lengths are not aligned to their type");
  if (extent(r->B, r->T, r->W, r->stride_b, r->stride_t) > kMaxExtent) return refuse(2, "strides too large");
  return 0;
}

// (the kernels' exponents are (x - max) * (scale * log2 e): 0 where x is the maximum)
bool usable(float temperature, float scale) {
  return temperature > 0.0f && std::isfinite(temperature) && scale > 0.0f && std::isfinite(scale * 1.4426950408889634f);
}

ctcbeam::RowsView view(const ctcbeam_rows* r) {
  return {r->data, r->lengths, r->stride_b, r->stride_t, r->type, r->B, r->T, r->W};
}

Span rows_span(const ctcbeam_rows* r) {
  return span(r->data, extent(r->B, r->T, r->W, r->stride_b, r->stride_t), element_size(r->type));
}

bool sizes_fit(int B, int T, int W) {
  return B > 0 && T > 0 && W > 0 && W <= CTCBEAM_MAX_LABELS && static_cast<Wide>(B) * T <= CTCBEAM_MAX_ROWS;
}

template <typename F>
F* by_type(int type, F* f32, F* f16, F* bf16) {
  return type == CTCBEAM_TYPE_F32 ? f32 : type == CTCBEAM_TYPE_F16 ? f16 : bf16;
}

int device_there() {
  int dev = -1;
  return hipGetDevice(&dev) == hipSuccess ? 0 : refuse(4, "no HIP device");
}

}  // namespace

extern "C" {

// (for either width of the scores, as the caller does not say it)
size_t ctcbeam_process_workspace_bytes(int B, int T, int W) {
  if (!sizes_fit(B, T, W)) return 0;
  int n, f;
  const ctcbeam::rows::ProcessPlan q = ctcbeam::rows::plan_process(B, T, W, 0, true, &n, &f);
  return q.spans == 1 ? 0 : static_cast<size_t>(B) * T * q.spans * sizeof(ctcbeam::Part);
}

size_t ctcbeam_top_workspace_bytes(int B, int T, int W, int k) {
  if (!sizes_fit(B, T, W) || k < 1 || k > CTCBEAM_MAX_TOP) return 0;
  size_t most = 0;
  for (int type : {CTCBEAM_TYPE_F32, CTCBEAM_TYPE_BF16}) {
    const int spans = ctcbeam::rows::plan_top(type, B, T, W, k).spans;
    if (spans > 1) most = std::max(most, static_cast<size_t>(B) * T * spans * (k + 1) * sizeof(uint64_t));
  }
  return most;
}

size_t ctcbeam_distill_workspace_bytes(int B, int T, int W) {
  if (!sizes_fit(B, T, W)) return 0;
  size_t most = 0;
  for (int type : {CTCBEAM_TYPE_F32, CTCBEAM_TYPE_BF16}) {
    const int spans = ctcbeam::rows::plan_distill(type, B, T, W).spans;
    if (spans > 1) most = std::max(most, static_cast<size_t>(B) * T * spans * sizeof(ctcbeam::SpanSums));
  }
  return most;
}

int ctcbeam_process_logits(const ctcbeam_rows* logits, const ctcbeam_process_opts* opts, float* out, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  static const ctcbeam_process_opts kNone = {nullptr, 0, 0, nullptr, nullptr, 1.0f, 0.0f, 0.0f, nullptr, 0, nullptr, 0, 0, 1, {0, 0, 0}};
  bool empty;
  if (int rc = check_rows(logits, &empty)) return rc;
  const ctcbeam_process_opts& o = opts ? *opts : kNone;
  if (o.history_size < 0) return refuse(1, "history_size must be >= 0");
  if (o.history_size > (1 << 30)) return refuse(2, "history_size above 2^30");
  if (o.history_stride < 0 || o.bias_stride < 0 || o.mask_stride_b < 0 || o.mask_stride_t < 0)
    return refuse(1, "strides must be >= 0");
  if (!o.penalties) {
    if (!(o.repetition > 0.0f) || !std::isfinite(o.repetition)) return refuse(1, "repetition must be positive and finite");
    if (!std::isfinite(o.presence) || !std::isfinite(o.frequency))
      return refuse(1, "presence and frequency must be finite");
  }
  if (empty) return 0;
  if (o.history_size > 0 && !o.history) return refuse(1, "null history");
  if (!out) return refuse(1, "null output pointer");
  if (misaligned(out, 4) || misaligned(o.history, 4) || misaligned(o.history_lengths, 4) || misaligned(o.penalties, 4) ||
      misaligned(o.bias, 4) || misaligned(o.mask, 4))
    return refuse(1, "an argument is not aligned to its type");
  const int B = logits->B, T = logits->T, W = logits->W, words = (W + 31) / 32;
  const bool with_history = o.history_size > 0;
  const Wide h = with_history ? extent(B, 1, o.history_size, o.history_stride, 0) : 0;
  const Wide bi = o.bias ? extent(B, 1, W, o.bias_stride, 0) : 0;
  const Wide ma = o.mask ? extent(B, T, words, o.mask_stride_b, o.mask_stride_t) : 0;
  if (h > kMaxExtent || bi > kMaxExtent || ma > kMaxExtent) return refuse(2, "strides too large");
  const Span so = span(out, static_cast<Wide>(B) * T * W, 4), si = rows_span(logits);
  const bool in_place = logits->data == out && logits->type == CTCBEAM_TYPE_F32 &&
                        (T == 1 || logits->stride_t == W) && (B == 1 || logits->stride_b == static_cast<int64_t>(T) * W);
  if (meet(so, si) && !in_place) return refuse(1, "out overlaps the logits (and is not the same contiguous fp32 rows)");
  const Span inputs[] = {span(logits->lengths, B, 4),   span(with_history ? o.history : nullptr, h, 4),
                         span(o.history_lengths, B, 4), span(o.penalties, 3 * static_cast<Wide>(B), 4),
                         span(o.bias, bi, 4),           span(o.mask, ma, 4)};
  if (meet_any(so, inputs)) return refuse(1, "out overlaps an input");
  if (workspace_bytes < ctcbeam_process_workspace_bytes(B, T, W) ||
      (!workspace && ctcbeam_process_workspace_bytes(B, T, W) > 0))
    return refuse(1, "workspace too small");
  if (misaligned(workspace, 16)) return refuse(1, "workspace is not aligned to 16 bytes");
  const Span sw = span(workspace, static_cast<Wide>(workspace_bytes), 1);
  if (meet_any(sw, {so, si}) || meet_any(sw, inputs)) return refuse(1, "workspace overlaps another argument");
  if (int rc = device_there()) return rc;
  ctcbeam::ProcessParams p{};
  p.in = view(logits);
  if (with_history) {
    p.history = o.history;
    p.history_lengths = o.history_lengths;
    p.history_stride = o.history_stride;
    p.H = o.history_size;
  }
  p.penalties = o.penalties;
  p.repetition = o.repetition;
  p.presence = o.presence;
  p.frequency = o.frequency;
  p.bias = o.bias;
  p.bias_stride = o.bias_stride;
  p.mask = o.mask;
  p.mask_stride_b = o.mask_stride_b;
  p.mask_stride_t = o.mask_stride_t;
  p.normalize = o.normalize != 0;
  p.out = out;
  return launched(by_type(p.in.type, ctcbeam::launch_process_f32, ctcbeam::launch_process_f16, ctcbeam::launch_process_bf16)(p, workspace, stream));
}

int ctcbeam_top_logits(const ctcbeam_rows* logits, int k, float temperature, float* values, int32_t* ids, float* tail,
                       void* workspace, size_t workspace_bytes, hipStream_t stream) {
  bool empty;
  if (int rc = check_rows(logits, &empty)) return rc;
  if (k < 1) return refuse(1, "k must be >= 1");
  if (k > CTCBEAM_MAX_TOP) return refuse(2, "k above CTCBEAM_MAX_TOP");
  if (k > logits->W) return refuse(1, "k above W");
  const float scale = 1.0f / temperature;
  if (!usable(temperature, scale)) return refuse(1, "temperature must be positive and finite, and so must log2(e)/temperature");
  if (empty) return 0;
  if (!values || !ids || !tail) return refuse(1, "null output pointer");
  if (misaligned(values, 4) || misaligned(ids, 4) || misaligned(tail, 4))
    return refuse(1, "an argument is not aligned to its type");
  const int B = logits->B, T = logits->T, W = logits->W;
  const Wide n = static_cast<Wide>(B) * T;
  const Span sv = span(values, n * k, 4), si = span(ids, n * k, 4), st = span(tail, n, 4);
  const Span sx = rows_span(logits), sl = span(logits->lengths, B, 4);
  if (meet_any(sv, {si, st, sx, sl}) || meet_any(si, {st, sx, sl}) || meet_any(st, {sx, sl}))
    return refuse(1, "an output overlaps another argument");
  if (workspace_bytes < ctcbeam_top_workspace_bytes(B, T, W, k) ||
      (!workspace && ctcbeam_top_workspace_bytes(B, T, W, k) > 0))
    return refuse(1, "workspace too small");
  if (misaligned(workspace, 16)) return refuse(1, "workspace is not aligned to 16 bytes");
  if (meet_any(span(workspace, static_cast<Wide>(workspace_bytes), 1), {sv, si, st, sx, sl}))
    return refuse(1, "workspace overlaps another argument");
  if (int rc = device_there()) return rc;
  ctcbeam::TopParams p{};
  p.in = view(logits);
  p.k = k;
  p.scale = scale;
  p.values = values;
  p.ids = ids;
  p.tail = tail;
  return launched(by_type(p.in.type, ctcbeam::launch_top_f32, ctcbeam::launch_top_f16, ctcbeam::launch_top_bf16)(p, workspace, stream));
}

int ctcbeam_distill(const ctcbeam_rows* student, const float* top_values, const int32_t* top_ids, const float* tail, int k,
                    float temperature, const float* weights, int64_t weight_stride_b, int64_t weight_stride_t,
                    float weight, float* loss, void* grad, int64_t grad_stride_b, int64_t grad_stride_t, void* workspace,
                    size_t workspace_bytes, hipStream_t stream) {
  bool empty;
  if (int rc = check_rows(student, &empty)) return rc;
  if (k < 1) return refuse(1, "k must be >= 1");
  if (k > CTCBEAM_MAX_TOP) return refuse(2, "k above CTCBEAM_MAX_TOP");
  const float scale = 1.0f / temperature;
  if (!usable(temperature, scale)) return refuse(1, "temperature must be positive and finite, and so must log2(e)/temperature");
  if (!weights && !std::isfinite(weight)) return refuse(1, "weight must be finite");
  if (weight_stride_b < 0 || weight_stride_t < 0 || grad_stride_b < 0 || grad_stride_t < 0)
    return refuse(1, "strides must be >= 0");
  if (empty) return 0;
  if (!top_values || !top_ids) return refuse(1, "null device pointer");
  if (!loss && !grad) return refuse(1, "neither loss nor grad is asked for");
  const int B = student->B, T = student->T, W = student->W, es = element_size(student->type);
  if (misaligned(top_values, 4) || misaligned(top_ids, 4) || misaligned(tail, 4) || misaligned(weights, 4) ||
      misaligned(loss, 4) || misaligned(grad, es))
    return refuse(1, "an argument is not aligned to its type");
  const Wide n = static_cast<Wide>(B) * T;
  const Wide we = weights ? extent(B, T, 1, weight_stride_b, weight_stride_t) : 0;
  const Wide ge = grad ? extent(B, T, W, grad_stride_b, grad_stride_t) : 0;
  if (we > kMaxExtent || ge > kMaxExtent) return refuse(2, "strides too large");
  if (grad) {
    // rows of the gradient may lie in either order, but not on each other
    const Wide sb = grad_stride_b, st = grad_stride_t;
    const bool apart = (T == 1 || st >= W) && (B == 1 || sb >= W) &&
                       (T == 1 || B == 1 || sb >= st * (T - 1) + W || st >= sb * (B - 1) + W);
    if (!apart) return refuse(1, "rows of grad overlap each other");
  }
  const Span sl = span(loss, n, 4), sg = span(grad, ge, es);
  const Span sx = rows_span(student), sn = span(student->lengths, B, 4), sv = span(top_values, n * k, 4),
             si = span(top_ids, n * k, 4), st = span(tail, n, 4), sw = span(weights, we, 4);
  if (meet_any(sl, {sg, sx, sn, sv, si, st, sw}) || meet_any(sg, {sx, sn, sv, si, st, sw}))
    return refuse(1, "an output overlaps another argument");
  if (workspace_bytes < ctcbeam_distill_workspace_bytes(B, T, W) ||
      (!workspace && ctcbeam_distill_workspace_bytes(B, T, W) > 0))
    return refuse(1, "workspace too small");
  if (misaligned(workspace, 16)) return refuse(1, "workspace is not aligned to 16 bytes");
  if (meet_any(span(workspace, static_cast<Wide>(workspace_bytes), 1), {sl, sg, sx, sn, sv, si, st, sw}))
    return refuse(1, "workspace overlaps another argument");
  if (int rc = device_there()) return rc;
  ctcbeam::DistillParams p{};
  p.in = view(student);
  p.k = k;
  p.scale = scale;
  p.values = top_values;
  p.ids = top_ids;
  p.tail = tail;
  p.weights = weights;
  p.weight_stride_b = weight_stride_b;
  p.weight_stride_t = weight_stride_t;
  p.weight = weight;
  p.loss = loss;
  p.grad = grad;
  p.grad_stride_b = grad_stride_b;
  p.grad_stride_t = grad_stride_t;
  return launched(by_type(p.in.type, ctcbeam::launch_distill_f32, ctcbeam::launch_distill_f16, ctcbeam::launch_distill_bf16)(p, workspace, stream));
}

}  // extern "C"

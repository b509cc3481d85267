// Operators on rows of scores (one row per frame): parameter blocks shared by
// the host entry points and the gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ctcbeam {

constexpr int kTypeF32 = 0, kTypeF16 = 1, kTypeBF16 = 2;
constexpr int kMaxLabels = 1 << 18;  // labels of a row
constexpr int kMaxTop = 128;         // listed labels of a row

// [B, T, W] scores; labels are adjacent, strides count elements.
struct RowsView {
  const void* data;
  const int32_t* lengths;  // [B] or null: all T frames
  int64_t stride_b, stride_t;
  int type, B, T, W;
};

struct ProcessParams {
  RowsView in;
  const int32_t* history;  // [B, H], rows history_stride apart; null: none
  const int32_t* history_lengths;
  int64_t history_stride;
  int H;
  const float* penalties;  // [B, 3] or null: the three scalars
  float repetition, presence, frequency;
  const float* bias;  // rows bias_stride apart (0: shared); null: none
  int64_t bias_stride;
  const uint32_t* mask;  // null: all labels allowed
  int64_t mask_stride_b, mask_stride_t;
  int normalize;
  float* out;  // [B, T, W]
};

struct TopParams {
  RowsView in;
  int k;
  float scale;  // 1 / temperature
  float* values;
  int32_t* ids;
  float* tail;
};

struct DistillParams {
  RowsView in;  // the student
  int k;
  float scale;  // 1 / temperature
  const float* values;
  const int32_t* ids;
  const float* tail;     // [B, T] or null: -inf
  const float* weights;  // rows of the gradient; null: the scalar
  int64_t weight_stride_b, weight_stride_t;
  float weight;
  float* loss;  // [B, T] or null
  void* grad;   // of the student's type, or null
  int64_t grad_stride_b, grad_stride_t;
};

// By element type, in units of their own (`workspace`: what the plans need).
#define CTCBEAM_ROW_LAUNCHES(type)                                                            \
  hipError_t launch_process_##type(const ProcessParams& p, void* workspace, hipStream_t s);   \
  hipError_t launch_top_##type(const TopParams& p, void* workspace, hipStream_t s);           \
  hipError_t launch_distill_##type(const DistillParams& p, void* workspace, hipStream_t s);
CTCBEAM_ROW_LAUNCHES(f32)
CTCBEAM_ROW_LAUNCHES(f16)
CTCBEAM_ROW_LAUNCHES(bf16)
#undef CTCBEAM_ROW_LAUNCHES

// What the parts of a row leave in a workspace: a maximum and a sum of
// exp2((x - max) * log2 e) ...
struct Part {
  float m, s;
};
// ... or, of a span of a student's row, the sum over its listed labels relative
// to m, the others' R relative to r, the listed labels' part of the loss but
// for log S, and their probability.
struct SpanSums {
  float m, listed_sum, r, R, terms, listed;
};

}  // namespace ctcbeam

// How the row operators cut their work: which kernel takes a call, how many
// threads a row gets, and whether rows are cut into spans.  Host code, shared by
// the launches and the workspace sizes.
//
// A kernel of N threads and `vecs` vectors of 16 bytes a thread holds rows of
// fewer than N * (vecs + 1) * (labels of a vector) labels.
#pragma once

#include <algorithm>

#include "ctcbeam_rows.h"

namespace ctcbeam {
namespace rows {

constexpr int kThreads = 256;  // per workgroup, but for the rows of more threads

struct ProcessPlan {
  int spans;   // per row
  int span;    // labels of a span (the last one may hold fewer)
  int frames;  // per workgroup
  int groups;  // of frames, per utterance
};

// Labels from which on a wave, and a workgroup of 256, do not hold a row of any
// type in registers as fp32.
constexpr int kRowOfWave = 64 * 36, kRowOfGroup = 256 * 36;

inline ProcessPlan plan_process(int B, int T, int W, int H, bool normalize, int* n, int* f) {
  const int64_t rows = static_cast<int64_t>(B) * T;
  ProcessPlan q{1, W, 1, T};
  if (W < kRowOfWave && rows >= 1024) {
    // a wave a row, also where an utterance has fewer frames than a workgroup
    // waves, whose others then leave at once: 4096 requests, T = 1, bf16, us by waves
    // / by workgroups: 33 labels 6.0 / 9.1, 1025 8.6 / 13.4, 2000 12.8 / 16.0, 2303
    // 14.6 / 13.1; fp32 33 labels 6.1 / 8.5, 1025 9.2 / 10.5, 2303 15.8 / 13.3.
    // 512 requests of 1025: 3.8 / 4.3, fp32 4.0 / 3.9
    *n = 64;
    *f = W < 64 * 20 ? 16 : 32;
    q.frames = 4;
  } else if (W < kRowOfGroup && (normalize || rows >= 512)) {
    // by a workgroup a row / by spans, fp32 (bf16 within 0.5 us): 256 rows of 9200
    // normalised 7.9 / 11.5, 1024 rows 15.1 / 26.9; not normalised, of one launch
    // either way, 1 row 4.3 / 2.8, 256 rows 7.0 / 6.8, 1024 rows 14.3 / 16.1, and of
    // 2400 labels 3.4 / 3.3 (256 rows), 3.9 / 5.1 (512 rows)
    *n = 256;
    *f = W < 256 * 12 ? 8 : W < 256 * 20 ? 16 : 32;
  } else {
    // spans: as long as the card stays full of them
    int span = 8192;
    while (span > 2048 && rows * ((W + span - 1) / span) < 512) span >>= 1;
    *n = 256;
    *f = span / 256;
    q.spans = (W + span - 1) / span;
    q.span = span;
  }
  // A workgroup's counts serve several frames where the history is longer than
  // a row and there are workgroups enough (else one frame a wave keeps more
  // rows in flight: B=64 T=400 W=1025 takes 45 us, with three frames 50).
  const int64_t groups = rows * q.spans / q.frames;
  const int more = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({16, groups / 2048, H / W})));
  q.frames = std::min(q.frames * more, T);
  q.groups = (T + q.frames - 1) / q.frames;
  return q;
}

struct TopPlan {
  int n, vecs;  // threads of a row (of a span), vectors of 16 bytes of a thread
  int spans;    // per row
  int span;     // labels of a span (the last one may hold fewer)
};

// A wave for each of many short rows; 256 threads for short rows; for longer
// ones the fewest threads that hold the row where there are rows for every
// compute unit, else 1024.
// By a wave / by 256 threads, k = 32, us, bf16: 33 labels, 512 rows 3.8 / 4.9, 1024 rows
// 3.9 / 5.4, 25600 rows 16 / 56; 1025 labels 5.0 / 5.9, 5.1 / 6.6, 26 / 78; 2303 labels
// 5.8 / 5.8, 6.0 / 6.6, 39 / 81; fp32, 2303 labels 6.0 / 5.9, 6.4 / 6.9, 53 / 70.
// By the fewest / by 1024 threads, us, bf16: 1 row of 32768 labels, k = 64, 13.6 / 7.6; 512
// rows 18.7 / 18.2, 1024 rows 25.8 / 34.1, 2048 rows 41 / 63; 2048 rows of 65536 72 / 100.
// 512 rows of 34700: k = 16 16.5 / 16.4, k = 128 25.0 / 24.4; 1024 rows 22 / 29, 33 / 45.
// fp32 crosses later: 17300 labels, k = 16, 512 rows 13.5 / 11.4, 1024 rows 18.5 / 17.7, 2048
// rows 31 / 32 (k = 128 20.6 / 16.5, 27.6 / 26.9, 47 / 49); 34700 labels 18.2 / 21.4, 33 / 43,
// 55 / 80.
inline TopPlan plan_top(int type, int B, int T, int W, int k) {
  const int64_t rows = static_cast<int64_t>(B) * T;
  const int vec = type == kTypeF32 ? 4 : 8;
  // threads and their vectors, by what they hold: N * (vecs + 1) * vec - 1 labels
  const auto holds = [&](int n, int vecs) { return W < n * (vecs + 1) * vec; };
  if (k <= 32 && rows >= 1024 && W < 64 * 36) return {64, holds(64, 16 / vec) ? 16 / vec : 32 / vec, 1, W};
  if (holds(256, 4)) return {256, holds(256, 1) ? 1 : holds(256, 2) ? 2 : 4, 1, W};
  if (rows >= 512) {
    if (holds(256, 16)) return {256, holds(256, 8) ? 8 : 16, 1, W};
    if (holds(512, 16)) return {512, 16, 1, W};
  }
  if (holds(1024, 16)) return {1024, holds(1024, 4) ? 4 : holds(1024, 8) ? 8 : 16, 1, W};
  // equal spans, in whole words of 64 labels, of what a workgroup of 1024 holds
  const int most = 1024 * 17 * vec - 64, spans = (W + most - 1) / most;
  return {1024, 16, spans, ((W + spans - 1) / spans + 63) / 64 * 64};
}

struct DistillPlan {
  int n, f;   // threads of a row (of a span), labels of a thread
  int spans;  // per row; 0: a workgroup holds the row in packed registers
  int span;   // labels of a span (the last one may hold fewer)
};

// A long row keeps the workgroup that holds it busy while few rows leave the
// card idle; spans use all of it, but read the row twice in two launches.  bf16,
// k = 64, loss and gradient, us by a workgroup of 1024 a row / by spans:
//   labels       1 row       128 rows    192 rows    256 rows
//   18400        7.9 / 9.8   8.9 / 12.5  9.5 / 13.8  9.9 / 14.3
//   32768        9.9 / 7.9  12.3 / 12.0 13.3 / 14.7 14.6 / 17.5
//   65536       15.7 / 7.7  19.3 / 16.4 20.2 / 21.1 23.3 / 27.2
//   131072      27.0 / 7.7  33.3 / 26.7 36.3 / 39.3 39.7 / 47.6
// k = 128 lies on the same sides (65536 labels, 128 rows 20.3 / 18.4, 160 rows 20.9 /
// 20.1, 192 rows 22.0 / 22.2).  fp32 rows of as many labels are twice the bytes, and
// spans pay for fewer of them, k = 16:
//   24600        7.7 / 8.3  11.1 / 15.0 12.6 / 17.6 13.9 / 18.9
//   32768        8.3 / 8.1  12.0 / 16.0 13.7 / 20.0 16.4 / 21.5
//   65536       12.7 / 8.0  18.7 / 21.5 25.8 / 36.5 30.8 / 51.5
constexpr int64_t kFewRows = 160;
constexpr int kLongRow = 24576;
// Rows from which on smaller workgroups, several of a compute unit, take rows of
// fewer than 512 * 17 vectors, us by them / by 1024 threads: 18400 labels, 512 rows
// 17.7 / 18.9, 2048 rows 40 / 64; 65536 labels, 512 rows 38 / 43,
// 2048 rows 131 / 171.  fp32, k = 16: 9300 labels, 256 rows 10.1 / 8.6, 512 rows 13.1 /
// 15.4, 2048 rows 40 / 58; 34700 labels 17.9 / 17.0, 32 / 39, 119 / 126; k = 128
// 20.3 / 18.7, 35 / 42, 130 / 143.
constexpr int64_t kManyRows = 512;

inline DistillPlan plan_distill(int type, int B, int T, int W) {
  const int64_t rows = static_cast<int64_t>(B) * T;
  // by a wave / by 256 threads, k = 16, us, bf16: 33 labels, 512 rows 4.2 / 4.8, 1024
  // rows 4.3 / 5.4; 1025 labels 4.8 / 5.8, 4.9 / 6.9, 25600 rows 31 / 77; 2303 labels 6.3 /
  // 5.3, 6.6 / 6.5, 53 / 77; fp32, 1025 labels 5.0 / 5.1, 5.3 / 6.0, 47 / 71; 2303
  // 6.9 / 5.5, 8.5 / 7.8, 97 / 90
  if (W < 64 * 36 && rows >= 1024) return {64, W < 64 * 20 ? 16 : 32, 1, W};
  if (W < 256 * 36) return {256, W < 256 * 12 ? 8 : W < 256 * 20 ? 16 : 32, 1, W};
  const int vec = type == kTypeF32 ? 4 : 8;
  const auto holds = [&](int n, int vecs) { return W < n * (vecs + 1) * vec; };
  if ((rows >= kFewRows || W < kLongRow) && holds(1024, 16)) {
    if (rows >= kManyRows && holds(512, 16)) return {holds(256, 16) ? 256 : 512, (holds(256, 8) ? 8 : 16) * vec, 0, W};
    return {1024, (holds(1024, 4) ? 4 : holds(1024, 8) ? 8 : 16) * vec, 0, W};
  }
  int span = 8192;
  while (span > 2048 && rows * ((W + span - 1) / span) < 512) span >>= 1;
  return {256, span / 256, (W + span - 1) / span, span};
}

}  // namespace rows
}  // namespace ctcbeam

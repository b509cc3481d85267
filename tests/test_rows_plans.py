"""How the operators on rows of scores cut their work, on the CPU: the plans
compiled for the host, over types, numbers of rows and all row lengths around
each line of the rules.  Whatever a plan picks must be compiled, hold the row (or
cover it with spans that it holds), and fit the launch limits."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIP = "/opt/rocm/include"

PROGRAM = r"""
#include "ctcbeam_rows_plan.h"
#include <cstdio>
#include <set>
using namespace ctcbeam;
using namespace ctcbeam::rows;
static long bad = 0, calls = 0;
static void check(bool ok, const char* op, int type, int B, int T, int W, int k) {
  ++calls;
  if (!ok && bad++ < 10) std::printf("%s type=%d B=%d T=%d W=%d k=%d\n", op, type, B, T, W, k);
}
static bool covers(int spans, int span, int W) {
  return spans > 1 && spans <= 65535 && span % 32 == 0 && long(spans) * span >= W && long(spans - 1) * span < W;
}
int main() {
  std::set<int> ws;
  for (int w = 1; w <= 300; ++w) ws.insert(w);
  for (int n : {64, 256, 512, 1024})
    for (int v : {4, 8})
      for (int q : {1, 2, 3, 4, 5, 8, 9, 16, 17})
        for (int d = -9; d <= 9; ++d) ws.insert(n * v * q + d);
  for (int w : {2048, 2303, 2304, 8192, 9215, 9216, 24575, 24576, 65536, 100001, 131072, 200000, 262143, 262144})
    for (int d = -2; d <= 2; ++d) ws.insert(w + d);
  const int bt[][2] = {{1, 1}, {1, 3}, {1, 4}, {2, 64}, {159, 1}, {160, 1}, {511, 1}, {512, 1}, {1, 1023}, {1024, 1}, {256, 4}, {64, 400}, {1, 2097152}, {2097152, 1}};
  for (int W : ws) {
    if (W < 1 || W > kMaxLabels) continue;
    for (auto& x : bt)
      for (int type : {kTypeF32, kTypeF16, kTypeBF16}) {
        const int B = x[0], T = x[1], vec = type == kTypeF32 ? 4 : 8;
        const long rows = long(B) * T;
        for (int H : {0, 1, 1000, 1 << 20})
          for (bool normalize : {false, true}) {
            int n, f, n0, f0;
            const ProcessPlan q = plan_process(B, T, W, H, normalize, &n, &f);
            bool ok = (n == 64 && (f == 16 || f == 32)) || (n == 256 && (f == 8 || f == 16 || f == 32));
            ok = ok && (q.spans == 1 ? W < n * (f + vec) && q.span >= W : n == 256 && covers(q.spans, q.span, W) && q.span <= n * f);
            ok = ok && q.frames >= 1 && long(q.groups) * q.frames >= T && long(q.groups - 1) * q.frames < T;
            ok = ok && long(B) * q.groups * kThreads < (1l << 32) && 4l * std::min(q.span, W) <= 60000;
            // the workspace, sized without a history, holds what a normalised call leaves
            ok = ok && (!normalize || plan_process(B, T, W, 0, true, &n0, &f0).spans == q.spans);
            check(ok, "process", type, B, T, W, 0);
          }
        for (int k : {1, 32, 33, 64, 65, 128}) {
          if (k > W) continue;
          const TopPlan q = plan_top(type, B, T, W, k);
          bool ok = q.n == 64 ? (q.vecs == 16 / vec || q.vecs == 32 / vec) && k <= 32
                  : q.n == 256 ? q.vecs == 1 || q.vecs == 2 || q.vecs == 4 || q.vecs == 8 || q.vecs == 16
                  : q.n == 512 ? q.vecs == 16 : q.n == 1024 && (q.vecs == 4 || q.vecs == 8 || q.vecs == 16);
          ok = ok && (q.spans == 1 ? W < q.n * (q.vecs + 1) * vec
                                   : q.n == 1024 && q.vecs == 16 && covers(q.spans, q.span, W) && q.span < 1024 * 17 * vec && q.spans * k * 8 <= 60000);
          ok = ok && rows * std::max(q.n, kThreads) < (1l << 32);
          check(ok, "top", type, B, T, W, k);
        }
        const DistillPlan q = plan_distill(type, B, T, W);
        const int vecs = q.f / vec;
        bool ok;
        if (q.spans == 0) {
          ok = q.n == 256 ? vecs == 8 || vecs == 16 : q.n == 512 ? vecs == 16 : q.n == 1024 && (vecs == 4 || vecs == 8 || vecs == 16);
          ok = ok && W < q.n * (vecs + 1) * vec;
        } else {
          ok = q.n == 64 ? q.f == 16 || q.f == 32 : q.n == 256 && (q.f == 8 || q.f == 16 || q.f == 32);
          ok = ok && (q.spans == 1 ? W < q.n * (q.f + vec) : q.n == 256 && covers(q.spans, q.span, W) && q.span <= q.n * q.f);
          ok = ok && (kThreads / q.n) * ((std::min(q.span, W) * (16l / vec) + 15) / 16 * 16) <= 60000;
        }
        ok = ok && rows * std::max(q.n, kThreads) < (1l << 32);
        check(ok, "distill", type, B, T, W, 0);
      }
  }
  std::printf("calls %ld bad %ld\n", calls, bad);
  return bad != 0;
}
"""


def test_every_plan_holds_its_rows(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists(os.path.join(HIP, "hip", "hip_runtime.h")):
        pytest.skip("needs g++ and the HIP headers")
    src, exe = tmp_path / "plans.cpp", tmp_path / "plans"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{HIP}",
                    f"-I{os.path.join(ROOT, 'paper_2508_07315_amd', 'csrc')}", str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout

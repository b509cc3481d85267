"""Which compiled kernel a call of the operators on rows of scores runs, from
the library's own plans, compiled for the host."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIP = "/opt/rocm/include"
TYPES = {"fp32": 0, "fp16": 1, "bf16": 2}

# Calls as lines "op type B T W k H normalize" (what an operator does not have
# is 0), each answered by a line of the kernels it launches
# (and of whether a workgroup's count of the history serves frame after frame); "all" answers with
# the kernels of all sizes.
PROGRAM = r"""
#include "ctcbeam_rows_plan.h"
#include <cstdio>
#include <cstring>
#include <set>
#include <string>
using namespace ctcbeam;
using namespace ctcbeam::rows;
static const char* kNames[] = {"float", "F16", "BF16"};
static std::string form(const char* kernel, int type, int a, int b, const char* last) {
  return std::string(kernel) + "<" + kNames[type] + ", " + std::to_string(a) + ", " + std::to_string(b) + last + ">;";
}
static std::string of(const std::string& op, int type, int B, int T, int W, int k, int H, bool normalize) {
  const int vec = type == kTypeF32 ? 4 : 8;
  if (op == "process") {
    int n, f;
    const ProcessPlan q = plan_process(B, T, W, H, normalize, &n, &f);
    const std::string shared = q.frames > kThreads / n ? "counts for several frames, " + std::to_string(n) + (q.spans > 1 ? ", spans;" : ";") : "";
    if (q.spans > 1 && normalize) return shared + form("process_kernel", type, n, f, ", 1") + form("process_kernel", type, n, f, ", 2");
    return shared + form("process_kernel", type, n, f, ", 0");
  }
  if (op == "top") {
    const TopPlan q = plan_top(type, B, T, W, k);
    return q.spans > 1 ? form("top_kernel", type, q.n, q.vecs, ", true") + "join_top_kernel;" : form("top_kernel", type, q.n, q.vecs, ", false");
  }
  const DistillPlan q = plan_distill(type, B, T, W);
  if (q.spans == 0) return form("distill_wide_kernel", type, q.n, q.f / vec, "");
  if (q.spans > 1) return form("distill_kernel", type, q.n, q.f, ", 1") + form("distill_kernel", type, q.n, q.f, ", 2");
  return form("distill_kernel", type, q.n, q.f, ", 0");
}
int main(int argc, char** argv) {
  char op[16];
  int type, B, T, W, k, H, normalize;
  if (argc > 1 && !std::strcmp(argv[1], "all")) {
    std::set<std::string> found;
    for (int rows : {1, 2, 100, 159, 160, 511, 512, 1023, 1024, 4096})
      for (int W = 1; W <= kMaxLabels; W += W < 2500 ? 1 : 61)
        for (int type = 0; type < 3; ++type) {
          for (int normalize = 0; normalize < 2; ++normalize) found.insert(of("process", type, rows, 1, W, 0, 0, normalize));
          for (int k : {1, 32, 33, 64, 65, 128})
            if (k <= W) found.insert(of("top", type, rows, 1, W, k, 0, false));
          found.insert(of("distill", type, rows, 1, W, 1, 0, false));
        }
    for (const std::string& s : found) std::printf("%s\n", s.c_str());
    return 0;
  }
  while (std::scanf("%15s %d %d %d %d %d %d %d", op, &type, &B, &T, &W, &k, &H, &normalize) == 8)
    std::printf("%s\n", of(op, type, B, T, W, k, H, normalize).c_str());
}
"""


class Forms:
    def __init__(self, folder):
        cxx = shutil.which("g++")
        if cxx is None or not os.path.exists(os.path.join(HIP, "hip", "hip_runtime.h")):
            pytest.skip("needs g++ and the HIP headers")
        src, self.exe = folder / "forms.cpp", str(folder / "forms")
        src.write_text(PROGRAM)
        subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{HIP}",
                        f"-I{os.path.join(ROOT, 'paper_2508_07315_amd', 'csrc')}", str(src), "-o", self.exe], check=True)

    def all(self):
        """The kernels that calls of some size launch."""
        r = subprocess.run([self.exe, "all"], capture_output=True, text=True, check=True)
        return {f for line in r.stdout.split("\n") for f in line.split(";") if f}

    def of(self, calls):
        """The kernels of each of (op, kind, B, T, W, k, H, normalize)."""
        text = "".join(f"{op} {TYPES[kind]} {B} {T} {W} {k} {H} {int(normalize)}\n" for op, kind, B, T, W, k, H, normalize in calls)
        r = subprocess.run([self.exe], input=text, capture_output=True, text=True, check=True)
        found = [[f for f in line.split(";") if f] for line in r.stdout.splitlines()]
        assert len(found) == len(calls)
        return found

"""The launch plan of the attention calls (csrc/attend.hpp, plain C++), compiled and run here:
its shapes are ones the kernels take, and the workspace sized without a window holds the plan of
any window."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_09916_amd", "csrc")

SOURCE = r"""
#include <stdio.h>
#include <vector>
#include "attend.hpp"
using namespace ikv;
static int bad = 0;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s (L %d Hq %d Hkv %d B %d n %d N %d fmt %d f32 %d window %d)\n", __LINE__, #x, a.L, a.Hq, a.Hkv, B, n, N, a.format, a.io_f32, w); ++bad; } } while (0)
int main() {
  const int Ls[] = {1, 2, 36, 80}, heads[][2] = {{1, 1}, {8, 2}, {32, 8}, {40, 8}, {20, 4}, {7, 1}, {9, 3}, {48, 6}, {128, 64}};
  const int Bs[] = {0, 1, 2, 5, 16, 64}, ns[] = {0, 1, 2, 5, 17, 64, 100, 509, 5000}, Ns[] = {0, 1, 63, 300, 513, 1025, 8192, 92300, 1000000};
  long runs = 0;
  for (int L : Ls) for (auto &h : heads) for (int B : Bs) for (int n : ns) for (int N : Ns) for (int fmt = 0; fmt < 3; ++fmt)
    for (int f32 = 0; f32 < (fmt ? 2 : 1); ++f32) for (int decode = 0; decode < 2; ++decode) {
      if (decode && n != 1) continue;
      AttendArgs a{};
      a.L = L, a.Hq = h[0], a.Hkv = h[1], a.D = 128, a.format = fmt, a.io_f32 = f32;
      std::vector<ikv_session> s(B ? B : 1);
      for (int b = 0; b < B; ++b) {
        s[b].N = b % 3 == 2 ? N / 3 : N;
        s[b].C = s[b].N;
        s[b].qe = s[b].N;
        s[b].qs = s[b].N > n ? s[b].N - n : 0;
      }
      int w = 0;
      const AttendPlan full = attend_plan(a, s.data(), B, decode, 0, 0);
      const int ws[] = {0, 1, 50, 1000, 4096, 2147483647};
      for (int win : ws) for (int sinks : {0, 4, 70000, 2147483647}) {
        w = win;
        const AttendPlan p = attend_plan(a, s.data(), B, decode, win ? sinks : 0, win);
        ++runs;
        CHECK(p.ws_floats <= full.ws_floats && p.ws_floats >= 0);
        CHECK(p.splits >= 1 && p.splits <= DEC_MAX_SPLITS);
        if (p.max_n == 0) continue;
        const int G = a.Hq / a.Hkv;
        if (p.few) {
          CHECK(p.rows == p.max_n * G && p.rows <= (fmt && !f32 ? 32 : 16));
          CHECK(p.heads >= 1 && a.Hkv % p.heads == 0 && p.parts >= 1 && p.heads * p.parts <= FEW_WAVES);
          const int nr = p.rows > 16 ? 2 : 1;
          CHECK((p.parts - 1) * p.heads * nr * (a.D / 4 + 2) * 64 * 4 + FEW_WAVES * 2 * 32 * 4 <= 65536);   // LDS
        } else {
          CHECK((p.rows == 128 || p.rows == 256) && p.blocks >= 1);
          CHECK((int64_t)p.blocks * p.rows >= (int64_t)p.max_n * G && (int64_t)(p.blocks - 1) * p.rows < (int64_t)p.max_n * G);
        }
        if (p.splits > 1) CHECK(p.ws_floats == (int64_t)B * L * a.Hkv * p.blocks * p.splits * p.rows * (a.D + 2));
      }
    }
  printf("%ld plans, %d bad\n", runs, bad);
  return bad != 0;
}
"""


def test_plans(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(SOURCE)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]

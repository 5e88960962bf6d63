"""Splits of the few-row attention over 4-bit rows (csrc/attend.hpp, plain C++, compiled and run here): where the counts
of workgroups fall badly on the rounds of 256 (28 layers: 224 or 448, seven eighths of their rounds), lists are not cut
as finely as they can be."""
import os
import shutil
import subprocess

import pytest

from test_attend_plan import CSRC, ROOT

SOURCE = r"""
#include <stdio.h>
#include <vector>
#include "attend.hpp"
using namespace ikv;
static AttendPlan plan(int L, int Hq, int Hkv, int B, int N) {
  AttendArgs a{};
  a.L = L, a.Hq = Hq, a.Hkv = Hkv, a.D = 128, a.format = KV_E2M1;
  std::vector<ikv_session> s(B);
  for (auto &x : s) x.N = x.C = x.qe = N, x.qs = N - 1;
  return attend_plan(a, s.data(), B, true, 0, 0);
}
int main() {
  int bad = 0;
  struct { int L, Hq, Hkv, B, N, most; } few[] = {
      {28, 28, 4, 1, 3000, 4}, {28, 28, 4, 1, 30000, 4}, {28, 28, 4, 2, 3000, 4}, {28, 28, 4, 4, 3000, 2}, {28, 28, 4, 4, 30000, 2},
      {28, 28, 4, 8, 3000, 1}, {28, 28, 4, 16, 8201, 1}, {28, 14, 2, 2, 3000, 4}, {28, 14, 2, 4, 3000, 2}, {28, 14, 2, 8, 8201, 1}};
  for (auto &x : few) {
    const AttendPlan p = plan(x.L, x.Hq, x.Hkv, x.B, x.N);
    if (!p.four || p.splits > x.most) {
      printf("L %d Hkv %d B %d N %d: %d splits\n", x.L, x.Hkv, x.B, x.N, p.splits);
      ++bad;
    }
  }
  // shapes whose counts meet the rounds well
  if (plan(36, 32, 8, 1, 8201).splits != 7 || plan(48, 40, 8, 1, 92300).splits != 5 || plan(36, 32, 8, 16, 3000).splits != 2) ++bad;
  // everywhere: not more splits than another count of them, with fewer rounds, that fills those to 85%
  for (int L = 1; L <= 96; ++L) for (int Hkv : {1, 2, 4, 5, 8, 10}) for (int B : {1, 2, 3, 4, 8, 16, 64}) for (int N : {600, 3000, 8201, 92300}) {
    const AttendPlan p = plan(L, 4 * Hkv, Hkv, B, N);
    const int64_t units = int64_t(L) * B * (p.pair ? Hkv / 2 : Hkv) / p.heads;
    for (int s = 1; s < p.splits; ++s)
      if (attend_fill(units * s) >= 85 && attend_rounds(units * s) < attend_rounds(units * p.splits)) {
        printf("L %d Hkv %d B %d N %d: %d splits, %d fill fewer rounds\n", L, Hkv, B, N, p.splits, s);
        ++bad;
        break;
      }
  }
  return bad != 0;
}
"""


def test_splits(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "rounds.cpp", tmp_path / "rounds"
    src.write_text(SOURCE)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]

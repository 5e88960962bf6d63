"""How the row kernels share a session's list out (csrc/quant_rows.hpp, plain C++), compiled and
run here: over every workgroup of a launch, the places of the rows that are listed, each once, and
none past them."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_09916_amd", "csrc")

SOURCE = r"""
#include <stdint.h>
#include <stdio.h>
#include "quant_rows.hpp"
using namespace ikv;
int main() {
  int bad = 0;
  for (int Hkv : {1, 2, 3, 8, 16, 32, 48, 64, 96, 4096, 65535}) for (int D : {64, 128})
    for (int longest : {1, 67, 8192, 1000003, QUANT_MOST}) for (int rows : {0, 1, 10, 8191, 5000000, QUANT_MOST}) {
      if (rows > longest) continue;
      const int per = Hkv * (D / 8), group = quant_group(per);
      int64_t sum = 0;
      int least = 0, most = 0;
      for (int64_t k0 = 0; k0 < longest; k0 += group) {
        const int n = quant_places(group, rows, int(k0), per);
        sum += n;
        least = std::min(least, n);
        most = std::max(most, n);
        if (k0 >= rows && n != 0) ++bad;
      }
      if (sum != int64_t(rows) * per || least < 0 || most > std::max(QT * QU, per)) {
        printf("Hkv %d D %d longest %d rows %d: %lld places of %lld, %d .. %d a workgroup\n", Hkv, D, longest, rows,
               (long long)sum, (long long)rows * per, least, most);
        ++bad;
      }
    }
  return bad != 0;
}
"""


def test_places(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "places.cpp", tmp_path / "places"
    src.write_text(SOURCE)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]

"""The grid of the row kernels (csrc/quant_rows.hpp, plain C++, compiled and run here): lists that are mostly
padding do not make it grow without end, and its workgroups, striding over a list, take each place of its rows
once."""
import shutil
import subprocess

import pytest

from test_quant_places import CSRC

SOURCE = r"""
#include <stdio.h>
#include "quant_rows.hpp"
using namespace ikv;
int main() {
  int bad = 0;
  for (int Hkv : {1, 2, 3, 8, 64, 4096}) for (int D : {64, 128}) for (int64_t units : {1, 36, 48 * 64, 36 * 4096, 65535 * 4})
    for (int most : {QUANT_GRID, QUANT_GRID_NEW}) for (int longest : {1, 67, 8201, 36000, 1000003, QUANT_MOST}) {
      const int per = Hkv * (D / 8), group = quant_group(per), grid = quant_groups(longest, group, units, most);
      const int64_t full = (int64_t(longest) + group - 1) / group;
      // as many as the list has work for, unless the launch would have more than `most`
      if (grid < 1 || (grid > 1 && grid * units > most) || grid > full || (full * units <= most && grid != full)) {
        printf("Hkv %d D %d units %lld longest %d: %d workgroups\n", Hkv, D, (long long)units, longest, grid);
        ++bad;
      }
      if (units > 36) continue;
      for (int rows : {0, 1, 66, 8201, longest}) {
        if (rows > longest) continue;
        int64_t sum = 0;
        for (int x = 0; x < grid; ++x)
          for (int k0 = x * group; k0 < rows; k0 += grid * group) {
            const int n = quant_places(group, rows, k0, per);
            if (n <= 0) ++bad;
            sum += n;
          }
        if (sum != int64_t(rows) * per) {
          printf("Hkv %d D %d longest %d rows %d: %lld places\n", Hkv, D, longest, rows, (long long)sum);
          ++bad;
        }
      }
    }
  return bad != 0;
}
"""


def test_grid(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text(SOURCE)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]

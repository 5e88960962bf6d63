"""The launch forms that tests/test_gpu_attend_wide.py names are those the plan gives (csrc/attend.hpp,
plain C++, compiled and run here); and a bound that allows weights of two bf16 parts refuses one."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from attend_wide import CASES, PARAMS
from oracle import quant_oracle as qo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_09916_amd", "csrc")

SOURCE = r"""
#include <stdio.h>
#include <vector>
#include "attend.hpp"
using namespace ikv;
// lines: L Hq Hkv D format io_f32 tokens sinks window sessions lengths...
int main() {
  AttendArgs a{};
  int f32, n, sinks, window, B;
  while (scanf("%d %d %d %d %d %d %d %d %d %d", &a.L, &a.Hq, &a.Hkv, &a.D, &a.format, &f32, &n, &sinks, &window, &B) == 10) {
    a.io_f32 = f32;
    std::vector<ikv_session> s(B);
    for (auto &x : s) {
      if (scanf("%d", &x.N) != 1) return 1;
      x.C = x.qe = x.N;
      x.qs = x.N - (n ? n : 1);
    }
    const AttendPlan p = attend_plan(a, s.data(), B, n == 0, sinks, window);
    printf("%d %d %d %d\n", p.few, p.heads, p.parts, p.splits);
  }
}
"""


def test_forms(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "forms.cpp", tmp_path / "forms"
    src.write_text(SOURCE)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    lines, want = [], []
    for name, code, io in PARAMS:
        form, L, Hq, Hkv, D, n, Ns, sinks, window, _ = CASES[name]
        lines.append(" ".join(map(str, [L, Hq, Hkv, D, ["bf16", "int8", "e4m3"].index(code), int(io == "f32"), n, sinks, window,
                                        len(Ns), *Ns])))
        want.append((name, (1, *form)))
    r = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=60, check=True)
    got = [tuple(map(int, x.split())) for x in r.stdout.splitlines()]
    assert [(name, g) for (name, _), g in zip(want, got)] == want
    assert {w[1:3] for _, w in want} >= {(4, 1), (4, 2), (2, 2), (2, 4)}


def bf16(x):
    """float64 values below 2^127 to the nearest bf16, ties to even."""
    m, e = np.frexp(np.asarray(x, np.float64))
    return np.ldexp(np.round(m * 256), e - 8)


def cancelling(N, D):
    """Query, keys and values [N, D] whose weights alternate between 1 and 0.50195 (half way between two bf16 numbers)
    and whose values cancel but for that: exact in every row format. -> (q, k, v)"""
    target = np.log(0.5 + 2.0 ** -9) * np.sqrt(D)
    q = np.zeros(D)
    q[0] = bf16(target)
    q[1] = bf16(target - q[0])
    odd = np.arange(N)[:, None] % 2
    sign = np.where(np.arange(D) % 3 == 1, -1.0, 1.0)
    return q, odd * np.ones(D), np.where(odd, 1.0, -0.5) * sign


@pytest.mark.parametrize("N,D", [(90, 64), (700, 128)])
def test_one_part_would_be_seen(N, D):
    q, k, v = cancelling(N, D)
    want, A, X = qo.attend(q[None, None], k[:, None], v[:, None])
    w = np.exp(k @ q / np.sqrt(D))
    assert np.abs(w[1::2] - (0.5 + 2.0 ** -9)).max() < 2.0 ** -14
    one = (bf16(w) @ v) / w.sum()                        # weights rounded once, their sum not
    two = (bf16(w) + bf16(w - bf16(w))) @ v / w.sum()
    E = ((D + 8) * X + 4 * (1 + X) + N + 8) * 2.0 ** -24
    tol = (2.0 ** -8 * np.abs(want) + (2.0 ** -17 + 2 * E[..., None]) * A)[0, 0]
    assert (np.abs(one - want[0, 0]) > 5 * tol).all() and (np.abs(two - want[0, 0]) < tol).all()

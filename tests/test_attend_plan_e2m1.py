"""The launch plan of the attention over 4-bit rows (csrc/attend.hpp, plain C++), compiled and run here:
its shapes are ones that the kernels take, and the workspace sized without a window holds the plan of
any window."""
import os
import shutil
import subprocess

import pytest

from test_attend_plan import CSRC, ROOT, SOURCE

WIDTHS = "for (int fmt = 0; fmt < 3; ++fmt)"


def _source():
    s = SOURCE
    for old, new in ((WIDTHS, "for (int fmt = 3; fmt < 4; ++fmt) for (int D : {64, 128})"), ("a.D = 128,", "a.D = D,"),
                     ("CHECK(p.heads >= 1 && a.Hkv % p.heads == 0 &&",
                      "CHECK(p.four == (D == 128 && !f32) && (!p.pair || p.four));\n"
                      "          if (p.four) CHECK((p.heads * p.parts == 4 || (p.heads * p.parts == 8 && p.rows <= 16)) && !(p.pair && p.rows > 16));\n"
                      "          CHECK(p.heads >= 1 && a.Hkv % (p.heads * (p.pair ? 2 : 1)) == 0 &&"),
                     ("CHECK((p.rows == 128 || p.rows == 256) && p.blocks >= 1);",
                      "CHECK((f32 ? p.rows == 128 || p.rows == 256 : p.rows == 128) && p.blocks >= 1);")):
        assert s.count(old) == 1, old
        s = s.replace(old, new)
    return s


def test_plans(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(_source())
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-4000:]

"""Pins of oracle/quant_oracle.py: hand-worked rows, ties, and closed forms."""
import math

import numpy as np
import pytest

from oracle import quant_oracle as qo


def test_e4m3_table():
    v = qo.e4m3_values()
    assert len(v) == 127 and v[0] == 0 and v[1] == 2.0 ** -9 and v[7] == 7 * 2.0 ** -9 and v[8] == 2.0 ** -6
    assert v[0x38] == 1.0 and v[0x3f] == 1.875 and v[-1] == 448.0 and np.all(np.diff(v) > 0)


def test_int8_by_hand():
    # a = 2: scale 2/127; x = 1 is 63.5, a tie: 64 is even; -1 likewise; 0.5 is 31.75; 3/127 is 1.5 at float64's rounding
    c, s = qo.quantise(np.array([2.0, 1.0, -1.0, 0.5, 3.0 / 127, 0.0]), "int8")
    assert s == np.float32(2 / 127)
    assert list(c.view(np.int8)) == [127, 64, -64, 32, 2, 0]


def test_int8_codes_by_rationals():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((40, 16)).astype(np.float32)
    x[:20] = np.round(x[:20] * 8) / 8                    # few bits: many ties
    c, _ = qo.quantise(x.astype(np.float64), "int8")
    for r in range(40):
        a = float(np.abs(x[r]).max())
        assert [qo.int8_code(float(y), a) for y in x[r]] == list(c[r].view(np.int8))


def test_e4m3_by_hand():
    # a = 448: scale 1; a = 449: scale 2 (224.5 -> 224); ties to the even code
    c, s = qo.quantise(np.array([448.0, 1.0625, 1.1875, -0.5, 2.0 ** -10, 3 * 2.0 ** -10]), "e4m3")
    assert s == 1 and list(qo.code_values(c, "e4m3")) == [448.0, 1.0, 1.25, -0.5, 0.0, 2.0 ** -8]
    c, s = qo.quantise(np.array([449.0, 1.0]), "e4m3")
    assert s == 2 and list(qo.code_values(c, "e4m3")) == [224.0, 0.5]


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_small_zero_and_non_finite_rows(code):
    c, s = qo.quantise(np.array([[0.0, 0.0], [2.0 ** -101, 0.0], [np.inf, 1.0], [np.nan, 1.0]]), code)
    assert np.isfinite(s[:2]).all() and np.isnan(s[2:]).all() and not c[0].any() and not c[2:].any()
    assert s[0] == s[1]
    # within half a step of the row's scale
    d = qo.code_values(c[:2], code) * s[:2, None].astype(float)
    assert np.abs(d - [[0, 0], [2.0 ** -101, 0]]).max() <= 2.0 ** -100 / 127 * 0.5


def test_seen_by_hand():
    assert qo.seen(5, 2, 0, 0).astype(int).tolist() == [[1, 1, 1, 1, 0], [1, 1, 1, 1, 1]]
    assert qo.seen(5, 2, 1, 2).astype(int).tolist() == [[1, 0, 1, 1, 0], [1, 0, 0, 1, 1]]
    assert qo.seen(1, 3, 1, 2).astype(int).tolist() == [[0], [0], [1]]


def test_attend_closed_forms():
    rng = np.random.default_rng(5)
    v = rng.standard_normal((6, 2, 4))
    # equal keys: a mean of the entries seen; two query heads a KV head
    out, spread, reach = qo.attend(np.ones((4, 2, 4)), np.zeros((6, 2, 4)), v, 1, 2)
    assert np.allclose(out[0, 0], v[[0, 3, 4], 0].mean(0)) and np.allclose(out[3, 1], v[[0, 4, 5], 1].mean(0))
    assert np.allclose(spread[0, 0], np.abs(v[[0, 3, 4], 0]).mean(0)) and not reach.any()
    # two entries, one logit apart by log 3
    k = np.zeros((2, 1, 4))
    k[1, 0, 0] = 2 * math.log(3)
    out, _, reach = qo.attend(np.array([[[1.0, 0, 0, 0]]]), k, v[:2, :1])
    assert np.allclose(out[0, 0], (v[0, 0] + 3 * v[1, 0]) / 4) and np.isclose(reach[0, 0], math.log(3))
    # more tokens than entries: the early ones see nothing
    out, _, _ = qo.attend(np.ones((1, 3, 4)), k, v[:2, :1])
    assert not out[0, 0].any() and np.allclose(out[0, 1], v[0, 0])

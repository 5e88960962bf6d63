"""RetentionStep's 8-bit calls refuse what they cannot do in the library's own way (no GPU needed)."""
import pytest

import synth
from paper_2606_09916_amd import ikv
from paper_2606_09916_amd.step import RetentionStep


@pytest.fixture()
def step():
    spec = synth.SessionSpec(N=60, C=20, pi=2, qs=50, qe=60, R=4, dead_frac=0.0)
    batch = synth.make_batch(synth.Shape(L=1, Hq=2, Hkv=1, D=64), [spec], seed=3, kv_dtype=synth.F32, layout="paged")
    return RetentionStep(batch, "cpu")


@pytest.mark.parametrize("code", ["int4", "", None, "INT8"])
def test_unknown_codes(step, code):
    with pytest.raises(ikv.IkvError, match="int8.*e4m3") as e:
        step.quantise(code)
    assert e.value.status == -1 and step.cache is None


def test_decode_before_there_is_a_cache(step):
    with pytest.raises(ikv.IkvError, match="quantise") as e:
        step.decode_quant()
    assert e.value.status == -1

"""Descriptors of the 8-bit cache at the far end of their fields' ranges are refused on the host,
with an error and without a trap (no GPU needed)."""
import pytest

from test_quant_args import EUNSUPPORTED, _cache, _load, _pool, _store


@pytest.mark.parametrize("call", [_store, _load])
@pytest.mark.parametrize("Hkv", [65536, 1 << 27, 1 << 28, 1 << 29, (1 << 31) - 1])
@pytest.mark.parametrize("D", [64, 128])
def test_more_heads_than_a_row_can_have(call, Hkv, D):
    assert call(_cache(Hq=Hkv, Hkv=Hkv, D=D), _pool(Hq=Hkv, Hkv=Hkv, D=D)) == EUNSUPPORTED

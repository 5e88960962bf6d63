"""Descriptors of the 8-bit cache at the far end of their fields' ranges are refused on the host,
with an error and without a trap (no GPU needed)."""
import ctypes

import pytest

from paper_2606_09916_amd import ikv
from test_quant_args import EUNSUPPORTED, _attend, _cache, _load, _pool, _sess, _store


@pytest.mark.parametrize("call", [_store, _load])
@pytest.mark.parametrize("Hkv", [65536, 1 << 27, 1 << 28, 1 << 29, (1 << 31) - 1])
@pytest.mark.parametrize("D", [64, 128])
def test_more_heads_than_a_row_can_have(call, Hkv, D):
    assert call(_cache(Hq=Hkv, Hkv=Hkv, D=D), _pool(Hq=Hkv, Hkv=Hkv, D=D)) == EUNSUPPORTED


@pytest.mark.parametrize("which", ["decode", "chunk", "chunk_quant"])
@pytest.mark.parametrize("L,Hkv,N", [(1 << 27, 1 << 30, (1 << 24) - 1), (1 << 30, 1 << 28, 300), ((1 << 31) - 1, 1 << 28, 5),
                                     (65536, 1, 8192), (1, 65536, 8192), (1, 1, (1 << 31) - 1)])
@pytest.mark.parametrize("window", [0, 4096])
def test_launches_that_no_grid_holds(which, L, Hkv, N, window):
    # the workspace call answers, and the call itself refuses
    kw = dict(L=L, Hq=Hkv, Hkv=Hkv, D=128, num_slots=(1 << 31) - 1)
    c, s = _pool(**kw) if which == "chunk" else _cache(**kw), _sess(N=N, qs=0, qe=N, C=N)
    n, lib = ctypes.c_size_t(0), ikv.lib()
    call = ikv.CALL_DECODE if which == "decode" else ikv.CALL_CHUNK
    if which == "chunk":
        assert lib.ikv_workspace_bytes(ctypes.byref(c), s, 1, call, 0, ctypes.byref(n)) == 0
    else:
        assert lib.ikv_quant_workspace_bytes(ctypes.byref(c), s, 1, call, ctypes.byref(n)) == 0
    assert _attend(which, c, s, window=window, wn=1 << 62) == EUNSUPPORTED

"""The calls of the quantised cache take a 4-bit cache and refuse bad ones on the host (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2606_09916_amd import ikv
from test_quant_args import EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE, PTR, _attend, _cache, _load, _pool, _sess, _store


def _four(**kw):
    return _cache(code=ikv.IKV_E2M1, **kw)


@pytest.mark.parametrize("field,value,code", [
    ("Hq", 7, ESHAPE), ("D", 32, EUNSUPPORTED), ("D", 96, EUNSUPPORTED), ("num_slots", 0, ESHAPE), ("dead_slot", 100, ESHAPE),
    ("io_dtype", 7, EINVAL), ("k_codes", PTR + 8, EINVAL), ("scales", PTR + 2, EINVAL), ("scales", None, EINVAL)])
def test_descriptor(field, value, code):
    c = _four(**{field: value})
    assert _store(c) == code and _load(c) == code and _attend("decode", c) == code and _attend("chunk_quant", c) == code


def test_scales_alignment():
    # one slot and head: 4 bytes at D = 64, 8 at D = 128; a layer of an odd number of slots may begin at either
    empty = _sess(N=0, qs=0, qe=0)
    assert _store(_four(scales=PTR + 4), s=empty) == 0
    assert _store(_four(D=128, scales=PTR + 4), _pool(D=128), empty) == EINVAL
    assert _store(_four(D=128, scales=PTR + 8), _pool(D=128), empty) == 0


@pytest.mark.parametrize("code", [2, 3, 5, -1])
def test_unknown_codes(code):
    assert _store(_cache(code=code)) == EINVAL and _attend("decode", _cache(code=code)) == EINVAL


def test_calls():
    assert _store(_four(), p=_pool(D=128)) == ESHAPE and _load(_four(), p=_pool(Hkv=4)) == ESHAPE
    assert _store(_four(), s=_sess(N=0, qs=0, qe=0)) == 0
    assert _attend("decode", _four(), q=None) == EINVAL and _attend("chunk_quant", _four(), window=-1) == EINVAL
    assert _attend("decode", _four(L=20000)) == EUNSUPPORTED


def test_workspace():
    n = ctypes.c_size_t(0)
    c, s = _four(L=1), _sess(N=5000, qs=4900, qe=5000, C=5000)
    assert ikv.lib().ikv_quant_workspace_bytes(ctypes.byref(c), s, 1, ikv.CALL_CHUNK, ctypes.byref(n)) == 0 and n.value > 0
    assert _attend("chunk_quant", c, s, wn=n.value - 1) == EWORKSPACE


def test_binding():
    kc, sc = torch.zeros(1, 4, 2, 32, dtype=torch.uint8), torch.zeros(1, 4, 2, 2, 2, dtype=torch.uint8)
    make = lambda k=kc, v=kc, s=sc, **kw: ikv.make_quant_pool(k, v, s, 1, 4, 2, 64, 4, **kw)  # noqa: E731
    assert make().code == ikv.IKV_E2M1 and make(io_dtype=torch.float32).io_dtype == ikv.IKV_F32
    for bad in (dict(v=kc.view(torch.int8)), dict(v=kc[:, :3].contiguous()), dict(v=kc.transpose(1, 2)), dict(s=sc.float()),
                dict(s=sc[..., :1]), dict(s=sc[:, :3].contiguous()), dict(io_dtype=torch.float16), dict(s=sc.to("meta"))):
        with pytest.raises(ikv.IkvError):
            make(**bad)
    # as many codes as bytes of an 8-bit cache are too many, and an 8-bit cache's bytes with byte scales are refused
    with pytest.raises(ikv.IkvError):
        ikv.make_quant_pool(kc.view(torch.int8), kc.view(torch.int8), sc, 1, 4, 2, 64, 4)

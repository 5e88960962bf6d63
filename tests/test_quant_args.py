"""The calls of the 8-bit cache and the chunk attention refuse bad arguments on the host,
before anything touches a device (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2606_09916_amd import ikv

EINVAL, ESHAPE, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -4
PTR = 0x10000


def _cache(**kw):
    c = ikv.QuantPool(L=2, Hq=8, Hkv=2, D=64, num_slots=100, dead_slot=0, code=ikv.IKV_INT8, io_dtype=ikv.IKV_BF16,
                      reserved=0, k_codes=PTR, v_codes=PTR, scales=PTR)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _pool(**kw):
    p = ikv.Pool(L=2, Hq=8, Hkv=2, D=64, num_slots=100, dead_slot=0, kv_dtype=ikv.IKV_BF16, k_pool=PTR, v_pool=PTR)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _sess(**kw):
    s = (ikv.Session * 1)()
    base = dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=50, pi=0, qs=40, qe=50, C=20, radix_prefix=0, R=4, nq=0)
    base.update(kw)
    for k, v in base.items():
        setattr(s[0], k, v)
    return ctypes.cast(s, ctypes.POINTER(ikv.Session))


def _store(c=None, p=None, s=None, sd=PTR, B=1, src=PTR, dst=PTR, n=PTR):
    return ikv.lib().ikv_quant_store(ctypes.byref(c or _cache()), ctypes.byref(p or _pool()), s or _sess(), sd, B, src,
                                     dst, n, None)


def _load(c=None, p=None, s=None, sd=PTR, B=1, src=PTR, dst=PTR, n=PTR):
    return ikv.lib().ikv_quant_load(ctypes.byref(c or _cache()), ctypes.byref(p or _pool()), s or _sess(), sd, B, src,
                                    dst, n, None)


def _attend(which, c=None, s=None, B=1, sd=PTR, q=PTR, live=PTR, n=PTR, sinks=0, window=0, out=PTR, ws=PTR, wn=1 << 40):
    f = {"decode": ikv.lib().ikv_decode_attend_quant, "chunk_quant": ikv.lib().ikv_attend_chunk_quant,
         "chunk": ikv.lib().ikv_attend_chunk}[which]
    c = c or (_pool() if which == "chunk" else _cache())
    return f(ctypes.byref(c), s or _sess(), sd, B, q, live, n, sinks, window, out, ws, wn, None)


def test_struct_layout():
    assert ctypes.sizeof(ikv.QuantPool) == 64
    assert ikv.QuantPool.num_slots.offset == 16 and ikv.QuantPool.k_codes.offset == 40


@pytest.mark.parametrize("field,value,code", [
    ("Hq", 7, ESHAPE), ("Hq", 18, EUNSUPPORTED), ("D", 96, EUNSUPPORTED), ("L", 0, ESHAPE), ("num_slots", 0, ESHAPE),
    ("num_slots", 1 << 31, ESHAPE), ("dead_slot", 100, ESHAPE), ("dead_slot", -1, ESHAPE), ("code", 2, EINVAL),
    ("io_dtype", 7, EINVAL), ("reserved", 1, EINVAL), ("k_codes", None, EINVAL), ("scales", None, EINVAL),
    ("v_codes", PTR + 8, EINVAL), ("scales", PTR + 4, EINVAL)])
def test_cache_descriptor(field, value, code):
    c = _cache(**{field: value})
    assert _store(c) == code and ikv.lib().ikv_last_error()
    assert _load(c) == code
    assert _attend("decode", c) == code
    assert _attend("chunk_quant", c) == code
    n = ctypes.c_size_t(7)
    assert ikv.lib().ikv_quant_workspace_bytes(ctypes.byref(c), _sess(), 1, ikv.CALL_DECODE, ctypes.byref(n)) == code
    assert n.value == 0


@pytest.mark.parametrize("call", [_store, _load])
def test_row_calls(call):
    for field, value in (("L", 3), ("Hkv", 4), ("D", 128)):
        assert call(p=_pool(**{field: value})) == ESHAPE
    assert call(p=_pool(k_pool=PTR + 4)) == EINVAL
    assert call(p=_pool(kv_dtype=9)) == EINVAL
    assert call(sd=None) == EINVAL and call(B=-1) == EINVAL
    assert call(s=_sess(N=-1)) == ESHAPE
    assert call(B=0, src=None, dst=None) == 0
    assert call(s=_sess(N=0, qs=0, qe=0)) == 0          # no rows: nothing is launched


def test_sizes_past_a_launch():
    big = _sess(N=1 << 24, qs=0, qe=1)
    assert _store(p=_pool(num_slots=1 << 25), s=big) == EUNSUPPORTED
    assert _load(p=_pool(num_slots=1 << 25), s=big) == EUNSUPPORTED
    assert _store(_cache(L=70000), _pool(L=70000)) == EUNSUPPORTED
    assert _attend("decode", _cache(L=20000)) == EUNSUPPORTED
    assert _attend("decode", s=_sess(N=(1 << 30) + 1, qs=0, qe=1)) == EUNSUPPORTED
    assert _attend("chunk", s=_sess(N=1 << 29, qs=0, qe=1 << 29)) == EUNSUPPORTED


def test_rows_of_an_identity_list_must_fit():
    assert _store(dst=None) == EINVAL and _load(src=None) == EINVAL
    assert _store(s=_sess(slot_off=60), src=None) == ESHAPE
    assert _load(s=_sess(slot_off=60), dst=None) == ESHAPE


@pytest.mark.parametrize("which", ["decode", "chunk", "chunk_quant"])
def test_attention_calls(which):
    for kw in (dict(q=None), dict(live=None), dict(n=None), dict(out=None), dict(sinks=-1), dict(window=-1),
               dict(sd=None), dict(q=PTR + 8), dict(out=PTR + 2)):
        assert _attend(which, **kw) == EINVAL, kw
    assert _attend(which, s=_sess(qe=60)) == ESHAPE
    assert _attend(which, B=0, q=None) == 0
    if which != "decode":
        assert _attend(which, s=_sess(qs=50)) == 0       # no new tokens: nothing is launched
    if which == "chunk":
        assert _attend(which, _pool(kv_dtype=ikv.IKV_F32)) == EUNSUPPORTED
        assert _attend(which, _pool(v_pool=PTR + 8)) == EINVAL


def test_workspace_call_ids():
    n = ctypes.c_size_t(0)
    f = ikv.lib().ikv_quant_workspace_bytes
    for call in (ikv.CALL_SCORE, ikv.CALL_PREFILL, 99):
        assert f(ctypes.byref(_cache()), _sess(), 1, call, ctypes.byref(n)) == EINVAL
    assert f(ctypes.byref(_cache()), _sess(), 1, ikv.CALL_CHUNK, None) == EINVAL
    assert f(ctypes.byref(_cache()), None, 0, ikv.CALL_CHUNK, ctypes.byref(n)) == 0 and n.value == 0


@pytest.mark.parametrize("which", ["decode", "chunk_quant"])
def test_workspace_too_small(which):
    n = ctypes.c_size_t(0)
    c, s = _cache(L=1), _sess(N=5000, qs=4900, qe=5000, C=5000)
    call = ikv.CALL_DECODE if which == "decode" else ikv.CALL_CHUNK
    assert ikv.lib().ikv_quant_workspace_bytes(ctypes.byref(c), s, 1, call, ctypes.byref(n)) == 0
    if n.value:
        assert _attend(which, c, s, wn=n.value - 1) == EWORKSPACE
        assert _attend(which, c, s, ws=None) == EWORKSPACE
        assert _attend(which, c, s, ws=PTR + 16) == EWORKSPACE


def test_binding_checks_tensors():
    kc = torch.zeros(1, 4, 2, 64, dtype=torch.int8)
    sc = torch.zeros(1, 4, 2, 2)
    make = lambda k=kc, v=kc, s=sc, **kw: ikv.make_quant_pool(k, v, s, 1, 4, 2, 64, 4, **kw)  # noqa: E731
    c = make()
    assert (c.code, c.io_dtype) == (ikv.IKV_INT8, ikv.IKV_BF16)
    assert make(kc.view(torch.float8_e4m3fn), kc.view(torch.float8_e4m3fn), io_dtype=torch.float32).code == ikv.IKV_E4M3
    for bad in (dict(k=kc.float()), dict(v=kc.view(torch.float8_e4m3fn)), dict(v=kc[:, :3].contiguous()),
                dict(v=kc.transpose(1, 2)), dict(s=sc.double()), dict(s=sc[..., :1]), dict(io_dtype=torch.float16)):
        with pytest.raises(ikv.IkvError):
            make(**bad)
    rows = [dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=3, pi=0, qs=1, qe=3, C=3, radix_prefix=0, R=1, nq=0)]
    sess = ikv.Sessions(rows, "cpu")
    live, n = torch.zeros(3, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    q = torch.zeros(1 * 4 * 2 * 64, dtype=torch.bfloat16)
    ws = ikv.Workspace("cpu")
    good = dict(q=q, live=live, n_live=n, out=q.clone())
    for bad in (dict(q=q.float()), dict(q=q[:-1]), dict(out=q.double()), dict(live=live.long()), dict(live=live[:2]),
                dict(n_live=n.long()), dict(q=torch.zeros(512, 2, dtype=torch.bfloat16)[:, 0])):
        a = {**good, **bad}
        with pytest.raises(ikv.IkvError):
            ikv.attend_chunk_quant(c, sess, a["q"], a["live"], a["n_live"], a["out"], ws)
    with pytest.raises(ikv.IkvError):
        ikv.quant_store(c, ikv.Pool(), sess, None, live.long())
    # well-formed, but not on a GPU
    with pytest.raises(ikv.IkvError, match="not on a GPU"):
        ikv.attend_chunk_quant(c, sess, q, live, n, q.clone(), ws)
    with pytest.raises(ikv.IkvError, match="not on a GPU"):
        ikv.quant_store(c, ikv.Pool(), sess, None, live)


@pytest.mark.parametrize("kw", [dict(sinks=1 << 31), dict(window=(1 << 32) + 5), dict(sinks=-1), dict(window=-1 << 32)])
def test_binding_checks_window(kw):
    # past 32 bits they would arrive as other numbers
    kc = torch.zeros(1, 4, 2, 64, dtype=torch.int8)
    c = ikv.make_quant_pool(kc, kc, torch.zeros(1, 4, 2, 2), 1, 4, 2, 64, 4)
    sess = ikv.Sessions([dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=3, pi=0, qs=1, qe=3, C=3,
                              radix_prefix=0, R=1, nq=0)], "cpu")
    live, n = torch.zeros(3, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    q = torch.zeros(1 * 4 * 2 * 64, dtype=torch.bfloat16)
    for f in (ikv.attend_chunk_quant, ikv.decode_attend_quant):
        with pytest.raises(ikv.IkvError, match="sinks is|window is"):
            f(c, sess, q, live, n, q.clone(), ikv.Workspace("cpu"), **kw)

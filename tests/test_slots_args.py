"""ikv_return_slots and ikv_take_slots refuse bad arguments on the host, before anything touches a
device (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2606_09916_amd import ikv
from test_quant_args import EINVAL, ESHAPE, EUNSUPPORTED, PTR, _sess


def _free(**kw):
    f = ikv.FreeSlots(num_slots=100, dead_slot=0, reserved=0, slots=PTR, count=PTR)
    for k, v in kw.items():
        setattr(f, k, v)
    return f


def _give(f=None, s=None, sd=PTR, B=1, lists=PTR, n=PTR):
    return ikv.lib().ikv_return_slots(ctypes.byref(f or _free()), s or _sess(), sd, B, lists, n, None)


def _take(f=None, s=None, sd=PTR, B=1, n_new=PTR, slot_maps=PTR, live=PTR, n_live=PTR, n_all=PTR, dst=PTR, n_taken=PTR):
    return ikv.lib().ikv_take_slots(ctypes.byref(f or _free()), s or _sess(), sd, B, n_new, slot_maps, live, n_live, n_all,
                                    dst, n_taken, None)


def test_struct_layout():
    assert ctypes.sizeof(ikv.FreeSlots) == 32 and ikv.FreeSlots.slots.offset == 16 and ikv.FreeSlots.count.offset == 24


@pytest.mark.parametrize("field,value,code", [
    ("num_slots", 0, ESHAPE), ("num_slots", 1 << 31, ESHAPE), ("dead_slot", -1, ESHAPE), ("dead_slot", 100, ESHAPE),
    ("reserved", 1, EINVAL), ("slots", None, EINVAL), ("count", None, EINVAL)])
def test_stack(field, value, code):
    assert _give(_free(**{field: value})) == code and ikv.lib().ikv_last_error()
    assert _take(_free(**{field: value})) == code


def test_arguments():
    assert ikv.lib().ikv_return_slots(None, _sess(), PTR, 1, PTR, PTR, None) == EINVAL
    for kw in (dict(lists=None), dict(n=None), dict(sd=None), dict(B=-1)):
        assert _give(**kw) == EINVAL, kw
    for kw in (dict(n_taken=None), dict(live=None), dict(n_live=None), dict(n_all=None), dict(live=None, n_live=None),
               dict(sd=None), dict(B=-1)):
        assert _take(**kw) == EINVAL, kw
    assert _give(s=_sess(qe=60)) == ESHAPE and _take(s=_sess(N=-1)) == ESHAPE
    assert _give(B=0, lists=None) == 0 and _take(B=0, n_taken=None) == 0


def test_sums_past_the_limit():
    s = (ikv.Session * 2)()
    for x, n in zip(s, (1 << 30, 1)):
        x.N, x.qe, x.R = n, n, 1
    p = ctypes.cast(s, ctypes.POINTER(ikv.Session))
    assert _give(s=p, B=2) == EUNSUPPORTED and _take(s=p, B=2) == EUNSUPPORTED
    s[0].N = s[0].qe = (1 << 31) - 1
    assert _give(s=p) == EUNSUPPORTED and _take(s=p) == EUNSUPPORTED


def test_binding():
    slots, count = torch.zeros(10, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    f = ikv.make_free_slots(slots, count, 10)
    for bad in (lambda: ikv.make_free_slots(slots.long(), count, 10), lambda: ikv.make_free_slots(slots, count, 11),
                lambda: ikv.make_free_slots(slots, count[:1], 10), lambda: ikv.make_free_slots(slots, count.to("meta"), 10),
                lambda: ikv.make_free_slots(torch.zeros(20, dtype=torch.int32)[::2], count, 10)):
        with pytest.raises(ikv.IkvError):
            bad()
    sess = ikv.Sessions([dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=3, pi=0, qs=1, qe=3, C=3, radix_prefix=0,
                              R=1, nq=0)], "cpu")
    three, one = torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for bad in (dict(slot_maps=three.long()), dict(live=three[:2]), dict(dst=three.float()), dict(n_live=one.long()),
                dict(n_all=one[:0]), dict(n_new=one.long()), dict(n_taken=one.long())):
        with pytest.raises(ikv.IkvError):
            ikv.take_slots(f, sess, **{**dict(n_taken=one, slot_maps=three, live=three, n_live=one, n_all=one, dst=three), **bad})
    with pytest.raises(ikv.IkvError):
        ikv.return_slots(f, sess, three[:2], one)
    with pytest.raises(ikv.IkvError, match="not on a GPU"):
        ikv.return_slots(f, sess, three, one)
    with pytest.raises(ikv.IkvError, match="not on a GPU"):
        ikv.take_slots(f, sess, one, dst=three)
    f.device = torch.device("meta")
    with pytest.raises(ikv.IkvError, match="on different devices"):
        ikv.take_slots(f, sess, one, dst=three)

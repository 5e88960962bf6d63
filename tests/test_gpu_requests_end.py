"""Requests over a shared prefix end: their own slots go back to the stack, the prefix's do not, and no later token
gets one of those."""
import numpy as np
import pytest

import oracle
from paper_2606_09916_amd import ikv
from test_gpu_slots import Stack, ints

pytestmark = pytest.mark.gpu

PREFIX = 40


def _requests(dev, Ns, spans):
    """Sessions whose first PREFIX positions share their slots; the second aliases slots of its own and of the prefix."""
    import torch
    num_slots = PREFIX + sum(Ns) + 20
    order = 1 + np.random.default_rng(7).permutation(num_slots - 1).astype(np.int32)
    maps, rows, at, off = [], [], PREFIX, 0
    for N, n in zip(Ns, spans):
        m = np.concatenate([order[:PREFIX], order[at:at + N - PREFIX]])
        maps.append(m)
        rows.append(dict(slot_off=off, mem_off=0, qspan_off=0, qpos_off=0, N=N, pi=PREFIX, qs=N - n, qe=N, C=N,
                         radix_prefix=PREFIX, R=1, nq=0))
        at, off = at + N - PREFIX, off + N
    maps[1][70], maps[1][90], maps[1][80] = maps[1][71], maps[1][100], maps[1][5]
    return num_slots, order[:PREFIX], maps, ikv.Sessions(rows, dev), torch.from_numpy(np.concatenate(maps)).to(dev)


def _end(sess, num_slots, S, dev):
    import torch
    total, B = len(S), sess.B
    keep = torch.zeros(total, dtype=torch.uint8, device=dev)
    for x in sess.host[:B]:
        keep[x.slot_off:x.slot_off + PREFIX] = 1
    freed, live = (torch.zeros(total, dtype=torch.int32, device=dev) for _ in range(2))
    n_freed, n_live = ints([0] * B, dev), ints([0] * B, dev)
    ikv.redirect_slots(sess, num_slots, S, 0, keep, freed, n_freed, live, n_live, ikv.Workspace(dev))
    return freed, n_freed, n_live


def test_the_prefix_stays(dev):
    import torch
    Ns, spans = [150, 260], [30, 60]
    num_slots, prefix, maps, sess, S = _requests(dev, Ns, spans)
    freed, n_freed, n_live = _end(sess, num_slots, S, dev)
    assert n_live.tolist() == [PREFIX] * 2 and int((S != 0).sum()) == 2 * PREFIX
    stack = Stack([], num_slots, dev)
    ikv.return_slots(stack.free, sess, freed, n_freed)
    want = [u for m in maps for u in oracle.redirect(m, np.arange(len(m)) < PREFIX, 0, PREFIX)[1].tolist()]
    got = stack()
    assert got == want and len(set(got)) == len(got)
    assert sorted(got) == sorted(set(np.concatenate([m[PREFIX:] for m in maps]).tolist()) - set(prefix.tolist()))
    assert not set(prefix.tolist()) & set(got)
    # all that is free goes to new tokens: none of them gets a slot of the prefix
    one = ikv.Sessions([dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=len(got), pi=0, qs=0, qe=len(got), C=len(got),
                             radix_prefix=0, R=1, nq=0)], dev)
    dst, taken = torch.zeros(len(got), dtype=torch.int32, device=dev), ints([0], dev)
    ikv.take_slots(stack.free, one, taken, dst=dst)
    assert taken.tolist() == [len(got)] and not set(prefix.tolist()) & set(dst.tolist())


def test_debug_mode_refuses_live_lists_over_one_prefix(dev, monkeypatch):
    monkeypatch.setenv("IKV_DEBUG", "1")
    num_slots, prefix, maps, sess, S = _requests(dev, [150, 260], [30, 60])
    stack = Stack([], num_slots, dev)
    with pytest.raises(ikv.IkvError, match=r"session 1: list\[0\]"):
        ikv.return_slots(stack.free, sess, S, ints([150, 260], dev))
    assert stack() == []

"""Slots returned to the stack of free ones and taken from it, exactly, against the oracle."""
import numpy as np
import pytest

from oracle import slots_oracle as so
from paper_2606_09916_amd import ikv

pytestmark = pytest.mark.gpu


def make_sessions(Ns, spans, dev, gap=0):
    rows, o = [], 0
    for N, (qs, qe) in zip(Ns, spans):
        rows.append(dict(slot_off=o, mem_off=0, qspan_off=0, qpos_off=0, N=N, pi=0, qs=qs, qe=qe, C=N, radix_prefix=0, R=1,
                         nq=0))
        o += N + gap
    return ikv.Sessions(rows, dev)


class Stack:
    def __init__(self, slots, num_slots, dev):
        import torch
        self.buf = torch.full((num_slots,), -7, dtype=torch.int32, device=dev)
        self.buf[:len(slots)] = torch.tensor(slots, dtype=torch.int32, device=dev)
        self.count = torch.tensor([len(slots), 0], dtype=torch.int32, device=dev)
        self.free = ikv.make_free_slots(self.buf, self.count, num_slots)

    def __call__(self):
        n, word = self.count.tolist()
        assert word == 0
        return self.buf[:n].tolist()


def ints(x, dev):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=dev)


# sessions' lengths, the counts given (outside [0, N] too), slots on the stack before
GIVE = [([5], [3], 4), ([0, 4, 0, 7], [0, 4, 3, 9], 0), ([30] * 3, [-2, 30, 1], 11), ([1] * 700, [1, 0, 1, 1, 0, 2, 1] * 100, 5),
        ([4000, 1, 9000], [3500, 1, 8999], 100), ([300] * 300, [300, 7] * 150, 1)]


@pytest.mark.parametrize("Ns,counts,before", GIVE)
@pytest.mark.parametrize("gap", [0, 3])
def test_return(dev, Ns, counts, before, gap):
    import torch
    g = np.random.default_rng(len(Ns))
    width = sum(Ns) + gap * len(Ns)
    num_slots = width + before + 9
    order = 1 + g.permutation(num_slots - 1)
    s = Stack(order[:before].tolist(), num_slots, dev)
    lists = order[before:before + width].astype(np.int32)
    sess = make_sessions(Ns, [(0, 0)] * len(Ns), dev, gap)
    t = torch.from_numpy(lists).to(dev)
    ikv.return_slots(s.free, sess, t, ints(counts, dev))
    offs = np.cumsum([0] + [N + gap for N in Ns])
    want = so.give_back(order[:before].tolist(), [lists[o:o + max(0, min(c, N))].tolist() for o, c, N in zip(offs, counts, Ns)],
                        num_slots)
    assert s() == want
    assert bool((s.buf[len(want):] == -7).all()) and np.array_equal(t.cpu().numpy(), lists)


def test_return_past_the_end(dev):
    s = Stack(list(range(1, 9)), 10, dev)
    guard = s.buf.new_full((16,), 3)
    s.buf = guard
    guard[:8] = ints(list(range(1, 9)), dev)
    s.free = ikv.make_free_slots(guard, s.count, 10)
    ikv.return_slots(s.free, make_sessions([6], [(0, 0)], dev), ints([9, 11, 12, 13, 14, 15], dev), ints([5], dev))
    assert s() == list(range(1, 9)) + [9, 11] and bool((guard[10:] == 3).all())


# lengths, spans, n_new (None: the spans), live entries before, slots on the stack
TAKE = [([5], [(2, 5)], None, [1], 10), ([5], [(2, 5)], None, [1], 3), ([5], [(2, 5)], None, [1], 2), ([5], [(2, 5)], None, [3], 9),
        ([9, 0, 4, 7], [(1, 4), (0, 0), (4, 4), (0, 7)], None, [2, 0, 4, 0], 50),
        ([9] * 5, [(4, 9)] * 5, [2, 0, 5, -3, 99], [3, 9, 5, 4, -1], 30), ([9] * 5, [(4, 9)] * 5, [2, 0, 5, 1, 1], [3, 1, 4, 99, 2], 7),
        ([4] * 600, [(2, 4)] * 600, [1, 2, 0] * 200, [0, 1, 2] * 200, 500), ([3000, 5, 2000], [(0, 3000), (1, 5), (300, 2000)], None,
                                                                             [0, 1, 30], 4705),
        ([257] * 513, [(1, 257)] * 513, None, [1] * 513, 256 * 500 + 3),
        # several tiles of sessions and several workgroups, counts on the GPU, idle and full sessions among them
        ([60] * 1300, [(20, 60)] * 1300, [40, 0, 17, 99, 1] * 260, [5, 60, 21, 20, 59, 0, 30, 61, -2, 44] * 130, 20000),
        ([60] * 1300, [(20, 60)] * 1300, [40, 0, 17, 99, 1] * 260, [5, 20, 21, 20, 59, 0, 13, 1, -2, 4] * 130, 90000)]


@pytest.mark.parametrize("Ns,spans,n_new,n_live,have", TAKE)
@pytest.mark.parametrize("form", ["all", "in_place", "dst", "maps", "live"])
def test_take(dev, Ns, spans, n_new, n_live, have, form):
    import torch
    gap, B = 2, len(Ns)
    offs = np.cumsum([0] + [N + gap for N in Ns])
    width, num_slots = int(offs[-1]), 2 * have + 7
    order = (1 + np.random.default_rng(B).permutation(num_slots - 1)).tolist()
    s = Stack(order[:have], num_slots, dev)
    sess = make_sessions(Ns, spans, dev, gap)
    maps, live, dst = (torch.full((width,), -k, dtype=torch.int32, device=dev) for k in (1, 2, 3))
    nl, nn = ints(n_live, dev), None if n_new is None else ints(n_new, dev)
    n_all = nl if form == "in_place" else torch.full_like(nl, -4)
    n_taken = nn if form == "in_place" and nn is not None else torch.full_like(nl, -5)
    has = {"maps": form in ("all", "in_place", "maps"), "live": form in ("all", "in_place", "live"), "dst": form not in ("maps", "live")}
    kw = dict(slot_maps=maps if has["maps"] else None, dst=dst if has["dst"] else None)
    if has["live"]:
        kw.update(live=live, n_live=nl, n_all=n_all)
    ikv.take_slots(s.free, sess, n_taken, n_new=nn, **kw)
    spans_n = [qe - qs for qs, qe in spans]
    wants = spans_n if n_new is None else [max(0, min(w, n)) for w, n in zip(n_new, spans_n)]
    room = [max(0, min(x, N)) for x, N in zip(n_live, Ns)]
    left, got = so.take(order[:have], wants, *((room, Ns) if has["live"] else (None, None)))
    wm, wl, wd = (np.full(width, -k, np.int32) for k in (1, 2, 3))
    for b in range(B):
        n, o = len(got[b]), offs[b]
        if has["maps"]:
            wm[o + spans[b][0]:o + spans[b][0] + n] = got[b]
        if has["live"]:
            wl[o + room[b]:o + room[b] + n] = got[b]
        if has["dst"]:
            wd[o:o + n] = got[b]
    assert s() == left and n_taken.tolist() == [len(x) for x in got]
    for name, x, w in (("maps", maps, wm), ("live", live, wl), ("dst", dst, wd)):
        assert np.array_equal(x.cpu().numpy(), w), name
    if has["live"]:
        assert n_all.tolist() == [r + len(x) for r, x in zip(room, got)]
    else:
        assert n_all.tolist() == [-4] * B
    assert s.buf[:have].tolist() == order[:have] and bool((s.buf[have:] == -7).all())
    if has["dst"]:                                        # and back: the stack as it was
        ikv.return_slots(s.free, sess, dst, n_taken)
        assert s() == order[:have]


def test_counts_out_of_range(dev):
    """A count that is no count: negative as none, more than the slots as all of them."""
    sess = make_sessions([4], [(0, 4)], dev)
    for count, want in ((-3, [0]), (99, [4])):
        s = Stack(list(range(1, 8)), 9, dev)
        s.count[0] = count
        n_taken, dst = ints([9], dev), ints([0] * 4, dev)
        ikv.take_slots(s.free, sess, n_taken, dst=dst)
        assert n_taken.tolist() == want
    s = Stack([1, 2], 4, dev)
    s.count[0] = -3
    ikv.return_slots(s.free, sess, ints([3, 0, 0, 0], dev), ints([1], dev))
    assert s() == [3]


def test_captured_and_replayed(dev):
    """A padded batch's step in a graph: each replay returns the slots freed before it and takes others."""
    import torch
    B, N = 70, 40
    num_slots = 5000
    order = (1 + np.random.default_rng(2).permutation(num_slots - 1)).tolist()
    s = Stack(order[:3000], num_slots, dev)
    sess = make_sessions([N] * B, [(N - 3, N)] * B, dev)
    maps, live, dst = (torch.zeros(N * B, dtype=torch.int32, device=dev) for _ in range(3))
    n_live, n_new, n_taken = (torch.zeros(B, dtype=torch.int32, device=dev) for _ in range(3))
    freed, n_freed = torch.zeros_like(live), torch.zeros_like(n_live)

    def step():
        ikv.return_slots(s.free, sess, freed, n_freed)
        ikv.take_slots(s.free, sess, n_taken, slot_maps=maps, live=live, n_live=n_live, n_all=n_live, dst=dst, n_new=n_new)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    stack, lists = order[:3000], [[] for _ in range(B)]
    back = [[] for _ in range(B)]
    for i in range(6):
        g = np.random.default_rng(i)
        wants = g.integers(0, 4, B)
        n_new.copy_(ints(wants.tolist(), dev))
        for b in range(B):
            if back[b]:
                freed[b * N:b * N + len(back[b])] = ints(back[b], dev)
        n_freed.copy_(ints([len(x) for x in back], dev))
        graph.replay()
        torch.cuda.synchronize()
        stack = so.give_back(stack, back, num_slots)
        stack, got = so.take(stack, wants.tolist(), [len(x) for x in lists], [N] * B)
        lists = [a + b for a, b in zip(lists, got)]
        assert s() == stack and n_taken.tolist() == [len(x) for x in got]
        assert n_live.tolist() == [len(x) for x in lists]
        for b in range(B):
            assert live[b * N:b * N + len(lists[b])].tolist() == lists[b]
            assert maps[(b + 1) * N - 3:(b + 1) * N - 3 + len(got[b])].tolist() == got[b]
        back = [x[:1] for x in got]
        for b in range(B):                                # what goes back was the newest: leave it off the list
            lists[b] = lists[b][:len(lists[b]) - len(got[b])] + got[b][1:]
            live[b * N:b * N + len(lists[b])] = ints(lists[b], dev) if lists[b] else live[:0]
        n_live.copy_(ints([len(x) for x in lists], dev))


def test_another_stream(dev):
    import torch
    s = Stack(list(range(1, 200)), 300, dev)
    sess = make_sessions([50, 60], [(0, 50), (10, 60)], dev)
    n_taken, dst = ints([0, 0], dev), ints([0] * 110, dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ikv.take_slots(s.free, sess, n_taken, dst=dst, stream=side)
    ikv.return_slots(s.free, sess, dst, n_taken, stream=side)
    ikv.take_slots(s.free, sess, n_taken, dst=dst, stream=side)
    side.synchronize()
    assert dst[:50].tolist() == list(range(100, 150)) and dst[50:100].tolist() == list(range(150, 200)) and s() == list(range(1, 100))


def test_debug_mode_names_bad_entries(dev, monkeypatch):
    monkeypatch.setenv("IKV_DEBUG", "1")
    sess = make_sessions([4, 4], [(0, 2), (0, 2)], dev)
    s = Stack([1, 2, 3], 12, dev)
    lists = [4, 5, 0, 0, 6, 7, 8, 9]
    for at, value, msg in ((1, 12, r"session 0: list\[1\]"), (4, -1, r"session 1: list\[0\]"), (5, 3, r"list\[1\] = 3 is the sentinel or free"),
                           (5, 4, r"session 1: list\[1\] = 4"), (6, 0, r"session 1: list\[2\] = 0")):
        bad = list(lists)
        bad[at] = value
        with pytest.raises(ikv.IkvError, match=msg):
            ikv.return_slots(s.free, sess, ints(bad, dev), ints([2, 4], dev))
    ikv.return_slots(s.free, sess, ints(lists, dev), ints([2, 4], dev))
    n_taken = ints([0, 0], dev)
    ikv.take_slots(s.free, sess, n_taken)
    assert s() == [1, 2, 3, 4, 5] and n_taken.tolist() == [2, 2]
    for i, value in ((0, 2), (1, 12), (4, 0)):
        kept = int(s.buf[i])
        s.buf[i] = value
        with pytest.raises(ikv.IkvError, match=r"free slots: slots\["):
            ikv.take_slots(s.free, sess, n_taken)
        s.buf[i] = kept
    for bad in ([13, 0], [-1, 0], [3, 1]):
        s.count.copy_(ints(bad, dev))
        with pytest.raises(ikv.IkvError, match="free slots: count"):
            ikv.take_slots(s.free, sess, n_taken)

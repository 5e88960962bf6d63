"""The 4-bit cache and the slot stack in a session's life: a retention event, its freed slots returned, slots
taken for a turn's new tokens, their rows stored, a chunk over the list, decode steps that take one slot each
(the same step captured and replayed), the rows read back, and the event's slots in the next session's
hands. And RetentionStep's own calls of both."""
import numpy as np
import pytest

import synth
from oracle import e2m1_oracle as eo
from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from paper_2606_09916_amd.step import RetentionStep
from test_gpu_quant_rows import sessions
from test_gpu_slots import Stack, ints

pytestmark = pytest.mark.gpu


def _batch(D, kv, seed):
    specs = [synth.SessionSpec(N=900, C=200, pi=4, qs=868, qe=900, R=16, dead_frac=0.1),
             synth.SessionSpec(N=500, C=300, pi=0, qs=468, qe=500, R=16, dead_frac=0.0)]
    return synth.make_batch(synth.Shape(L=2, Hq=8, Hkv=2, D=D), specs, seed=seed, kv_dtype=kv, layout="paged")


@pytest.mark.parametrize("D,kv", [(128, synth.BF16), (64, synth.F32), (64, synth.BF16), (128, synth.F32)])
def test_step_quantises_what_it_keeps(dev, D, kv):
    import torch
    st = RetentionStep(_batch(D, kv, 82), dev)
    st.init_dead_slot()
    st.step()
    st.quantise("int8")
    for _ in range(2):
        st.quantise("e2m1")                              # another code: other buffers; again: the same
        assert st.k_codes.shape[-1] == D // 2 and st.code_scales.shape[-1] == D // 32
        u, P = (2.0 ** -8, 2.0 ** -17) if kv == synth.BF16 else (2.0 ** -24, 2.0 ** -25)
        for sinks, window in ((0, 0), (3, 64)):
            st.decode_quant(sinks, window)
            for b in range(2):
                off, n = st.sess[b].slot_off, int(st.n_live[b])
                at = st.live[off:off + n].long()
                rows = []
                for i, (pool, codes) in enumerate(((st.k_pool, st.k_codes), (st.v_pool, st.v_codes))):
                    c, s = eo.quantise(pool[:, at].double().cpu().numpy())
                    assert np.array_equal(codes[:, at].cpu().numpy(), c)
                    assert np.array_equal(st.code_scales[:, at][..., i, :].cpu().numpy(), s)
                    rows.append(eo.values(c, s))
                for l in range(2):
                    want, A, X = qo.attend(st.q_dec[b, l].double().cpu().numpy()[:, None], rows[0][l], rows[1][l], sinks, window)
                    E = ((D + 8) * X + 4 * (1 + X) + n + 8) * 2.0 ** -24
                    tol = u * np.abs(want) + (P + 2 * E[..., None]) * A
                    assert np.all(np.abs(st.out[b, l].double().cpu().numpy()[:, None] - want) <= tol)
        st.k_pool.mul_(0.5)
        st.v_pool.add_(1.0)
    freed = [st.freed[st.sess[b].slot_off:st.sess[b].slot_off + int(st.n_freed[b])].tolist() for b in range(2)]
    s = Stack([], st.num_slots, dev)
    st.return_freed(s.free)
    assert s() == freed[0] + freed[1] and len(s()) > 0
    with pytest.raises(ikv.IkvError, match="not of this one"):
        st.return_freed(Stack([], st.num_slots + 1, dev).free)
    st.quantise("e4m3")
    assert st.k_codes.dtype == torch.float8_e4m3fn


@pytest.mark.parametrize("captured", [False, True])
def test_a_turn(dev, captured):
    import torch
    L, Hq, Hkv, D = 2, 8, 2, 128
    st = RetentionStep(_batch(D, synth.BF16, 83), dev)
    st.init_dead_slot()
    st.step()
    st.quantise("e2m1")
    stack = Stack([], st.num_slots, dev)
    st.return_freed(stack.free)
    gone = stack()
    nl = st.n_live.tolist()
    B, new, steps = 2, [37, 5], 4
    # the turn's lists: the kept slots, room for the new tokens and the decode steps
    Ns = [n + t + steps for n, t in zip(nl, new)]
    rows, o, oc = [], 0, 0
    for b in range(B):
        rows.append(dict(slot_off=o, mem_off=0, qspan_off=0, qpos_off=0, N=Ns[b], pi=0, qs=nl[b], qe=nl[b] + new[b], C=Ns[b],
                         radix_prefix=0, R=1, nq=0))
        o += Ns[b]
    sess = ikv.Sessions(rows, dev)
    live, dst = (torch.zeros(o, dtype=torch.int32, device=dev) for _ in range(2))
    for b in range(B):
        live[rows[b]["slot_off"]:rows[b]["slot_off"] + nl[b]] = st.live[st.sess[b].slot_off:st.sess[b].slot_off + nl[b]]
    n_all, n_taken = ints([0, 0], dev), ints([0, 0], dev)
    ikv.take_slots(stack.free, sess, n_taken, live=live, n_live=st.n_live, n_all=n_all, dst=dst)
    assert n_taken.tolist() == new and n_all.tolist() == [a + b for a, b in zip(nl, new)]
    assert stack() == gone[:len(gone) - sum(new)]
    taken = [dst[rows[b]["slot_off"]:rows[b]["slot_off"] + new[b]].tolist() for b in range(B)]
    assert taken[0] + taken[1] == gone[len(gone) - sum(new):]

    # their rows, from a pool of new rows laid out like the lists
    g = torch.Generator(device=dev).manual_seed(5)
    rn = lambda *z: torch.randn(*z, generator=g, device=dev).bfloat16()  # noqa: E731
    held = {}                                            # slot: what its rows stand for
    def stored(which, slots, x):                         # x [L, n, Hkv, D]
        v = eo.values(*eo.quantise(x.double().cpu().numpy()))
        for i, u in enumerate(slots):
            held[which, u] = v[:, i]

    for b in range(B):
        at = live[rows[b]["slot_off"]:rows[b]["slot_off"] + nl[b]].long()
        for which, pool in (("k", st.k_pool), ("v", st.v_pool)):
            stored(which, at.tolist(), pool[:, at])
    kn, vn = rn(L, o, Hkv, D), rn(L, o, Hkv, D)
    ikv.quant_store(st.cache, ikv.make_pool(kn, vn, L, Hq, Hkv, D, o, 0), sess, None, dst, n_taken)
    for b in range(B):
        off = rows[b]["slot_off"]
        for which, x in (("k", kn), ("v", vn)):
            stored(which, taken[b], x[:, off:off + new[b]])

    ws = ikv.Workspace(dev)
    def check(q, out, ns, lens, sinks, window, P):
        at = 0
        for b in range(B):
            slots = live[rows[b]["slot_off"]:rows[b]["slot_off"] + lens[b]].tolist()
            n = ns[b]
            qq, got = (x[at:at + L * Hq * n * D].view(L, Hq, n, D).double().cpu().numpy() for x in (q, out))
            at += L * Hq * n * D
            for l in range(L):
                k, v = (np.stack([held[w, u][l] for u in slots]) for w in "kv")
                want, A, X = qo.attend(qq[l], k, v, sinks, window)
                E = ((D + 8) * X + 4 * (1 + X) + lens[b] + 8) * 2.0 ** -24
                assert np.all(np.abs(got[l] - want) <= 2.0 ** -8 * np.abs(want) + (P + 2 * E[..., None]) * A)

    q = rn(sum(new) * L * Hq * D)
    out = torch.empty_like(q)
    ikv.attend_chunk_quant(st.cache, sess, q, live, n_all, out, ws, sinks=2, window=150)
    check(q, out, new, n_all.tolist(), 2, 150, 2.0 ** -8)

    # decode steps: a slot each, its row, the list with it
    lens = n_all.tolist()
    one = ikv.Sessions([dict(r, qs=0, qe=1) for r in rows], dev)
    k1, v1 = torch.zeros(L, o, Hkv, D, dtype=torch.bfloat16, device=dev), torch.zeros(L, o, Hkv, D, dtype=torch.bfloat16, device=dev)
    fresh = ikv.make_pool(k1, v1, L, Hq, Hkv, D, o, 0)
    qd = torch.zeros(B * L * Hq * D, dtype=torch.bfloat16, device=dev)
    od = torch.zeros_like(qd)
    n_new = ints([0, 0], dev)                            # nothing yet: the calls warm up

    def step():
        ikv.take_slots(stack.free, one, n_taken, live=live, n_live=n_all, n_all=n_all, dst=dst, n_new=n_new)
        ikv.quant_store(st.cache, fresh, one, None, dst, n_taken)
        ikv.decode_attend_quant(st.cache, one, qd, live, n_all, od, ws, sinks=2, window=150)

    run = step
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    assert n_all.tolist() == lens
    for t in range(steps):
        wants = [1, 1 if t != 1 else 0]                  # in the second step the second session is idle
        n_new.copy_(ints(wants, dev))
        qd.copy_(rn(B * L * Hq * D))
        before = stack()
        for b in range(B):
            off = rows[b]["slot_off"]
            k1[:, off], v1[:, off] = rn(L, Hkv, D), rn(L, Hkv, D)
        run()
        torch.cuda.synchronize()
        assert n_taken.tolist() == wants and stack() == before[:len(before) - sum(wants)]
        mine = before[len(before) - sum(wants):]
        for b in range(B):
            if wants[b]:
                off, u = rows[b]["slot_off"], mine.pop(0)
                assert int(live[off + lens[b]]) == u
                stored("k", [u], k1[:, off:off + 1])
                stored("v", [u], v1[:, off:off + 1])
                lens[b] += 1
        assert n_all.tolist() == lens
        check(qd, od, [1, 1], lens, 2, 150, 2.0 ** -17)
    # the rows read back are what was held
    k2, v2 = torch.zeros(L, o, Hkv, D, dtype=torch.bfloat16, device=dev), torch.zeros(L, o, Hkv, D, dtype=torch.bfloat16, device=dev)
    ikv.quant_load(st.cache, ikv.make_pool(k2, v2, L, Hq, Hkv, D, o, 0), sess, live, None, n_all)
    for b in range(B):
        off = rows[b]["slot_off"]
        for which, x in (("k", k2), ("v", v2)):
            want = np.stack([held[which, int(u)] for u in live[off:off + lens[b]]], 1)
            assert np.array_equal(x[:, off:off + lens[b]].double().cpu().numpy(), want)
    # the requests end: all their slots go back
    before = stack()
    ikv.return_slots(stack.free, sess, live, n_all)
    assert stack() == before + [int(u) for b in range(B) for u in live[rows[b]["slot_off"]:rows[b]["slot_off"] + lens[b]]]
    assert len(set(stack())) == len(stack())


def test_two_stacks_on_two_streams(dev):
    """Calls on different stacks do not share anything."""
    import torch
    n = 40000
    a, b = Stack(list(range(1, n)), n, dev), Stack(list(range(1, n)), n, dev)
    sess = sessions([19000, 20000], dev, 18000)
    out = [[torch.zeros(39000, dtype=torch.int32, device=dev), ints([0, 0], dev)] for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for s, (dst, taken), st in zip((a, b), out, streams):
            ikv.take_slots(s.free, sess, taken, dst=dst, stream=st)
            ikv.return_slots(s.free, sess, dst, taken, stream=st)
    torch.cuda.synchronize()
    assert a() == b() == list(range(1, n)) and torch.equal(out[0][0], out[1][0])
    assert out[0][0][:18000].tolist() == list(range(n - 36000, n - 18000))

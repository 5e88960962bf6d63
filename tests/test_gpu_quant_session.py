"""The 8-bit cache in a session's life: a retention event on the bf16 pool, the kept rows
moved into the cache, decode steps that append tokens, a chunk over both forms, and the rows
read back for the next event's scores."""
import numpy as np
import pytest

import synth
from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from paper_2606_09916_amd.step import RetentionStep
from test_gpu_quant_rows import _code_type, sessions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_session(dev, code):
    import torch
    L, Hq, Hkv, D = 2, 8, 2, 128
    spec = synth.SessionSpec(N=1200, C=300, pi=4, qs=1136, qe=1200, R=16, dead_frac=0.1)
    batch = synth.make_batch(synth.Shape(L=L, Hq=Hq, Hkv=Hkv, D=D), [spec], seed=81, kv_dtype=synth.BF16, layout="paged")
    st = RetentionStep(batch, dev)
    st.init_dead_slot()
    st.step()
    nl = int(st.n_live[0])
    new, cap = 6, nl + 6
    slots = st.num_slots + new
    ct = _code_type(code)
    kc, vc = (torch.zeros(L, slots, Hkv, D, dtype=torch.int8, device=dev).view(ct) for _ in range(2))
    sc = torch.ones(L, slots, Hkv, 2, device=dev)
    cache = ikv.make_quant_pool(kc, vc, sc, L, Hq, Hkv, D, slots, st.dead)
    # the event's kept rows, same slots
    ikv.quant_store(cache, st.pool, st.sess, st.live, st.live, st.n_live)

    def held(which, l, at):
        c = (kc if which == "k" else vc)[l].view(torch.uint8)[at].cpu().numpy()
        return qo.code_values(c, code) * sc[l][at][..., 0 if which == "k" else 1].double().cpu().numpy()[..., None]

    def check(got, q, n, N, sinks, window):
        at = live[:N].long()
        for l in range(L):
            want, A, X = qo.attend(q.view(L, Hq, n, D)[l].double().cpu().numpy(), held("k", l, at), held("v", l, at),
                                   sinks, window)
            E = ((D + 8) * X + 4 * (1 + X) + N + 8) * 2.0 ** -24
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2 * E[..., None]) * A
            assert np.all(np.abs(got.view(L, Hq, n, D)[l].double().cpu().numpy() - want) <= tol)

    # decode: each step writes its token's rows and reads the list with them
    live = torch.cat([st.live[:nl], torch.arange(st.num_slots, slots, device=dev, dtype=torch.int32)])
    n_live = torch.tensor([nl], dtype=torch.int32, device=dev)
    g = torch.Generator(device=dev).manual_seed(4)
    rn = lambda *z: torch.randn(*z, generator=g, device=dev).bfloat16()  # noqa: E731
    k_new, v_new = rn(L, new, Hkv, D), rn(L, new, Hkv, D)
    ws, sess = ikv.Workspace(dev), sessions([cap], dev, new)
    one = sessions([1], dev)
    for t in range(new):
        fresh = ikv.make_pool(k_new[:, t:t + 1].contiguous(), v_new[:, t:t + 1].contiguous(), L, Hq, Hkv, D, 1, 0)
        ikv.quant_store(cache, fresh, one, None, live[nl + t:nl + t + 1].clone())
        n_live += 1
        q = rn(L * Hq * D)
        out = torch.empty_like(q)
        ikv.decode_attend_quant(cache, sess, q, live, n_live, out, ws, sinks=4, window=100)
        check(out, q, 1, nl + t + 1, 4, 100)
    # the same tokens as one chunk, over the cache and over a bf16 pool with the rows read back
    q = rn(L * Hq * new * D)
    out, out16 = torch.empty_like(q), torch.empty_like(q)
    ikv.attend_chunk_quant(cache, sess, q, live, n_live, out, ws)
    check(out, q, new, cap, 0, 0)
    k2, v2 = (torch.zeros(L, slots, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    back = ikv.make_pool(k2, v2, L, Hq, Hkv, D, slots, st.dead)
    ikv.quant_load(cache, back, sess, live, live, n_live)
    at = live.long()
    for which, x in (("k", k2), ("v", v2)):
        for l in range(L):
            want = held(which, l, at)
            assert np.all(np.abs(x[l][at].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want))
    ikv.attend_chunk(back, sess, q, live, n_live, out16, ws)
    # read back, the rows differ by a bf16 rounding (int8) or not at all (e4m3)
    d = (out16.float() - out.float()).abs().max() / out.float().abs().max()
    assert float(d) <= 2.0 ** -5
    # the next event's scores on the rows read back
    import oracle
    rows = [dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=cap, pi=4, qs=nl, qe=cap, C=100, radix_prefix=4, R=16,
                 nq=0)]
    s2 = ikv.Sessions(rows, dev)
    scores = torch.zeros(cap, device=dev)
    ikv.init_dead_slot(back)
    ikv.score_history(back, s2, live, st.M, scores, ws)
    k_host = k2.view(torch.int16).cpu().numpy().view(np.uint16)
    S = live.cpu().numpy()
    sets = oracle.sets(S, 4, nl, cap, 100, st.dead)
    want = oracle.scores(k_host, S, sets, st.M.cpu().numpy().reshape(L, Hkv * 16, D), Hkv, 16)
    c = sets["cand"]
    assert np.all(np.abs(scores.cpu().numpy()[c] - want[c]) <= 1e-3 * np.abs(want[c]) + 1e-6 * np.abs(want[c]).max())


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("D,kv", [(128, synth.BF16), (64, synth.F32)])
def test_step_quantises_what_it_keeps(dev, code, D, kv):
    """RetentionStep.quantise and decode_quant after an event, two sessions, both pool types."""
    L, Hq, Hkv = 2, 8, 2
    specs = [synth.SessionSpec(N=900, C=200, pi=4, qs=868, qe=900, R=16, dead_frac=0.1),
             synth.SessionSpec(N=500, C=300, pi=0, qs=468, qe=500, R=16, dead_frac=0.0)]
    batch = synth.make_batch(synth.Shape(L=L, Hq=Hq, Hkv=Hkv, D=D), specs, seed=82, kv_dtype=kv, layout="paged")
    st = RetentionStep(batch, dev)
    st.init_dead_slot()
    st.step()
    full = st.host("out")
    st.quantise(code)
    u, P = (2.0 ** -8, 2.0 ** -8) if kv == synth.BF16 else (2.0 ** -24, 2.0 ** -22)
    for sinks, window in ((0, 0), (3, 64)):
        st.decode_quant(sinks, window)
        for b in range(2):
            off, n = st.sess[b].slot_off, int(st.n_live[b])
            at = st.live[off:off + n].long()
            for l in range(L):
                k, v = (qo.code_values(c[l].view(torch_uint8())[at].cpu().numpy(), code)
                        * st.code_scales[l][at][..., i].double().cpu().numpy()[..., None]
                        for i, c in enumerate((st.k_codes, st.v_codes)))
                want, A, X = qo.attend(st.q_dec[b, l].double().cpu().numpy()[:, None], k, v, sinks, window)
                E = ((D + 8) * X + 4 * (1 + X) + n + 8) * 2.0 ** -24
                tol = u * np.abs(want) + (P + 2 * E[..., None]) * A
                assert np.all(np.abs(st.out[b, l].double().cpu().numpy()[:, None] - want) <= tol)
    assert full.shape == st.host("out").shape


def torch_uint8():
    import torch
    return torch.uint8

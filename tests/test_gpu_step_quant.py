"""RetentionStep.quantise takes the live rows of the step's own pool, keys as keys and values as
values, and the decode over them is the attention of those rows: both against the oracle's codes of
the pool, not against what the step wrote."""
import numpy as np
import pytest

import synth
from oracle import quant_oracle as qo
from paper_2606_09916_amd.step import RetentionStep

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("D,kv", [(128, synth.BF16), (64, synth.F32)])
def test_codes_are_the_pools(dev, code, D, kv):
    import torch
    L, Hq, Hkv = 3, 8, 2
    specs = [synth.SessionSpec(N=700, C=150, pi=4, qs=668, qe=700, R=16, dead_frac=0.1),
             synth.SessionSpec(N=400, C=500, pi=0, qs=368, qe=400, R=16, dead_frac=0.0)]
    batch = synth.make_batch(synth.Shape(L=L, Hq=Hq, Hkv=Hkv, D=D), specs, seed=91, kv_dtype=kv, layout="paged")
    st = RetentionStep(batch, dev)
    st.init_dead_slot()
    st.step()
    buffers = None
    for _ in range(2):
        st.quantise(code)
        assert buffers in (None, st.k_codes.data_ptr())  # quantising again writes the buffers that are there
        buffers = st.k_codes.data_ptr()
        st.decode_quant(2, 100)
        u, P = (2.0 ** -8, 2.0 ** -17) if kv == synth.BF16 else (2.0 ** -24, 2.0 ** -25)
        for b in range(2):
            off, n = st.sess[b].slot_off, int(st.n_live[b])
            at = st.live[off:off + n].long()
            rows = {}
            for i, (pool, codes) in enumerate(((st.k_pool, st.k_codes), (st.v_pool, st.v_codes))):
                c, s = qo.quantise(pool[:, at].double().cpu().numpy(), code)
                assert np.array_equal(codes.view(torch.uint8)[:, at].cpu().numpy(), c)
                assert np.array_equal(st.code_scales[:, at][..., i].cpu().numpy(), s)
                rows[i] = qo.code_values(c, code) * s[..., None].astype(np.float64)
            for l in range(L):
                want, A, X = qo.attend(st.q_dec[b, l].double().cpu().numpy()[:, None], rows[0][l], rows[1][l], 2, 100)
                E = ((D + 8) * X + 4 * (1 + X) + n + 8) * 2.0 ** -24
                tol = u * np.abs(want) + (P + 2 * E[..., None]) * A
                assert np.all(np.abs(st.out[b, l].double().cpu().numpy()[:, None] - want) <= tol)
        st.k_pool.mul_(0.5)                              # other rows in the pool for the second time
        st.v_pool.add_(1.0)

"""The calls of the 8-bit cache and the chunk attention refuse descriptors and workspaces whose
memory is on another device than the sessions': the kernels would read host memory, or another
GPU's. (No GPU needed: "meta" stands for the other device.)"""
import pytest
import torch

from paper_2606_09916_amd import ikv

OTHER = torch.device("meta")


def _args(N=700, n=40):
    rows = [dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=N, pi=0, qs=N - n, qe=N, C=N, radix_prefix=0, R=1, nq=0)]
    sess = ikv.Sessions(rows, "cpu")
    q = torch.zeros(n * 4 * 64, dtype=torch.bfloat16)
    return sess, q, torch.zeros(N, dtype=torch.int32), torch.ones(1, dtype=torch.int32)


def _cache(dev, scales=None):
    kc = torch.zeros(1, 4, 2, 64, dtype=torch.int8, device=dev)
    return ikv.make_quant_pool(kc, kc, torch.zeros(1, 4, 2, 2, device=scales or dev), 1, 4, 2, 64, 4)


def _pool(dev):
    k = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16, device=dev)
    p = ikv.make_pool(k, k, 1, 4, 2, 64, 4)
    p.k_pool = p.v_pool = 0x10000                        # "meta" tensors have no address
    return p


def test_cache_in_two_places():
    with pytest.raises(ikv.IkvError, match="on different devices"):
        _cache("cpu", OTHER)


def test_descriptors_elsewhere():
    sess, q, live, n = _args()
    far = _cache("cpu")
    far.device = OTHER
    ws = ikv.Workspace("cpu")
    for call in (lambda: ikv.attend_chunk_quant(far, sess, q, live, n, q.clone(), ws),
                 lambda: ikv.decode_attend_quant(far, sess, q, live, n, q.clone(), ws),
                 lambda: ikv.attend_chunk(_pool(OTHER), sess, q, live, n, q.clone(), ws),
                 lambda: ikv.quant_store(far, _pool("cpu"), sess, live, live),
                 lambda: ikv.quant_store(_cache("cpu"), _pool(OTHER), sess, live, live),
                 lambda: ikv.quant_load(far, _pool("cpu"), sess, live, live),
                 lambda: ikv.quant_load(_cache("cpu"), _pool(OTHER), sess, live, live)):
        with pytest.raises(ikv.IkvError, match="on different devices"):
            call()
    for call in (lambda: ikv.attend_chunk(_pool("cpu"), sess, q, live, n, q.clone(), ws),
                 lambda: ikv.quant_load(_cache("cpu"), _pool("cpu"), sess, live, live)):
        with pytest.raises(ikv.IkvError, match="not on a GPU"):
            call()


def test_workspace_elsewhere():
    sess, q, live, n = _args()
    assert ikv.quant_workspace_bytes(_cache("cpu"), sess, ikv.CALL_CHUNK) > 0
    with pytest.raises(ikv.IkvError, match="on different devices"):
        ikv.attend_chunk_quant(_cache("cpu"), sess, q, live, n, q.clone(), ikv.Workspace(OTHER))

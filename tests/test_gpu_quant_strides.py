"""Lists so long that the row kernels' workgroups stride over them (a launch's most are 2^17, 2^15 where there is
no source list): rows at either end of a stride, few among entries of the dead slot, bit for bit against the
oracles."""
import numpy as np
import pytest

from oracle import e2m1_oracle as eo
from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from test_gpu_e2m1_rows import empty_four
from test_gpu_quant_rows import _dt, empty_cache, sessions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", ["int8", "e4m3", "e2m1"])
@pytest.mark.parametrize("dtype,D,new_rows", [("bf16", 128, False), ("f32", 64, False), ("bf16", 64, True)])
def test_long_padded_lists(dev, code, dtype, D, new_rows):
    import torch
    L, Hkv = 1, 64                                       # an entry is a workgroup's work
    N = 40001 if new_rows else 150001
    most = 1 << (15 if new_rows else 17)
    at = sorted({0, 1, 63, most - 1, most, most + 1, N - 3, N - 2} | set(range(7, N - 2, 997 if new_rows else 4999)))
    places = torch.tensor(at)
    slots = len(at) + 5
    pslots = N if new_rows else slots
    g = torch.Generator(device=dev).manual_seed(N)
    own = places if new_rows else 2 + torch.randperm(len(at), generator=torch.Generator().manual_seed(1))
    k, v = (torch.zeros(L, pslots, Hkv, D, dtype=_dt(dtype), device=dev) for _ in range(2))
    for x in (k, v):
        x[:, own.to(dev)] = torch.randn(L, len(at), Hkv, D, generator=g, device=dev).to(_dt(dtype))
    kc, vc, sc = empty_four(L, slots, Hkv, D, dev) if code == "e2m1" else empty_cache(code, L, slots, Hkv, D, dev)
    dst, src = torch.zeros(N, dtype=torch.int32), torch.zeros(N, dtype=torch.int32)
    to = 1 + torch.randperm(slots - 1, generator=torch.Generator().manual_seed(2))[:len(at)]
    dst[places], src[places] = to.int(), own.int()
    dst[N - 1] = int(set(range(1, slots)).difference(to.tolist()).pop())          # behind the rows: not taken
    sess, n_rows = sessions([N], dev), torch.tensor([N - 1], dtype=torch.int32, device=dev)
    cache = ikv.make_quant_pool(kc, vc, sc, L, Hkv, Hkv, D, slots, 0, io_dtype=_dt(dtype))
    ikv.quant_store(cache, ikv.make_pool(k, v, L, Hkv, Hkv, D, pslots, 0), sess, None if new_rows else src.to(dev),
                    dst.to(dev), n_rows)
    want = []
    for codes, x, i in ((kc, k, 0), (vc, v, 1)):
        rows = x[:, own.to(dev)].double().cpu().numpy()
        wc, ws = eo.quantise(rows) if code == "e2m1" else qo.quantise(rows, code)
        full = np.full(tuple(codes.shape), 5, np.uint8)
        full[:, to.numpy()] = wc
        assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), full)
        got = sc[..., i, :] if code == "e2m1" else sc[..., i]
        full = np.full(tuple(got.shape), 77 if code == "e2m1" else 0.25, ws.dtype if code == "e2m1" else np.float32)
        full[:, to.numpy()] = ws
        assert np.array_equal(got.cpu().numpy(), full)
        want.append(torch.from_numpy(eo.values(wc, ws)) if code == "e2m1" else
                    torch.from_numpy(qo.code_values(wc, code).astype(np.float32) * ws[..., None].astype(np.float32)))
    # back into a pool of as many rows: the load's list too is mostly of the dead slot
    k2, v2 = (torch.full((L, slots, Hkv, D), 3.0, dtype=_dt(dtype), device=dev) for _ in range(2))
    ikv.quant_load(cache, ikv.make_pool(k2, v2, L, Hkv, Hkv, D, slots, 0), sess, dst.to(dev), dst.to(dev), n_rows)
    for x, w in zip((k2, v2), want):
        full = torch.full_like(x, 3.0).cpu()
        full[:, to] = w.to(x.dtype)
        assert torch.equal(x.cpu(), full)


# bytes of the pool's rows: 36 * 8 * 128 * 4 of an entry of N
@pytest.mark.parametrize("N,store,load", [(100, "k_quant_store", "k_quant_load"), (900, "k_quant_store", "k_quant_load"),
                                          (1021, "k_quant_store", "k_quant_load<past>"),
                                          (2000, "k_quant_store<past>", "k_quant_load<past>")])
@pytest.mark.parametrize("code", ["int8", "e2m1"])
def test_rows_that_the_caches_keep(dev, code, N, store, load):
    """Which calls write through the caches, for the one that reads next, and which past them."""
    import torch
    L, Hkv, D = 36, 8, 128
    k, v = (torch.zeros(L, 9, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    kc, vc, sc = empty_four(L, 9, Hkv, D, dev) if code == "e2m1" else empty_cache(code, L, 9, Hkv, D, dev)
    pool, cache = ikv.make_pool(k, v, L, Hkv, Hkv, D, 9, 0), ikv.make_quant_pool(kc, vc, sc, L, Hkv, Hkv, D, 9, 0)
    ids, n = torch.ones(N, dtype=torch.int32, device=dev), torch.ones(1, dtype=torch.int32, device=dev)
    row = dict(slot_off=0, mem_off=0, qspan_off=0, qpos_off=0, N=N, pi=0, qs=N, qe=N, C=N, radix_prefix=0, R=1, nq=0)

    def launched(call, **kw):
        ikv.timing(True)
        call(cache, pool, ikv.Sessions([{**row, **kw}], dev), ids, ids, n)
        torch.cuda.synchronize()
        ikv.timing(False)
        return [name for name, _ in ikv.timing_read()]

    assert launched(ikv.quant_store) == [store] and launched(ikv.quant_load) == [load]
    # a list with room for a history of which the budget keeps a few
    assert launched(ikv.quant_store, C=500) == ["k_quant_store"] and launched(ikv.quant_load, C=500) == ["k_quant_load"]

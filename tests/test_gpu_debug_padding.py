"""IKV_DEBUG=1 and padded lists: an entry whose cache slot is the dead one is skipped, and what its
pool id holds does not matter, as without the checks."""
import pytest

from paper_2606_09916_amd import ikv
from test_gpu_quant_rows import empty_cache, sessions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("debug", ["0", "1"])
def test_padded_entries(dev, monkeypatch, debug):
    import torch
    monkeypatch.setenv("IKV_DEBUG", debug)
    L, Hkv, D, N = 1, 2, 64, 8
    k = torch.randn(L, N, Hkv, D, device=dev)
    kc, vc, sc = empty_cache("int8", L, N + 1, Hkv, D, dev)
    cache = ikv.make_quant_pool(kc, vc, sc, L, Hkv, Hkv, D, N + 1, 0)
    sess = sessions([N], dev)
    cache_ids = torch.tensor([0, 1, 2, 0, 4, 5, 0, 7], dtype=torch.int32, device=dev)
    pool_ids = torch.tensor([-1, 1, 2, N, 4, 5, 2 ** 31 - 1, 7], dtype=torch.int32, device=dev)
    pad = cache_ids == 0
    ikv.quant_store(cache, ikv.make_pool(k, k, L, Hkv, Hkv, D, N, 0), sess, pool_ids, cache_ids)
    assert bool((kc[:, [0, 3, 6, 8]].view(torch.int8) == 5).all()) and bool((sc[:, [0, 3, 6, 8]] == 0.25).all())
    back, back_v = torch.full_like(k, 3.0), torch.full_like(k, 3.0)
    pool = ikv.make_pool(back, back_v, L, Hkv, Hkv, D, N, 0)
    ikv.quant_load(cache, pool, sess, cache_ids, pool_ids)
    assert bool((back[:, pad] == 3).all())
    # half a step a / 254, and two float32 roundings (scale, product) of at most a: 2 * 2^-24 * 254 steps < 2^-14 of it
    step = k[:, ~pad].abs().amax(-1, keepdim=True) / 254
    assert bool(((back[:, ~pad] - k[:, ~pad]).abs() <= step * (1 + 2.0 ** -14)).all())
    if debug == "0":
        return
    # entries that are not skipped are still named
    bad = pool_ids.clone()
    bad[4] = N
    with pytest.raises(ikv.IkvError, match=r"src\[4\]"):
        ikv.quant_store(cache, pool, sess, bad, cache_ids)
    with pytest.raises(ikv.IkvError, match=r"dst\[4\]"):
        ikv.quant_load(cache, pool, sess, cache_ids, bad)

"""Rows of many KV heads into the 8-bit cache and back where the sessions' lists are far longer
than the rows listed: workgroups of millions of entries past them have nothing to do."""
import numpy as np
import pytest

from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from test_gpu_quant_rows import empty_cache, sessions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("Hkv,N", [(32, 5_000_100), (16, 9_000_100)])
def test_few_rows_of_a_long_list(dev, code, Hkv, N):
    import torch
    D, slots, rows, short = 128, 40, 10, 7
    lengths = [N, short]
    k, v = (torch.randn(1, slots, Hkv, D, device=dev).bfloat16() for _ in range(2))
    kc, vc, sc = empty_cache(code, 1, slots, Hkv, D, dev)
    # entries past the rows name slots that must stay as they are
    src, dst = torch.full((N + short,), 39, dtype=torch.int32), torch.full((N + short,), 38, dtype=torch.int32)
    src[:rows], dst[:rows] = torch.arange(rows), torch.arange(1, 1 + rows)
    src[N:], dst[N:] = torch.arange(20, 20 + short), torch.arange(21, 21 + short)
    n_rows = torch.tensor([rows, short], dtype=torch.int32, device=dev)
    from_, to = (torch.cat([x[:rows], x[N:]]).long() for x in (src, dst))
    sess = sessions(lengths, dev)
    cache = ikv.make_quant_pool(kc, vc, sc, 1, Hkv, Hkv, D, slots, 0)
    ikv.quant_store(cache, ikv.make_pool(k, v, 1, Hkv, Hkv, D, slots, 0), sess, src.to(dev), dst.to(dev), n_rows)
    want = {}
    for name, codes, x, i in (("k", kc, k, 0), ("v", vc, v, 1)):
        wc, ws = qo.quantise(x[:, from_.to(dev)].double().cpu().numpy(), code)
        full, fs = np.full((1, slots, Hkv, D), 5, np.uint8), np.full((1, slots, Hkv), 0.25, np.float32)
        full[:, to.numpy()], fs[:, to.numpy()] = wc, ws
        assert np.array_equal(codes.view(torch.uint8).cpu().numpy(), full), name
        assert np.array_equal(sc[..., i].cpu().numpy(), fs), name
        want[name] = (qo.code_values(wc, code).astype(np.float32) * ws[..., None]).astype(np.float32)
    k2, v2 = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    ikv.quant_load(cache, ikv.make_pool(k2, v2, 1, Hkv, Hkv, D, slots, 0), sess, dst.to(dev), src.to(dev), n_rows)
    for name, x in (("k", k2), ("v", v2)):
        full = torch.full_like(x, 3.0).cpu()
        full[:, from_] = torch.from_numpy(want[name]).to(x.dtype)
        assert torch.equal(x.cpu(), full), name

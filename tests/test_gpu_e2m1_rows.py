"""Rows into the 4-bit cache and back, bit for bit against the float64 oracle."""
import numpy as np
import pytest

from oracle import e2m1_oracle as eo
from paper_2606_09916_amd import ikv
from test_gpu_quant_rows import _dt, awkward_rows, sessions

pytestmark = pytest.mark.gpu


def empty_four(L, slots, Hkv, D, dev, fill=5):
    import torch
    kc = torch.full((L, slots, Hkv, D // 2), fill, dtype=torch.uint8, device=dev)
    return kc, kc.clone(), torch.full((L, slots, Hkv, 2, D // 32), 77, dtype=torch.uint8, device=dev)


def awkward_blocks(L, slots, Hkv, D, dtype, dev, seed):
    """awkward_rows, and blocks of a row that differ by many powers of two, next to each tie and scale border."""
    import torch
    x = awkward_rows(L, slots, Hkv, D, dtype, dev, seed).float()
    g = torch.Generator(device=dev).manual_seed(seed + 99)
    kind = torch.randint(0, 5, (L, slots, Hkv, D // 32, 1), generator=g, device=dev)
    size = torch.exp2(torch.randint(-60, 60, kind.shape, generator=g, device=dev).float())
    ties = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, .2507, 5.02, 6.98], device=dev)
    t = ties[torch.randint(0, 12, (L, slots, Hkv, D // 32, 32), generator=g, device=dev)]
    t = t * (torch.randint(0, 2, t.shape, generator=g, device=dev) * 2 - 1)
    y = x.unflatten(-1, (-1, 32))
    y = torch.where(kind == 1, y * size, y)
    y = torch.where(kind == 2, t * size, y)
    y = torch.where(kind == 3, t * 2.0 ** 125, y)                            # past the largest scale; past float32 for some
    return y.flatten(-2).to(_dt(dtype)).contiguous()


def same(a, b):
    import torch
    return torch.equal(torch.nan_to_num(a, nan=7.0, posinf=8.0, neginf=9.0), torch.nan_to_num(b, nan=7.0, posinf=8.0, neginf=9.0))


@pytest.mark.parametrize("dtype,L,Hkv,D,lengths", [
    ("bf16", 1, 1, 64, [1]), ("bf16", 3, 8, 128, [37, 0, 5]), ("f32", 2, 2, 64, [33, 64]), ("f32", 1, 3, 128, [50]),
    ("bf16", 2, 3, 128, [129]), ("bf16", 5, 4, 64, [1, 1, 1, 1, 1, 1, 1]), ("f32", 1, 1, 128, [1]), ("bf16", 1, 5, 64, [77])])
def test_store_and_load(dev, dtype, L, Hkv, D, lengths):
    import torch
    total = sum(lengths)
    pslots, cslots = 2 * total + 3, 3 * total + 2
    k, v = (awkward_blocks(L, pslots, Hkv, D, dtype, dev, s) for s in (total, total + 1))
    kc, vc, sc = empty_four(L, cslots, Hkv, D, dev)
    g = torch.Generator().manual_seed(total)
    src = torch.randperm(pslots, generator=g)[:total].int()
    dst = (1 + torch.randperm(cslots - 1, generator=g)[:total]).int()
    dst[torch.rand(total, generator=g) < 0.1] = 0                            # padding: the dead slot
    n_rows = torch.tensor([max(0, N - i) for i, N in enumerate(lengths)], dtype=torch.int32)
    used = torch.cat([torch.arange(N) < n for N, n in zip(lengths, n_rows.tolist())]) & (dst != 0)
    sess = sessions(lengths, dev)
    pool = ikv.make_pool(k, v, L, Hkv, Hkv, D, pslots, 0)
    cache = ikv.make_quant_pool(kc, vc, sc, L, Hkv, Hkv, D, cslots, 0)
    ikv.quant_store(cache, pool, sess, src.to(dev), dst.to(dev), n_rows.to(dev))
    want = {}
    from_, to = src[used].long(), dst[used].long()
    for name, codes, x, i in (("k", kc, k, 0), ("v", vc, v, 1)):
        wc, ws = eo.quantise(x[:, from_.to(dev)].double().cpu().numpy())
        full = np.full(tuple(codes.shape), 5, np.uint8)
        full[:, to.numpy()] = wc
        assert np.array_equal(codes.cpu().numpy(), full), name
        fs = np.full(tuple(sc[..., i, :].shape), 77, np.uint8)
        fs[:, to.numpy()] = ws
        assert np.array_equal(sc[..., i, :].cpu().numpy(), fs), name
        want[name] = torch.from_numpy(eo.values(wc, ws))
    # back, to rows of the pool's type, exactly; rows that are not listed stay
    k2, v2 = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    back = ikv.make_pool(k2, v2, L, Hkv, Hkv, D, pslots, 0)
    ikv.quant_load(cache, back, sess, dst.to(dev), src.to(dev), n_rows.to(dev))
    for name, x in (("k", k2), ("v", v2)):
        full = torch.full_like(x, 3.0).cpu().double()
        full[:, from_] = want[name]
        assert same(x.cpu().double(), full), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_with_every_scale(dev, dtype):
    """Whoever wrote them: bytes 0 .. 255 of the scale, all 256 pairs of codes."""
    import torch
    kc = torch.arange(256, device=dev).to(torch.uint8).view(1, 1, 4, 64).expand(1, 256, 4, 64).contiguous()
    sc = torch.arange(256, device=dev).to(torch.uint8).view(1, 256, 1, 1, 1).expand(1, 256, 4, 2, 4).contiguous()
    k, v = (torch.zeros(1, 256, 4, 128, dtype=_dt(dtype), device=dev) for _ in range(2))
    sess = sessions([256], dev)
    cache = ikv.make_quant_pool(kc, kc.clone(), sc, 1, 4, 4, 128, 256, 255)
    order = torch.randperm(256, generator=torch.Generator().manual_seed(1)).int().to(dev)
    ikv.quant_load(cache, ikv.make_pool(k, v, 1, 4, 4, 128, 256, 0), sess, order, order)
    want = torch.from_numpy(eo.values(kc.cpu().numpy(), sc[..., 0, :].cpu().numpy())).to(_dt(dtype)).double()
    want[0, 255] = 0                                     # the sentinel of this cache is left out
    assert same(k.cpu().double(), want) and same(v.cpu().double(), want)


def test_new_rows_and_one_layer(dev):
    """A pool of new rows (no source list), into one layer of a larger cache, on another stream."""
    import torch
    L, Hkv, D, N = 3, 2, 128, 20
    k, v = torch.randn(L, N, Hkv, D, device=dev).bfloat16(), torch.randn(L, N, Hkv, D, device=dev).bfloat16()
    kc, vc, sc = empty_four(L, N + 1, Hkv, D, dev)
    sess, dst = sessions([N], dev), (1 + torch.arange(N, device=dev)).int()
    one = ikv.make_quant_pool(kc[1:2], vc[1:2], sc[1:2], 1, Hkv, Hkv, D, N + 1, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ikv.quant_store(one, ikv.make_pool(k[1:2], v[1:2], 1, Hkv, Hkv, D, N, 0), sess, None, dst, stream=side)
    side.synchronize()
    for codes, x, i in ((kc, k, 0), (vc, v, 1)):
        wc, ws = eo.quantise(x[1].double().cpu().numpy())
        assert np.array_equal(codes[1, 1:].cpu().numpy(), wc) and np.array_equal(sc[1, 1:, :, i].cpu().numpy(), ws)
        assert bool((codes[0] == 5).all()) and bool((codes[2] == 5).all()) and bool((codes[1, 0] == 5).all())
    assert bool((sc[0] == 77).all()) and bool((sc[2] == 77).all()) and bool((sc[1, 0] == 77).all())


def test_debug_mode_names_bad_rows(dev, monkeypatch):
    import torch
    monkeypatch.setenv("IKV_DEBUG", "1")
    L, Hkv, D, N = 1, 2, 64, 8
    k = torch.randn(L, N, Hkv, D, device=dev)
    kc, vc, sc = empty_four(L, N + 1, Hkv, D, dev)
    cache = ikv.make_quant_pool(kc, vc, sc, L, Hkv, Hkv, D, N + 1, 0)
    pool, sess = ikv.make_pool(k, k, L, Hkv, Hkv, D, N, 0), sessions([N], dev)
    dst = (1 + torch.arange(N, device=dev)).int()
    for at, value, msg in ((3, N + 1, r"dst\[3\]"), (5, 2, "listed twice")):
        bad = dst.clone()
        bad[at] = value
        with pytest.raises(ikv.IkvError, match=msg):
            ikv.quant_store(cache, pool, sess, None, bad)
    assert bool((kc == 5).all())
    ikv.quant_store(cache, pool, sess, None, dst)
    assert np.array_equal(kc[0, 1:].cpu().numpy(), eo.quantise(k[0].double().cpu().numpy())[0])

"""Rows into the 8-bit cache and back, bit for bit against the float64 oracle."""
import numpy as np
import pytest

from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv

pytestmark = pytest.mark.gpu


def _dt(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _code_type(code):
    import torch
    return torch.int8 if code == "int8" else torch.float8_e4m3fn


def sessions(lengths, dev, n=0):
    rows, o = [], 0
    for N in lengths:
        rows.append(dict(slot_off=o, mem_off=0, qspan_off=0, qpos_off=0, N=N, pi=0, qs=max(0, N - n), qe=N, C=N,
                         radix_prefix=0, R=1, nq=0))
        o += N
    return ikv.Sessions(rows, dev)


def empty_cache(code, L, slots, Hkv, D, dev, fill=5):
    import torch
    kc = torch.full((L, slots, Hkv, D), fill, dtype=torch.int8, device=dev).view(_code_type(code))
    return kc, kc.clone(), torch.full((L, slots, Hkv, 2), 0.25, device=dev)


def awkward_rows(L, slots, Hkv, D, dtype, dev, seed):
    """Rows with ties, zeros, tiny and huge values, infinities and NaN among ordinary ones."""
    import torch
    g = torch.Generator(device=dev).manual_seed(seed)
    x = torch.randn(L, slots, Hkv, D, generator=g, device=dev)
    kind = torch.randint(0, 12, (L, slots, Hkv, 1), generator=g, device=dev)
    x = torch.where(kind == 1, (x * 4).round() / 4, x)                       # few bits: ties
    x = torch.where(kind == 2, torch.zeros_like(x), x)
    x = torch.where(kind == 3, x * 2.0 ** -103, x)                           # at the least scale
    x = torch.where(kind == 4, x * 2.0 ** -130, x)                           # subnormal
    x = torch.where(kind == 5, x * 2.0 ** 124, x)
    x = torch.where(kind == 6, x * torch.exp(4 * torch.randn(D, generator=g, device=dev)), x)
    x[kind.expand_as(x) == 7] = x[kind.expand_as(x) == 7].sign() * 0.4375    # 448 * 2^-10
    x = x.to(_dt(dtype))
    first = torch.arange(D, device=dev) == D - 3
    x = torch.where((kind == 8) & first, torch.full_like(x, float("inf")), x)
    x = torch.where((kind == 9) & first, torch.full_like(x, float("nan")), x)
    return x


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,L,Hkv,D,lengths", [
    ("bf16", 1, 1, 64, [1]), ("bf16", 3, 8, 128, [37, 0, 5]), ("f32", 2, 2, 64, [33, 64]), ("f32", 1, 3, 128, [50]),
    ("bf16", 2, 3, 128, [129]), ("bf16", 5, 4, 64, [1, 1, 1, 1, 1, 1, 1])])
def test_store_and_load(dev, code, dtype, L, Hkv, D, lengths):
    import torch
    total = sum(lengths)
    pslots, cslots = 2 * total + 3, 3 * total + 2
    k, v = (awkward_rows(L, pslots, Hkv, D, dtype, dev, s) for s in (total, total + 1))
    kc, vc, sc = empty_cache(code, L, cslots, Hkv, D, dev)
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
        wc, ws = qo.quantise(x[:, from_.to(dev)].double().cpu().numpy(), code)
        got = codes.view(torch.uint8).cpu().numpy()
        full = np.full_like(got, 5)
        full[:, to.numpy()] = wc
        assert np.array_equal(got, full), name
        gs = sc[..., i].cpu().numpy()
        fs = np.full_like(gs, 0.25)
        fs[:, to.numpy()] = ws
        assert np.array_equal(gs, fs, equal_nan=True), name
        want[name] = (qo.code_values(wc, code).astype(np.float32) * ws[..., None]).astype(np.float32)
    # back, to rows of the pool's type; rows that are not listed stay
    k2, v2 = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    back = ikv.make_pool(k2, v2, L, Hkv, Hkv, D, pslots, 0)
    ikv.quant_load(cache, back, sess, dst.to(dev), src.to(dev), n_rows.to(dev))
    for name, x in (("k", k2), ("v", v2)):
        full = torch.full_like(x, 3.0).cpu()
        full[:, from_] = torch.from_numpy(want[name]).to(x.dtype)            # one rounding of the float32 product
        assert torch.equal(torch.nan_to_num(x.cpu(), nan=7.0), torch.nan_to_num(full, nan=7.0)), name
        assert torch.equal(x.cpu().isnan(), full.isnan()), name


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_identity_lists_and_all_rows(dev, code):
    import torch
    L, Hkv, D, N = 2, 2, 128, 70
    k = torch.randn(L, N + 4, Hkv, D, device=dev).bfloat16()
    v = torch.randn(L, N + 4, Hkv, D, device=dev).bfloat16()
    kc, vc, sc = empty_cache(code, L, N + 9, Hkv, D, dev)
    sess = sessions([N], dev)
    dst = (N + 8 - torch.arange(N, device=dev)).int()
    cache = ikv.make_quant_pool(kc, vc, sc, L, Hkv, Hkv, D, N + 9, 0)
    ikv.quant_store(cache, ikv.make_pool(k, v, L, Hkv, Hkv, D, N + 4, 0), sess, None, dst)
    wc, ws = qo.quantise(k[:, :N].double().cpu().numpy(), code)
    assert np.array_equal(kc.view(torch.uint8)[:, dst.long()].cpu().numpy(), wc)
    assert np.array_equal(sc[:, dst.long(), :, 0].cpu().numpy(), ws)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    ikv.quant_load(cache, ikv.make_pool(k2, v2, L, Hkv, Hkv, D, N + 4, 0), sess, dst)
    step = (k[:, :N].float().abs().amax(-1, keepdim=True) / 254 if code == "int8" else k[:, :N].float().abs() * 2.0 ** -4
            + sc[:, dst.long(), :, :1] * 2.0 ** -10)
    assert bool(((k2[:, :N].float() - k[:, :N].float()).abs() <= step * (1 + 2.0 ** -6) + k[:, :N].float().abs() * 2.0 ** -8).all())
    assert not k2[:, N:].any() and not v2[:, N:].any()


def test_one_layer_of_a_larger_cache(dev):
    import torch
    L, Hkv, D, N = 3, 2, 64, 20
    k = torch.randn(L, N, Hkv, D, device=dev)
    kc, vc, sc = empty_cache("int8", L, N + 1, Hkv, D, dev)
    sess, dst = sessions([N], dev), (1 + torch.arange(N, device=dev)).int()
    one = ikv.make_quant_pool(kc[1:2], vc[1:2], sc[1:2], 1, Hkv, Hkv, D, N + 1, 0)
    ikv.quant_store(one, ikv.make_pool(k[1:2], k[1:2], 1, Hkv, Hkv, D, N, 0), sess, None, dst)
    assert np.array_equal(kc[1, 1:].view(torch.uint8).cpu().numpy(), qo.quantise(k[1].double().cpu().numpy(), "int8")[0])
    assert bool((kc[0].view(torch.int8) == 5).all()) and bool((kc[2].view(torch.int8) == 5).all())
    assert bool((sc[0] == 0.25).all()) and bool((sc[2] == 0.25).all()) and bool((sc[1, 0] == 0.25).all())


def test_debug_mode_names_bad_rows(dev, monkeypatch):
    import torch
    monkeypatch.setenv("IKV_DEBUG", "1")
    L, Hkv, D, N = 1, 2, 64, 8
    k = torch.randn(L, N, Hkv, D, device=dev)
    kc, vc, sc = empty_cache("int8", L, N + 1, Hkv, D, dev)
    cache = ikv.make_quant_pool(kc, vc, sc, L, Hkv, Hkv, D, N + 1, 0)
    pool, sess = ikv.make_pool(k, k, L, Hkv, Hkv, D, N, 0), sessions([N], dev)
    dst = (1 + torch.arange(N, device=dev)).int()
    for at, value, msg in ((3, N + 1, r"dst\[3\]"), (0, -1, r"dst\[0\]"), (5, 2, "listed twice")):
        bad = dst.clone()
        bad[at] = value
        with pytest.raises(ikv.IkvError, match=msg) as e:
            ikv.quant_store(cache, pool, sess, None, bad)
        assert e.value.status == -1
    bad = (dst - 1).clone()
    bad[4] = N
    with pytest.raises(ikv.IkvError, match=r"src\[4\]"):
        ikv.quant_store(cache, pool, sess, bad, dst)
    with pytest.raises(ikv.IkvError, match="listed twice"):
        ikv.quant_load(cache, pool, sess, dst, torch.zeros_like(dst))
    assert bool((kc.view(torch.int8) == 5).all())
    two = dst.clone()
    two[:2] = 0                                          # the dead slot may be listed often
    ikv.quant_store(cache, pool, sess, None, two)
    ikv.quant_load(cache, pool, sess, two)
    torch.cuda.synchronize()
    assert not (kc.view(torch.int8)[0, 3:] == 5).all()

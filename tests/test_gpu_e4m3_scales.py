"""E4M3 rows whose scales are not powers of two, as another writer may hold them (max / 448, say): a
row stands for code * scale all the same, for one token and for chunks of any length.

The bound is that of tests/test_gpu_attend.py; where the chunk kernel has to round the products
code * scale to bf16 (each off by 2^-8 of itself), a logit moves by up to X 2^-8, which changes a
weight by exp(2 X 2^-8) - 1 at most once divided by their sum, and a value by 2^-8: A of both."""
import numpy as np
import pytest

from oracle import quant_oracle as qo
from test_gpu_attend import Setup

pytestmark = pytest.mark.gpu

# Hq, Hkv, D, N, tokens: one and two row blocks of a wave, 128 and 256 rows, several splits
FORMS = [(4, 2, 128, 300, 1), (4, 2, 64, 300, 3), (8, 2, 128, 300, 7), (4, 2, 128, 200, 20), (4, 1, 64, 500, 30),
         (4, 2, 128, 300, 150), (4, 1, 128, 1500, 70)]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D,N,n", FORMS)
@pytest.mark.parametrize("which", ["any", "few", "negative"])
def test_any_scale(dev, io, Hq, Hkv, D, N, n, which):
    import torch
    s = Setup(dev, "e4m3", io, 2, Hq, Hkv, D, [N], n, seed=N + n)
    g = torch.Generator(device=dev).manual_seed(n)
    by = 1 + 0.999 * torch.rand(s.sc.shape, generator=g, device=dev)
    if which == "few":                                   # a power of two in most rows
        by = torch.where(torch.rand(s.sc.shape, generator=g, device=dev) < 0.9, torch.ones_like(by), by)
    s.sc *= -by if which == "negative" else by
    q = s.queries(n, size=0.5)
    long = n * (Hq // Hkv) > (32 if io == "bf16" else 16)
    u, P = (2.0 ** -8, 2.0 ** -8 if long else 2.0 ** -17) if io == "bf16" else (2.0 ** -24, 2.0 ** -22)
    for sinks, window in ((0, 0), (3, 40)):
        out = s.run(q, sinks, window, decode=n == 1).view(2, Hq, n, D).double().cpu().numpy()
        for l in range(2):
            k, v = (s.rows(w, l, s.live.long()).double().cpu().numpy() for w in ("k", "v"))
            want, A, X = qo.attend(q.view(2, Hq, n, D)[l].double().cpu().numpy(), k, v, sinks, window)
            E = ((D + 8) * X + 4 * (1 + X) + N + 8) * 2.0 ** -24
            R = np.expm1(2 * X * 2.0 ** -8) + 2.0 ** -8 * np.exp(2 * X * 2.0 ** -8) if long else 0 * X
            tol = u * np.abs(want) + (P + 2 * E + R)[..., None] * A
            assert np.all(np.abs(out[l] - want) <= tol)


@pytest.mark.parametrize("n", [3, 50])
def test_the_exponent_alone_is_not_enough(dev, n):
    """One value scale of 1.75 among equal weights: half way to the next power."""
    import torch
    s = Setup(dev, "e4m3", "bf16", 1, 4, 1, 128, [100], n)
    s.k.view(torch.uint8)[:] = 0
    s.v.view(torch.uint8)[:] = 0x38                      # 1.0
    s.sc[:] = 1.75
    out = s.run(s.queries(n))
    assert bool((out == 1.75).all())


@pytest.mark.parametrize("n", [1, 3, 50])
def test_zero_and_tiny_scales(dev, n):
    import torch
    s = Setup(dev, "e4m3", "f32", 1, 4, 1, 128, [100], n)
    s.k.view(torch.uint8)[:] = 0
    s.v.view(torch.uint8)[:] = 0x38
    for scale in (0.0, 2.0 ** -126, 2.0 ** -120 * 1.5):
        s.sc[:] = scale
        out = s.run(s.queries(n), decode=n == 1)
        assert bool(((out - scale).abs() <= scale * 2.0 ** -16 + 2.0 ** -126).all())

"""Rows of the 8-bit cache that a token does not see add nothing to it, whatever bytes
and scales they hold: E4M3's NaN codes, codes whose product with the scale passes the largest
float, scales that are infinite of either sign. Tokens that see such a value row get what it
stands for.

Outputs of the tokens that see no changed row, and channels whose values did not change, have to
be the bytes of the run before the change: a row's own weights and sums do not depend on it."""
import pytest

from oracle import quant_oracle as qo
from test_gpu_attend import Setup

pytestmark = pytest.mark.gpu

SINKS, WINDOW = 2, 20
# (KV heads, heads per KV head, D, tokens) that one wave takes as one 16-row block, or two
FEW = [(2, 2, 128, 1), (2, 2, 128, 6), (1, 4, 64, 3)]
FEW_2 = [(2, 2, 128, 13), (1, 8, 64, 4)]
# blocks of 128 and of 256 rows
TILES = [(2, 2, 128, 50), (1, 4, 64, 30), (2, 2, 128, 140), (1, 4, 64, 300)]
FORMS = [(io, f) for io in ("bf16", "f32") for f in FEW + FEW_2 + TILES]


def _changed(N, n):
    """Entries before every window and after the sinks; one in the middle of the chunk, if it is long; the last."""
    return list(range(SINKS + 3, N - n - WINDOW)), ([N - n // 2] if n > 3 else []) + ([N - 1] if n > 1 else [])


def _runs(dev, code, io, form, change, N=500):
    """(output before, output after, tokens that see a changed value row), [heads, tokens, D]."""
    import torch
    Hkv, G, D, n = form
    s = Setup(dev, code, io, 1, Hkv * G, Hkv, D, [N], n)
    q = s.queries(n)
    run = lambda: s.run(q, SINKS, WINDOW, decode=n == 1).view(Hkv * G, n, D)  # noqa: E731
    clean = run()
    s.check(clean.flatten(), q, [n], SINKS, WINDOW)
    hidden, some = _changed(N, n)
    change(s, s.live.long()[hidden], s.live.long()[some])
    sees = torch.from_numpy(qo.seen(N, n, SINKS, WINDOW)[:, some].any(1)).to(dev)
    assert n == 1 or (bool(sees.any()) and not bool(sees.all()))
    return clean, run(), sees


@pytest.mark.parametrize("io,form", FORMS)
@pytest.mark.parametrize("byte", [0x7f, 0xff])
def test_nan_codes(dev, io, form, byte):
    import torch
    chan = [0, 5, form[2] - 1]

    def change(s, hidden, some):
        k, v = s.k.view(torch.uint8), s.v.view(torch.uint8)
        k[:, hidden] = byte
        v[:, hidden] = byte
        for c in chan:
            v[:, some, :, c] = byte

    clean, out, sees = _runs(dev, "e4m3", io, form, change)
    assert torch.equal(out[:, ~sees], clean[:, ~sees])
    spoiled = torch.zeros(form[2], dtype=torch.bool, device=dev)
    spoiled[chan] = True
    assert out[:, sees][..., spoiled].isnan().all()
    assert torch.equal(out[:, sees][..., ~spoiled], clean[:, sees][..., ~spoiled])


@pytest.mark.parametrize("io,form", FORMS)
def test_codes_past_the_largest_float(dev, io, form):
    # 256 * 2^120, as the store itself writes the top of the range, and 448 * 2^127
    import torch

    def change(s, hidden, some):
        for x, i in ((s.k, 0), (s.v, 1)):
            x.view(torch.uint8)[:, hidden] = 0x78
            s.sc[:, hidden, :, i] = 2.0 ** 120
            x.view(torch.uint8)[:, hidden[::2]] = 0xfe
            s.sc[:, hidden[::2], :, i] = 2.0 ** 127
        s.v.view(torch.uint8)[:, some] = 0x78
        s.sc[:, some, :, 1] = 2.0 ** 120

    clean, out, sees = _runs(dev, "e4m3", io, form, change)
    assert torch.equal(out[:, ~sees], clean[:, ~sees])
    assert not (out[:, sees].abs() < 2.0 ** 100).any()


@pytest.mark.parametrize("io,form", FORMS)
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("scale", [float("-inf"), float("inf"), float("nan")])
def test_scales_that_are_not_finite(dev, code, io, form, scale):
    import torch

    def change(s, hidden, some):
        s.sc[:, hidden] = scale
        s.sc[:, some, :, 1] = scale

    clean, out, sees = _runs(dev, code, io, form, change)
    assert torch.equal(out[:, ~sees], clean[:, ~sees])
    assert not torch.isfinite(out[:, sees]).any()

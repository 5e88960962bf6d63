"""4-bit values that stand for infinities (scale bytes 253 and 254, which another writer may use): a channel of a token
that sees one is that infinity, wherever in its list the entry lies (in a block that every token sees whole, or in
one that some token does not; first or last split), and nothing else changes. No logit here is far from the others,
so every weight is positive."""
import pytest

from four import Four
from test_gpu_e2m1_attend import FORMS

pytestmark = pytest.mark.gpu


def _put(s, entry, code, byte):
    """Channels 0 and 1 of the entry's value rows: this code; the rest of their block stands for zero."""
    slot = s.live.long()[entry]
    s.v[:, slot, :, 0] = code
    s.v[:, slot, :, 1:16] = 0
    s.sc[:, slot, :, 1, 0] = byte


@pytest.mark.parametrize("N,sinks,window", [(500, 0, 0), (2900, 0, 0), (2900, 4, 1500)])
@pytest.mark.parametrize("io,form", FORMS)
def test_seen_infinities(dev, io, form, N, sinks, window):
    import torch
    Hkv, G, D, n = form
    s = Four(dev, io, 1, Hkv * G, Hkv, D, [N], n, shared=True)
    s.sc[..., 0, :] = 125                                # keys below 1.5: no logit is far from another
    q = s.queries(n)
    run = lambda: s.run(q, sinks, window, decode=n == 1).view(Hkv * G, n, D)  # noqa: E731
    clean = run()
    v, sc = s.v.clone(), s.sc.clone()
    inf = float("inf")
    own = N - n + torch.arange(n, device=dev)
    def sees(e):
        return (e <= own) & ((window == 0) | (e < sinks) | (e > own - window))

    for entry in (3, 40, N // 2 + 7, N - n - 1, N - (n + 1) // 2, N - 1):
        if entry < 0:
            continue
        for code, byte, want in ((0x66, 253, inf), (0xff, 253, -inf), (0x44, 254, inf), (0xed, 254, -inf)):
            s.v.copy_(v)
            s.sc.copy_(sc)
            _put(s, entry, code, byte)
            out, see = run(), sees(entry)
            assert (out[:, see][..., :2] == want).all(), (entry, code)
            assert torch.equal(out[:, ~see], clean[:, ~see]) and torch.equal(out[..., 32:], clean[..., 32:]), (entry, code)
            assert out[..., 2:].isfinite().all()
    # both signs
    s.v.copy_(v)
    s.sc.copy_(sc)
    _put(s, 40, 0x66, 253)
    _put(s, N - n - 1 if N > n + 41 else 41, 0xee, 254)
    out, a, b = run(), sees(40), sees(N - n - 1 if N > n + 41 else 41)
    assert out[:, a & b][..., :2].isnan().all()
    assert (out[:, a & ~b][..., :2] == inf).all() and (out[:, ~a & b][..., :2] == -inf).all()
    assert torch.equal(out[..., 32:], clean[..., 32:])


@pytest.mark.parametrize("io,form", FORMS)
def test_nan_blocks_beside_infinite_ones(dev, io, form):
    """A block that stands for NaN, seen, is NaN on its channels however the blocks beside it are handled."""
    import torch
    Hkv, G, D, n = form
    s = Four(dev, io, 1, Hkv * G, Hkv, D, [700], n, shared=True)
    s.sc[..., 0, :] = 125
    q = s.queries(n)
    run = lambda: s.run(q, decode=n == 1).view(Hkv * G, n, D)  # noqa: E731
    clean = run()
    s.sc[:, s.live.long()[41], :, 1, 1] = 255            # channels 32 to 63
    out = run()
    assert out[..., 32:64].isnan().all() and torch.equal(out[..., :32], clean[..., :32])
    _put(s, 45, 0x66, 253)
    out = run()
    assert out[..., 32:64].isnan().all() and (out[..., :2] == float("inf")).all() and out[..., 2:32].isfinite().all()
    assert torch.equal(out[..., 64:], clean[..., 64:])

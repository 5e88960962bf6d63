"""Pins of the 4-bit rows' oracle: hand-worked blocks, every tie, the scale rule, blocks that are not finite."""
import numpy as np
import pytest

from oracle import e2m1_oracle as eo


def _one(block):
    x = np.zeros(32)
    x[:len(block)] = block
    codes, byte = eo.quantise(x[None])
    c = np.stack([codes[0] & 15, codes[0] >> 4], -1).reshape(-1)
    return c[:len(block)].tolist(), int(byte[0, 0])


def test_hand_worked_block():
    # largest 7: scale 1; ties 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5 go to the even code
    got = _one([7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5.01, 0.26, -0.25, 6, 0])
    assert got == ([7, 0, 2, 2, 4, 4, 6, 6, 15, 1, 8, 7, 0], 127)


@pytest.mark.parametrize("a,e", [(7.0, 0), (7.0000001, 1), (3.5, -1), (3.6, 0), (6.0, 0), (14.0, 1), (0.0, -102), (2.0 ** -100, -102),
                                 (2.0 ** 127, 125), (1.75 * 2.0 ** 127, 125), (3.3e38, 125), (2.0 ** -99, -101)])
def test_scale(a, e):
    assert _one([a])[1] == e + 127
    assert eo.scale_exponent(max(a, eo.LEAST)) == e
    assert 7 * 2.0 ** e >= max(a, eo.LEAST) or e == eo.MOST


def test_values_of_every_code():
    codes = np.arange(16, dtype=np.uint8)
    packed = np.concatenate([codes[0::2] | codes[1::2] << 4] * 2)
    v = eo.values(packed[None], np.array([[128]], np.uint8))[0]
    assert v[:8].tolist() == [0, 1, 2, 3, 4, 6, 8, 12] and v[8:16].tolist() == [-0.0, -1, -2, -3, -4, -6, -8, -12]
    assert np.signbit(v[8]) and v[16:].tolist() == v[:16].tolist()


def test_each_code_is_its_own_nearest():
    packed = np.arange(256, dtype=np.uint8)[None, None].repeat(2, 1).reshape(1, 512)
    v = eo.values(packed, np.full((1, 32), 100, np.uint8))
    codes, _ = eo.quantise(np.where(np.arange(1024) % 32 == 0, 7 * 2.0 ** -27, v))      # the scale's own largest value first
    keep = np.arange(512) % 16 != 0
    same = codes[0][keep] == packed[0][keep]
    assert same.all()


def test_nearest_by_brute_force():
    g = np.random.default_rng(5)
    x = g.standard_normal((200, 64)) * np.exp2(g.integers(-90, 90, (200, 1)))
    codes, byte = eo.quantise(x)
    v = eo.values(codes, byte)
    s = np.exp2(byte.astype(float) - 127).repeat(32, -1)
    best = np.abs(np.abs(x)[..., None] - eo.MAGNITUDES * s[..., None]).min(-1)
    assert np.array_equal(np.abs(np.abs(x) - np.abs(v)), best)
    assert np.all(np.abs(x - v) <= np.where(np.abs(x) >= s, np.abs(x) / 5, s / 4) * (1 + 2.0 ** -40))


def test_blocks_that_are_not_finite():
    x = np.ones((1, 128))
    x[0, 40], x[0, 100] = np.nan, -np.inf
    codes, byte = eo.quantise(x)
    assert byte[0].tolist() == [125, 255, 125, 255] and not codes[0, 16:32].any() and not codes[0, 48:].any()
    v = eo.values(codes, byte)
    assert np.array_equal(np.isnan(v[0]), np.repeat([False, True, False, True], 32)) and v[0, :32].tolist() == [1.0] * 32


@pytest.mark.parametrize("plant", ["up % 2 == 0|up % 2 == 1", "np.exp2(e - 1) >= a, e - 1, e)|np.exp2(e - 1) >= a, e - 1, e) + 1",
                                   "codes >> 4|codes >> 3", "np.signbit(x)|x > 0", "e + 127).astype|e + 126).astype",
                                   "np.minimum(e, MOST)|e", "np.maximum(np.abs(x).max(-1), LEAST)|np.abs(x).max(-1) + 1e-300",
                                   "[..., 1::2] << 4|[..., 0::2] << 4", "code | 8|code | 4"])
def test_pins_notice(plant):
    """A mistake planted in the oracle fails one of the pins above."""
    import inspect
    old, new = plant.split("|", 1) if plant != "code | 8|code | 4" else ("code | 8", "code | 4")
    src = inspect.getsource(eo)
    assert old in src
    space = {}
    exec(compile(src.replace(old, new), "planted", "exec"), space)
    kept = {k: getattr(eo, k) for k in ("quantise", "values")}
    failed = False
    try:
        for k in kept:
            setattr(eo, k, space[k])
        with np.errstate(all="ignore"):
            for pin in (test_hand_worked_block, test_values_of_every_code, test_nearest_by_brute_force,
                        test_blocks_that_are_not_finite, test_each_code_is_its_own_nearest,
                        lambda: [test_scale(a, e) for a, e in ((7.0, 0), (0.0, -102), (3.3e38, 125), (6.5, 0))]):
                try:
                    pin()
                except Exception:
                    failed = True
    finally:
        for k, f in kept.items():
            setattr(eo, k, f)
    assert failed

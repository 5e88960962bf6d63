"""Attention over the 4-bit cache (one token, a chunk), with windows and sinks, against the float64
oracle on the rows the cache stands for, within the bound that tests/test_gpu_attend.py derives."""
import numpy as np
import pytest

from attend_wide import CASES
from four import Four
from oracle import e2m1_oracle as eo
from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from test_attend_wide import cancelling
from test_gpu_attend import SHAPES
from test_gpu_quant_rows import sessions
from test_gpu_unseen_rows import FEW, FEW_2, TILES, SINKS, WINDOW, _changed

pytestmark = pytest.mark.gpu
IO = ["bf16", "f32"]


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("L,Hq,Hkv,D", SHAPES)
def test_decode(dev, io, L, Hq, Hkv, D):
    s = Four(dev, io, L, Hq, Hkv, D, [1, 33, 700, 64, 2], 1, seed=Hq)
    q = s.queries(5)
    for sinks, window in ((0, 0), (4, 50), (0, 1), (3, 1000), (100, 7)):
        s.check(s.run(q, sinks, window, decode=True), q, [1] * 5, sinks, window)


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("lengths", [[5000], [3000, 17, 1203], [2049] * 3])
def test_decode_long_lists(dev, io, lengths):
    s = Four(dev, io, 1, 8, 2, 128, lengths, 1, seed=len(lengths), heavy=True)
    q = s.queries(len(lengths), size=2.0)
    for sinks, window in ((0, 0), (4, 1024), (70, 129)):
        s.check(s.run(q, sinks, window, decode=True), q, [1] * len(lengths), sinks, window)


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("L,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("n", [2, 37])
def test_chunk(dev, io, L, Hq, Hkv, D, n):
    s = Four(dev, io, L, Hq, Hkv, D, [37, 130, 401], n, seed=Hq + n)
    q = s.queries(3 * n)
    for sinks, window in ((0, 0), (4, 50), (0, 1), (65, 63)):
        s.check(s.run(q, sinks, window), q, [n] * 3, sinks, window)


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("N,n", [(300, 300), (1111, 257), (2500, 64), (3000, 5)])
def test_chunk_sizes(dev, io, N, n):
    s = Four(dev, io, 1, 4, 1, 128, [N], n, seed=N, heavy=True)
    q = s.queries(n)
    for sinks, window in ((0, 0), (5, 200)):
        s.check(s.run(q, sinks, window), q, [n], sinks, window)


@pytest.mark.parametrize("L,Hq,Hkv", [(1, 4, 1), (2, 7, 1), (1, 24, 3), (3, 6, 3), (2, 8, 2), (40, 10, 5)])
@pytest.mark.parametrize("n", [1, 2, 4])
def test_short_lists_of_odd_and_even_heads(dev, L, Hq, Hkv, n):
    """One KV head a wave (odd numbers of them) or two, eight waves a head or four, 8, 16 and 32 rows."""
    s = Four(dev, "bf16", L, Hq, Hkv, 128, [400, 257, 300], n, seed=Hq + n)
    q = s.queries(3 * n)
    for sinks, window in ((0, 0), (3, 40)):
        s.check(s.run(q, sinks, window, decode=n == 1), q, [n] * 3, sinks, window)


@pytest.mark.parametrize("io", IO)
def test_ragged_chunks(dev, io):
    s = Four(dev, io, 2, 8, 2, 128, [1, 55, 0, 40], 40)
    q = s.queries(sum(s.ns))
    assert s.ns == [1, 40, 0, 40]
    for sinks, window in ((0, 0), (2, 9)):
        s.check(s.run(q, sinks, window), q, s.ns, sinks, window)


@pytest.mark.parametrize("n", [3, 30])
def test_lists_shorter_than_their_chunk(dev, n):
    s = Four(dev, "bf16", 1, 8, 2, 128, [50, 60, 70], n, n_live=[0, 2, 70])
    q = s.queries(3 * n)
    out = s.run(q, 1, 5)
    s.check(out, q, [n] * 3, 1, 5)
    per = out.numel() // 3
    assert not out[:per].any()                           # nothing to see: zeros
    assert not out[per:2 * per].view(8, n, 128)[:, :n - 2].any() and out[per:2 * per].view(8, n, 128)[:, n - 2:].any()
    d = s.queries(3, seed=9)
    got = s.run(d, decode=True)
    s.check(got, d, [1] * 3)
    assert not got[:got.numel() // 3].any()


FORMS = [(io, f) for io in IO for f in FEW + FEW_2 + TILES]


def _runs(dev, io, form, change, N=500):
    """(output before, output after, tokens that see a changed value row), [heads, tokens, D]."""
    import torch
    Hkv, G, D, n = form
    s = Four(dev, io, 1, Hkv * G, Hkv, D, [N], n)
    q = s.queries(n)
    run = lambda: s.run(q, SINKS, WINDOW, decode=n == 1).view(Hkv * G, n, D)  # noqa: E731
    clean = run()
    s.check(clean.flatten(), q, [n], SINKS, WINDOW)
    hidden, some = _changed(N, n)
    change(s, s.live.long()[hidden], s.live.long()[some])
    sees = torch.from_numpy(qo.seen(N, n, SINKS, WINDOW)[:, some].any(1)).to(dev)
    return clean, run(), sees


@pytest.mark.parametrize("io,form", FORMS)
def test_unseen_scales_of_nan(dev, io, form):
    """Blocks that stand for NaN: nothing to tokens that do not see them, NaN on their channels to those that do."""
    import torch
    block = form[2] // 32 - 1

    def change(s, hidden, some):
        s.sc[:, hidden] = 255
        s.sc[:, some, :, 1, block] = 255

    clean, out, sees = _runs(dev, io, form, change)
    assert torch.equal(out[:, ~sees], clean[:, ~sees])
    assert out[:, sees][..., 32 * block:].isnan().all()
    assert torch.equal(out[:, sees][..., :32 * block], clean[:, sees][..., :32 * block])


@pytest.mark.parametrize("io,form", FORMS)
def test_keys_of_nan(dev, io, form):
    """A key block that stands for NaN spoils the tokens that see it, and no others."""
    import torch

    def change(s, hidden, some):
        s.sc[:, some if len(some) else hidden, :, 0, 1] = 255

    clean, out, sees = _runs(dev, io, form, change)
    assert torch.equal(out[:, ~sees], clean[:, ~sees]) and out[:, sees].isnan().all()


@pytest.mark.parametrize("io,form", FORMS)
@pytest.mark.parametrize("byte,code", [(253, 0x66), (253, 0xff), (254, 0x44), (254, 0xdc)])
def test_unseen_values_past_the_largest_float(dev, io, form, byte, code):
    import torch

    def change(s, hidden, some):
        for x, i in ((s.k, 0), (s.v, 1)):
            x[:, hidden] = code
            s.sc[:, hidden, :, i] = byte
        s.v[:, some, :, 0] = code                        # channels 0 and 1; the block's others stand for zero
        s.v[:, some, :, 1:16] = 0
        s.sc[:, some, :, 1, 0] = byte

    clean, out, sees = _runs(dev, io, form, change)
    assert torch.equal(out[:, ~sees], clean[:, ~sees])
    assert not (out[:, sees][..., :2].abs() < 2.0 ** 100).any()
    assert torch.equal(out[:, sees][..., 32:], clean[:, sees][..., 32:])


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("n", [1, 3, 40])
def test_finite_values_beside_those_past_the_largest(dev, io, n):
    """A scale of 2^126 whose finite codes weigh as what they are, in a row that some token does not see. All
    logits are zero: every entry's weight is 1 / 90."""
    import torch
    N = 90
    s = Four(dev, io, 1, 4, 2, 64, [N], n)
    last = s.live.long()[N - 1]
    s.k[:] = 0
    s.sc[:, last, :, 1] = 253
    s.v[:, last] = 0x21                                  # 0.5 and 1 times 2^126
    q = s.queries(n)
    out = s.run(q, decode=n == 1).double().view(4, n, 32, 2)
    want = torch.tensor([2.0 ** 125, 2.0 ** 126], dtype=torch.float64, device=dev) / N
    assert ((out[:, n - 1] - want).abs() <= want * 2.0 ** -7).all() and (out[:, :n - 1].abs() < 2.0 ** 20).all()


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("n", [1, 50])
def test_logits_far_from_zero(dev, io, n):
    """Logits that rise, fall and jump by hundreds along the list."""
    import torch
    ramp = torch.linspace(-1, 1, 700, device=dev)
    for f in (ramp, -ramp, (ramp * 40).sin(), ramp * 0 - 1, ramp * 0 + 1):
        t = Four(dev, io, 1, 4, 1, 128, [700], n)
        q = t.queries(n)
        k = torch.zeros(1, t.slots, 1, 128, device=dev)
        k[0, t.live.long(), 0] = q.view(4, n, 128)[0, 0].float() * f[:, None] * 20
        t.k.copy_(t.fill(k, 0))
        t.check(t.run(q, decode=n == 1), q, [n])


@pytest.mark.parametrize("n", [1, 3, 40])
def test_small_and_large_scales(dev, n):
    """Rows at the ends of what the store writes: blocks of nearly nothing beside ordinary ones, huge values."""
    import torch
    s = Four(dev, "f32", 1, 4, 2, 128, [300], n)
    s.sc[..., 0, 1] = 25
    s.sc[..., 1, 2] = 25
    s.sc[..., 1, 3] = 220
    q = s.queries(n)
    s.check(s.run(q, 3, 100, decode=n == 1), q, [n], 3, 100)


def test_same_bytes_twice_and_on_another_stream(dev):
    import torch
    s = Four(dev, "bf16", 2, 8, 2, 128, [900, 300], 33)
    q = s.queries(66)
    a, b = s.run(q, 4, 128), s.run(q, 4, 128)
    assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = s.run(q, 4, 128, ws=ikv.Workspace(dev))
    side.synchronize()
    assert torch.equal(a, c)


def test_captured_and_replayed(dev):
    """A token's rows written and attended in a captured graph, replayed on changing inputs."""
    import torch
    N = 300
    s = Four(dev, "bf16", 2, 8, 2, 128, [N], 1)
    q = s.queries(1)
    out = torch.zeros_like(q)
    fresh = torch.zeros(2, 1, 2, 128, dtype=torch.bfloat16, device=dev)
    src = ikv.make_pool(fresh, fresh, 2, 8, 2, 128, 1, 0)
    one, dst = sessions([1], dev), s.live[N - 1:].clone()

    def step():
        ikv.quant_store(s.pool, src, one, None, dst)
        ikv.decode_attend_quant(s.pool, s.sess, q, s.live, s.nl, out, s.ws, sinks=3, window=200)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        fresh.copy_(torch.randn(2, 1, 2, 128, device=dev))
        q.copy_(s.queries(1, seed=20 + i))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
        s.check(out, q, [1], 3, 200)


def test_debug_mode_names_bad_entries(dev, monkeypatch):
    import torch
    s = Four(dev, "bf16", 1, 8, 2, 128, [40, 30], 3)
    q = s.queries(6)
    want = s.run(q)
    monkeypatch.setenv("IKV_DEBUG", "1")
    assert torch.equal(s.run(q), want)
    s.live[45] = s.slots
    for decode in (False, True):
        with pytest.raises(ikv.IkvError, match=r"session 1: live\[5\]"):
            s.run(s.queries(2) if decode else q, decode=decode)


@pytest.mark.parametrize("n,n_live", [(3, [0, 2, 200]), (60, [1, 59, 200])])
def test_the_largest_window_and_sinks(dev, n, n_live):
    s = Four(dev, "bf16", 1, 4, 1, 128, [200] * 3, n, n_live=n_live)
    q = s.queries(3 * n)
    big = 2 ** 31 - 1
    for sinks, window in ((0, big), (big, big), (big, 1), (0, 200)):
        s.check(s.run(q, sinks, window), q, [n] * 3, sinks, window)


@pytest.mark.parametrize("N,n", [(40, 2), (5000, 1), (5000, 6), (300, 90), (6000, 40)])
def test_a_query_that_is_not_finite_spoils_its_row_only(dev, N, n):
    import torch
    s = Four(dev, "bf16", 1, 4, 1, 128, [N], n)
    q = s.queries(n)
    clean = s.run(q).view(4, n, 128)
    for bad_value in (float("nan"), float("inf")):
        p = q.clone()
        p.view(4, n, 128)[2, n // 2, 7] = bad_value
        out = s.run(p).view(4, n, 128)
        bad = torch.zeros(4, n, dtype=torch.bool, device=dev)
        bad[2, n // 2] = True
        assert out[bad].isnan().all() and torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("D", [64, 128])
def test_one_layer_of_a_cache_with_an_odd_number_of_slots(dev, D):
    """Layers whose scales begin at any slot's alignment."""
    import torch
    s = Four(dev, "bf16", 3, 4, 1, D, [201], 9)
    assert s.slots % 2 == 1
    q = s.queries(9)
    out = s.run(q).view(3, -1)
    for l in range(3):
        one = ikv.make_quant_pool(s.k[l:l + 1], s.v[l:l + 1], s.sc[l:l + 1], 1, 4, 1, D, s.slots, 0)
        got = torch.empty_like(out[l])
        ikv.attend_chunk_quant(one, s.sess, q.view(3, -1)[l].clone(), s.live, s.nl, got, ikv.Workspace(dev))
        assert torch.equal(got, out[l])
        d = q.view(3, 4, 9, D)[l, :, 0].contiguous().flatten()
        one_out = torch.empty_like(d)
        ikv.decode_attend_quant(one, s.sess, d, s.live, s.nl, one_out, ikv.Workspace(dev))
        k, v = (s.rows(w, l, s.live.long()).numpy() for w in "kv")
        want, A, X = qo.attend(d.view(4, 1, D).double().cpu().numpy(), k, v)
        E = ((D + 8) * X + 4 * (1 + X) + 201 + 8) * 2.0 ** -24
        assert np.all(np.abs(one_out.view(4, 1, D).double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -17 + 2 * E[..., None]) * A)


@pytest.mark.parametrize("Hkv,D,slots", [(8, 128, 8_500_000), (1, 64, 17_000_000)])
def test_offsets_past_32_bits_and_many_slots(dev, Hkv, D, slots):
    """A layer of more than 4 GB, and more than 2^24 slots: rows at the far end."""
    import torch
    N, G = 700, 2
    s = Four(dev, "bf16", 1, G * Hkv, Hkv, D, [N], 40)
    far = s.live.clone()
    far[::2] = slots - 1 - far[::2]
    big = [torch.empty(1, slots, Hkv, D // 2, dtype=torch.uint8, device=dev) for _ in range(2)]
    for x, y in zip(big, (s.k, s.v)):
        x[0, far.long()] = y[0, s.live.long()]
    sc = torch.empty(1, slots, Hkv, 2, D // 32, dtype=torch.uint8, device=dev)
    sc[0, far.long()] = s.sc[0, s.live.long()]
    t = Four(dev, "bf16", 1, G * Hkv, Hkv, D, [N], 40)
    t.live = far
    t.pool = ikv.make_quant_pool(*big, sc, 1, G * Hkv, Hkv, D, slots, 0)
    t5, s5 = (sessions([N], dev, 5) for _ in range(2))
    for n, st, ss in ((40, t.sess, s.sess), (5, t5, s5)):
        t.sess, s.sess = st, ss
        q = s.queries(n)
        assert torch.equal(t.run(q, 3, 300), s.run(q, 3, 300))
    q = s.queries(1)
    assert torch.equal(t.run(q, decode=True), s.run(q, decode=True))
    # written and read back there
    k = torch.randn(1, N, Hkv, D, device=dev).bfloat16()
    ikv.quant_store(t.pool, ikv.make_pool(k, k, 1, Hkv, Hkv, D, N, 0), t.sess, None, far)
    back = torch.zeros_like(k)
    ikv.quant_load(t.pool, ikv.make_pool(back, back.clone(), 1, Hkv, Hkv, D, N, 0), t.sess, far)
    want = eo.values(*eo.quantise(k[0].double().cpu().numpy()))
    assert np.array_equal(back[0].double().cpu().numpy(), want)


WIDE = [(name, io) for name, c in CASES.items() if name != "chunk_bf16_parts2" for io in IO
        if (io == "f32") == ("f32" in name) or name in ("heads4_splits6", "heads2_parts4")]


@pytest.mark.parametrize("name,io", WIDE)
def test_forms(dev, name, io):
    """The launch forms of models' shapes, to the weights' own loss, and one layer at a time: another form."""
    import torch
    _, L, Hq, Hkv, D, tokens, lengths, sinks, window, _ = CASES[name]
    n = tokens or 1
    s = Four(dev, io, L, Hq, Hkv, D, lengths, n, seed=L + n, shared=True)
    q = s.queries(n * len(lengths))
    out = s.run(q, sinks, window, decode=tokens == 0)
    assert bool(torch.isfinite(out).all())
    s.bounds(out, q, n, sinks, window, sorted({0, 1, L // 2, L - 1}))
    size = L * Hq * n * D
    for l in {0, L - 1}:
        one = ikv.make_quant_pool(s.k[l:l + 1], s.v[l:l + 1], s.sc[l:l + 1], 1, Hq, Hkv, D, s.slots, 0, io_dtype=s.io_t)
        ql = torch.cat([q[b * size:(b + 1) * size].view(L, -1)[l] for b in range(len(lengths))])
        got = torch.empty_like(ql)
        f = ikv.decode_attend_quant if tokens == 0 else ikv.attend_chunk_quant
        f(one, s.sess, ql, s.live, s.nl, got, ikv.Workspace(dev), sinks=sinks, window=window)
        ol = torch.cat([out[b * size:(b + 1) * size].view(L, -1)[l] for b in range(len(lengths))])
        far = (got.float() - ol.float()).abs().max() / ol.float().abs().max()
        assert float(far) <= (2.0 ** -7 if io == "bf16" else 2.0 ** -12)


@pytest.mark.parametrize("io,Hq,Hkv,D,N,n", [(io, *p) for io in IO for p in ((8, 2, 128, 700, 1), (8, 2, 64, 90, 3), (4, 1, 128, 2100, 4))]
                         + [("bf16", 8, 1, 128, 400, 4)])
def test_weights_in_parts(dev, io, Hq, Hkv, D, N, n):
    """Weights half way between two bf16 numbers, values that cancel but for them."""
    import torch
    s = Four(dev, io, 1, Hq, Hkv, D, [N], n, seed=N, shared=True)
    q, k, v = cancelling(N, D)
    at = s.live.long()
    for x, i in ((k, 0), (v, 1)):
        t = torch.from_numpy(x).double()[:, None].expand(N, Hkv, D)
        c, sc = eo.quantise(t.numpy())
        (s.k, s.v)[i][0, at] = torch.from_numpy(c).to(dev)
        s.sc[0, at, :, i] = torch.from_numpy(sc).to(dev)
    qq = torch.from_numpy(q).to(s.io_t).to(dev).expand(Hq * n, D).reshape(-1).contiguous()
    s.bounds(s.run(qq, decode=n == 1), qq, n, 0, 0, [0])

"""Attention over the 8-bit cache (one token, a chunk) and of a chunk over a bf16 pool, with
windows and sinks, against the float64 oracle on the rows the cache stands for.

The bound, per output: with u the half step of the output's type (bf16 2^-8, float32 2^-24),
A = sum_j w_j |v_j| over the entries seen (w the softmax weights) and X the largest
sum_d |q_d k_d| / sqrt(D) of them,
  |out - exact| <= u |exact| + (P + 2 E) A,
E the relative error of a float32 weight: the logit's sum of D products and its scaling,
(D + 8) 2^-24 X, the exponential and its argument, 4 * 2^-24 (1 + X); the same again for the
sum of weights, whose N terms add (N + 8) 2^-24; P what a weight loses where it is rounded for
the matrix cores: 2^-8 (bf16) for bf16 outputs, 2^-22 (three bf16 parts) for float32 ones."""
import numpy as np
import pytest

from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from test_gpu_quant_rows import _code_type, sessions

pytestmark = pytest.mark.gpu


class Setup:
    """A cache or pool, sessions' lists and queries; `rows(l)` what layer l's rows stand for."""

    def __init__(self, dev, code, io, L, Hq, Hkv, D, lengths, n, n_live=None, seed=1, heavy=False):
        import torch
        self.code, self.io, self.L, self.Hq, self.Hkv, self.D, self.n, self.dev = code, io, L, Hq, Hkv, D, n, dev
        g = torch.Generator(device=dev).manual_seed(seed)
        rn = lambda *z: torch.randn(*z, generator=g, device=dev)  # noqa: E731
        total = sum(lengths)
        self.slots = 2 * total + 5
        k = rn(L, self.slots, Hkv, D) * torch.exp(0.5 * rn(D)) * (1 + 3 * heavy * (rn(self.slots, 1, 1) > 1.5))
        v = (rn(L, self.slots, Hkv, D) + rn(D)) * torch.exp(rn(self.slots, 1, 1))
        self.live = (1 + torch.randperm(self.slots - 1, generator=g, device=dev)[:total]).int()
        self.lengths, self.n_live = lengths, list(lengths) if n_live is None else n_live
        self.nl = torch.tensor(self.n_live, dtype=torch.int32, device=dev)
        self.sess = sessions(lengths, dev, n)
        self.ns = [min(n, N) for N in lengths]           # sessions() clamps the span to the list
        self.io_t = torch.bfloat16 if io == "bf16" else torch.float32
        if code == "bf16":
            self.k, self.v = k.bfloat16(), v.bfloat16()
        else:
            self.k, self.v, self.sc = (torch.zeros(z, device=dev) for z in (1, 1, (L, self.slots, Hkv, 2)))
            parts = []
            for i, x in ((0, k), (1, v)):
                c, s = qo.quantise(x.double().cpu().numpy(), code)
                parts.append(torch.from_numpy(c).to(dev).view(_code_type(code)))
                self.sc[..., i] = torch.from_numpy(s).to(dev)
            self.k, self.v = parts
        self.ws = ikv.Workspace(dev)
        self.desc()

    def desc(self):
        a = (self.L, self.Hq, self.Hkv, self.D, self.slots, 0)
        self.pool = (ikv.make_pool(self.k, self.v, *a) if self.code == "bf16" else
                     ikv.make_quant_pool(self.k, self.v, self.sc, *a, io_dtype=self.io_t))

    def queries(self, tokens, seed=2, size=1.0):
        import torch
        g = torch.Generator(device=self.dev).manual_seed(seed)
        return (torch.randn(tokens * self.L * self.Hq * self.D, generator=g, device=self.dev) * size).to(self.io_t)

    def rows(self, which, l, slots):
        x = getattr(self, which)[l][slots] if self.code == "bf16" else self._codes(which, l, slots)
        return x

    def _codes(self, which, l, slots):
        import torch
        c = getattr(self, which)[l].view(torch.uint8)[slots].cpu().numpy()
        s = self.sc[l][slots][..., 0 if which == "k" else 1].double().cpu().numpy()
        return torch.from_numpy(qo.code_values(c, self.code) * s[..., None])

    def check(self, out, q, ns, sinks=0, window=0):
        """Every output against the oracle; returns the largest error in units of its bound."""
        import torch
        u, P = (2.0 ** -8, 2.0 ** -8) if self.io == "bf16" else (2.0 ** -24, 2.0 ** -22)
        D, worst, o, at = self.D, 0.0, 0, 0
        assert bool(torch.isfinite(out).all())
        for N0, N, n in zip(self.lengths, self.n_live, ns):
            slots = self.live[o:o + N].long()
            o += N0
            sh = (self.L, self.Hq, n, D)
            sz = self.L * self.Hq * n * D
            qq, got = q[at:at + sz].view(sh).double().cpu().numpy(), out[at:at + sz].view(sh).double().cpu().numpy()
            at += sz
            for l in range(self.L):
                k, v = (self.rows(w, l, slots).double().cpu().numpy() for w in ("k", "v"))
                want, A, X = qo.attend(qq[l], k, v, sinks, window)
                E = ((D + 8) * X + 4 * (1 + X) + N + 8) * 2.0 ** -24
                tol = u * np.abs(want) + (P + 2 * E[..., None]) * A
                err = np.abs(got[l] - want)
                bad = err > tol
                assert not bad.any(), (f"{int(bad.sum())} of {bad.size} outputs out of bound, the worst "
                                       f"{np.nanmax(np.where(tol > 0, err / np.maximum(tol, 1e-300), 0)):.2f} times it")
                worst = max(worst, float(np.max(err / np.maximum(tol, 1e-300), initial=0.0)))
        return worst

    def run(self, q, sinks=0, window=0, decode=False, ws=None):
        import torch
        out = torch.full_like(q, 9.0)
        f = (ikv.decode_attend_quant if decode else ikv.attend_chunk if self.code == "bf16" else ikv.attend_chunk_quant)
        f(self.pool, self.sess, q, self.live, self.nl, out, ws or self.ws, sinks=sinks, window=window)
        return out


SHAPES = [(1, 1, 1, 64), (2, 8, 2, 64), (1, 8, 1, 128), (2, 10, 2, 128), (1, 12, 4, 128), (1, 24, 8, 64), (1, 6, 2, 128),
          (1, 7, 1, 128), (1, 4, 4, 128)]
IO = [("int8", "bf16"), ("e4m3", "bf16"), ("int8", "f32"), ("e4m3", "f32")]


@pytest.mark.parametrize("code,io", IO)
@pytest.mark.parametrize("L,Hq,Hkv,D", SHAPES)
def test_decode(dev, code, io, L, Hq, Hkv, D):
    s = Setup(dev, code, io, L, Hq, Hkv, D, [1, 33, 700, 64, 2], 1, seed=Hq)
    q = s.queries(5)
    for sinks, window in ((0, 0), (4, 50), (0, 1), (3, 1000), (100, 7)):
        s.check(s.run(q, sinks, window, decode=True), q, [1] * 5, sinks, window)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("lengths", [[5000], [3000, 17, 1203], [2049] * 3])
def test_decode_long_lists(dev, code, lengths):
    s = Setup(dev, code, "bf16", 1, 8, 2, 128, lengths, 1, seed=len(lengths), heavy=True)
    q = s.queries(len(lengths), size=2.0)
    for sinks, window in ((0, 0), (4, 1024), (70, 129)):
        s.check(s.run(q, sinks, window, decode=True), q, [1] * len(lengths), sinks, window)


@pytest.mark.parametrize("code,io", IO + [("bf16", "bf16")])
@pytest.mark.parametrize("L,Hq,Hkv,D", SHAPES)
@pytest.mark.parametrize("n", [2, 37])
def test_chunk(dev, code, io, L, Hq, Hkv, D, n):
    s = Setup(dev, code, io, L, Hq, Hkv, D, [37, 130, 401], n, seed=Hq + n)
    q = s.queries(3 * n)
    for sinks, window in ((0, 0), (4, 50), (0, 1), (65, 63)):
        s.check(s.run(q, sinks, window), q, [n] * 3, sinks, window)


@pytest.mark.parametrize("code,io", IO + [("bf16", "bf16")])
@pytest.mark.parametrize("N,n", [(300, 300), (1111, 257), (2500, 64), (3000, 5)])
def test_chunk_sizes(dev, code, io, N, n):
    s = Setup(dev, code, io, 1, 4, 1, 128, [N], n, seed=N, heavy=True)
    q = s.queries(n)
    for sinks, window in ((0, 0), (5, 200)):
        s.check(s.run(q, sinks, window), q, [n], sinks, window)


@pytest.mark.parametrize("code", ["int8", "bf16"])
def test_ragged_chunks(dev, code):
    # sessions() takes one n, clamped to each list: chunks of 1, 40, 0 and 40 tokens
    s = Setup(dev, code, "bf16", 2, 8, 2, 128, [1, 55, 0, 40], 40)
    q = s.queries(sum(s.ns))
    assert s.ns == [1, 40, 0, 40]
    for sinks, window in ((0, 0), (2, 9)):
        s.check(s.run(q, sinks, window), q, s.ns, sinks, window)


@pytest.mark.parametrize("code", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("n", [3, 30])
def test_lists_shorter_than_their_chunk(dev, code, n):
    s = Setup(dev, code, "bf16", 1, 8, 2, 128, [50, 60, 70], n, n_live=[0, 2, 70])
    q = s.queries(3 * n)
    out = s.run(q, 1, 5)
    s.check(out, q, [n] * 3, 1, 5)
    per = out.numel() // 3
    assert not out[:per].any()                           # nothing to see: zeros
    assert not out[per:2 * per].view(8, n, 128)[:, :n - 2].any() and out[per:2 * per].view(8, n, 128)[:, n - 2:].any()
    if code != "bf16":
        d = s.queries(3, seed=9)
        got = s.run(d, decode=True)
        s.check(got, d, [1] * 3)
        assert not got[:got.numel() // 3].any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n", [3, 40, 300])
def test_unseen_rows_may_hold_anything_bf16(dev, n, bad):
    N, w = 500, 20
    s = Setup(dev, "bf16", "bf16", 1, 4, 2, 128, [N], n)
    q = s.queries(n)
    clean = s.run(q, 2, w)
    slots = s.live.long()
    last = slots[N - 1]
    s.v[:, last] = bad                                   # seen by the last token only
    s.v[:, slots[5:N - n - w]] = bad                     # before every window, after the sinks
    s.k[:, slots[5:N - n - w]] = bad
    out = s.run(q, 2, w).view(4, n, 128)
    import torch
    assert torch.equal(out[:, :n - 1], clean.view(4, n, 128)[:, :n - 1])
    assert not torch.isfinite(out[:, n - 1]).any()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("n", [1, 3, 40, 300])
def test_unseen_rows_may_hold_anything_quant(dev, code, n):
    import torch
    N, w = 500, 20
    s = Setup(dev, code, "bf16", 1, 4, 2, 128, [N], n)
    q = s.queries(n)
    clean = s.run(q, 2, w, decode=n == 1)
    slots = s.live.long()
    s.sc[:, slots[5:N - n - w]] = float("nan")
    if n > 1:
        s.sc[:, slots[N - 1], :, 1] = float("nan")
    out = s.run(q, 2, w, decode=n == 1)
    if n == 1:
        assert torch.equal(out, clean)
    else:
        out = out.view(4, n, 128)
        assert torch.equal(out[:, :n - 1], clean.view(4, n, 128)[:, :n - 1])
        assert out[:, n - 1].isnan().all()


@pytest.mark.parametrize("code,io", [("int8", "f32"), ("e4m3", "bf16")])
@pytest.mark.parametrize("n", [1, 50])
def test_logits_far_from_zero(dev, code, io, n):
    """Logits that rise, fall and jump by hundreds along the list."""
    import torch
    s = Setup(dev, code, io, 1, 4, 1, 128, [700], n)
    ramp = torch.linspace(-1, 1, 700, device=dev)
    q = s.queries(n)
    for f in (ramp, -ramp, (ramp * 40).sin(), ramp * 0 - 1, ramp * 0 + 1):
        t = Setup(dev, code, io, 1, 4, 1, 128, [700], n)
        k = torch.zeros(1, t.slots, 1, 128, device=dev)
        k[0, t.live.long(), 0] = q.view(4, n, 128)[0, 0].float() * f[:, None] * 20
        c, sc = qo.quantise(k.double().cpu().numpy(), code)
        t.k.view(torch.uint8).copy_(torch.from_numpy(c).to(dev))
        t.sc[..., 0] = torch.from_numpy(sc).to(dev)
        t.check(t.run(q, decode=n == 1), q, [n])


@pytest.mark.parametrize("code", ["int8", "bf16"])
def test_same_bytes_twice_and_on_another_stream(dev, code):
    import torch
    s = Setup(dev, code, "bf16", 2, 8, 2, 128, [900, 300], 33)
    q = s.queries(66)
    a, b = s.run(q, 4, 128), s.run(q, 4, 128)
    assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = s.run(q, 4, 128, ws=ikv.Workspace(dev))
    side.synchronize()
    assert torch.equal(a, c)


@pytest.mark.parametrize("code", ["e4m3", "bf16"])
def test_captured_and_replayed(dev, code):
    """A token's rows written and attended in a captured graph, replayed on changing inputs."""
    import torch
    N = 300
    s = Setup(dev, code, "bf16", 2, 8, 2, 128, [N], 1)
    q = s.queries(1)
    out = torch.zeros_like(q)
    fresh = torch.zeros(2, 1, 2, 128, dtype=torch.bfloat16, device=dev)
    src = ikv.make_pool(fresh, fresh, 2, 8, 2, 128, 1, 0)
    one, dst = sessions([1], dev), s.live[N - 1:].clone()

    def step():
        if code == "bf16":
            s.k[:, dst.long()] = fresh
            ikv.attend_chunk(s.pool, s.sess, q, s.live, s.nl, out, s.ws, sinks=3, window=200)
        else:
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
    s = Setup(dev, "int8", "bf16", 1, 8, 2, 128, [40, 30], 3)
    q = s.queries(6)
    want = s.run(q)
    monkeypatch.setenv("IKV_DEBUG", "1")
    assert torch.equal(s.run(q), want)
    s.live[45] = s.slots
    with pytest.raises(ikv.IkvError, match=r"session 1: live\[5\]"):
        s.run(q)
    with pytest.raises(ikv.IkvError, match=r"session 1: live\[5\]"):
        s.run(s.queries(2), decode=True)


@pytest.mark.parametrize("code", ["int8", "bf16"])
@pytest.mark.parametrize("n,n_live", [(3, [0, 2, 200]), (60, [1, 59, 200])])
def test_the_largest_window_and_sinks(dev, code, n, n_live):
    s = Setup(dev, code, "bf16", 1, 4, 1, 128, [200] * 3, n, n_live=n_live)
    q = s.queries(3 * n)
    big = 2 ** 31 - 1
    for sinks, window in ((0, big), (big, big), (big, 1), (0, 200)):
        s.check(s.run(q, sinks, window), q, [n] * 3, sinks, window)


@pytest.mark.parametrize("code", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("N,n", [(40, 2), (5000, 1), (5000, 6), (300, 90), (6000, 40)])
def test_a_query_that_is_not_finite_spoils_its_row_only(dev, code, N, n):
    import torch
    s = Setup(dev, code, "bf16", 1, 4, 1, 128, [N], n)
    q = s.queries(n)
    clean = s.run(q).view(4, n, 128)
    q.view(4, n, 128)[2, n // 2, 7] = float("nan")
    out = s.run(q).view(4, n, 128)
    bad = torch.zeros(4, n, dtype=torch.bool, device=dev)
    bad[2, n // 2] = True
    assert out[bad].isnan().all() and torch.equal(out[~bad], clean[~bad])


@pytest.mark.parametrize("code,Hkv,D,slots", [("int8", 8, 128, 4_300_000), ("bf16", 8, 128, 2_200_000),
                                              ("e4m3", 1, 64, 17_000_000)])
def test_offsets_past_32_bits_and_many_slots(dev, code, Hkv, D, slots):
    """A layer of more than 4 GB, and more than 2^24 slots: rows at the far end."""
    import torch
    N, G = 700, 2
    s = Setup(dev, code, "bf16", 1, G * Hkv, Hkv, D, [N], 40)
    far = s.live.clone()
    far[::2] = slots - 1 - far[::2]
    big = [torch.empty(1, slots, Hkv, D, dtype=s.k.dtype, device=dev) for _ in range(2)]
    for x, y in zip(big, (s.k, s.v)):
        raw = torch.int16 if code == "bf16" else torch.int8
        x.view(raw)[0, far.long()] = y.view(raw)[0, s.live.long()]
    a = (1, G * Hkv, Hkv, D, slots, 0)
    if code != "bf16":
        sc = torch.empty(1, slots, Hkv, 2, device=dev)
        sc[0, far.long()] = s.sc[0, s.live.long()]
    t = Setup(dev, code, "bf16", 1, G * Hkv, Hkv, D, [N], 40)
    t.live = far
    t.pool = ikv.make_pool(*big, *a) if code == "bf16" else ikv.make_quant_pool(*big, sc, *a)
    t5, s5 = (sessions([N], dev, 5) for _ in range(2))
    for n, st, ss in ((40, t.sess, s.sess), (5, t5, s5)):
        t.sess, s.sess = st, ss
        q = s.queries(n)
        assert torch.equal(t.run(q, 3, 300), s.run(q, 3, 300))
    if code == "bf16":
        return
    q = s.queries(1)
    assert torch.equal(t.run(q, decode=True), s.run(q, decode=True))
    # written and read back there
    k = torch.randn(1, N, Hkv, D, device=dev).bfloat16()
    rows = ikv.make_pool(k, k, 1, Hkv, Hkv, D, N, 0)
    ikv.quant_store(t.pool, rows, t.sess, None, far)
    back = torch.zeros_like(k)
    ikv.quant_load(t.pool, ikv.make_pool(back, back.clone(), 1, Hkv, Hkv, D, N, 0), t.sess, far)
    c, w = qo.quantise(k[0].double().cpu().numpy(), code)
    want = torch.from_numpy(qo.code_values(c, code).astype(np.float32) * w[..., None]).bfloat16()
    assert torch.equal(back[0].cpu(), want)


@pytest.mark.parametrize("N,m,n", [(400, 97, 2), (400, 160, 20), (500, 130, 70), (3000, 1600, 3), (3000, 1600, 40)])
def test_keys_of_minus_infinity(dev, N, m, n):
    # the oldest m entries have the logit -inf in every row: as if they were not in the list
    import torch
    s = Setup(dev, "bf16", "bf16", 1, 4, 1, 128, [N], n, seed=N + n)
    s.k[0, s.live[:m].long(), 0, 0] = float("-inf")
    q = s.queries(n)
    q.view(-1, 128)[:, 0] = q.view(-1, 128)[:, 0].abs() + 0.5
    out = s.run(q)
    s.live, s.lengths, s.n_live = s.live[m:], [N - m], [N - m]
    s.check(out, q, [n])


@pytest.mark.parametrize("N,n", [(3, 2), (90, 90), (2000, 2)])
def test_rows_of_minus_infinity_alone(dev, N, n):
    # a softmax over nothing but -inf is NaN; a token that sees no entry at all stays zero
    import torch
    s = Setup(dev, "bf16", "bf16", 1, 4, 1, 64, [N], n, seed=N)
    s.k[..., 0] = float("-inf")
    q = s.queries(n)
    q.view(-1, 64)[:, 0] = q.view(-1, 64)[:, 0].abs() + 0.5
    assert s.run(q).isnan().all()
    s.nl.fill_(1)
    out = s.run(q).view(4, n, 64)
    assert out[:, :n - 1].eq(0).all() and out[:, n - 1].isnan().all()

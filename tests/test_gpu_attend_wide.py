"""Few-row attention in the launch forms that models' shapes take: waves of adjacent KV heads in a
workgroup, with and without waves that share a head's entries, with and without splits; one and two
16-row blocks. And the few-row kernels' weights: two bf16 parts for bf16 outputs, three for float32.

The bound is that of tests/test_gpu_attend.py with P, what a weight loses, as these kernels have it:
2^-17 relative (the second part is off by half a step of at most 2^-8 of the weight, which lies in
[2^-9, 2^-8) times its power of two: 2^-17), 2^-25 with three parts."""
import numpy as np
import pytest

from attend_wide import CASES, PARAMS
from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from test_attend_wide import cancelling
from test_gpu_attend import Setup
from test_gpu_quant_rows import _code_type, sessions

pytestmark = pytest.mark.gpu


class Wide(Setup):
    """A cache or pool that all sessions list slots of, filled with codes as they come."""

    def __init__(self, dev, code, io, L, Hq, Hkv, D, lengths, n, seed):
        import torch
        self.code, self.io, self.L, self.Hq, self.Hkv, self.D, self.n, self.dev = code, io, L, Hq, Hkv, D, n, dev
        g = torch.Generator(device=dev).manual_seed(seed)
        self.slots = max(lengths) + 9
        self.live = torch.cat([1 + torch.randperm(self.slots - 1, generator=g, device=dev)[:N] for N in lengths]).int()
        self.lengths = self.n_live = lengths
        self.nl = torch.tensor(lengths, dtype=torch.int32, device=dev)
        self.sess, self.ns = sessions(lengths, dev, n), [n] * len(lengths)
        self.io_t = torch.bfloat16 if io == "bf16" else torch.float32
        shape = (L, self.slots, Hkv, D)
        rows = lambda: torch.randn(shape, generator=g, device=dev)  # noqa: E731
        if code == "bf16":
            self.k, self.v = rows().bfloat16(), (rows() + 0.5).bfloat16()
        else:
            as_code = {"int8": lambda x: (x * 40).round().clamp(-127, 127).to(torch.int8),
                       "e4m3": lambda x: (x * 60).clamp(-448, 448).to(_code_type(code))}[code]
            self.k, self.v = as_code(rows()), as_code(rows() + 0.5)
            self.sc = torch.exp2(torch.randint(-7, -4, (L, self.slots, Hkv, 2), generator=g, device=dev).float())
            if code == "int8":
                self.sc *= 1 + torch.rand(self.sc.shape, generator=g, device=dev)
        self.ws = ikv.Workspace(dev)
        self.desc()

    def bounds(self, out, q, n, sinks, window, layers):
        """Outputs of these layers against the oracle, the bound with this kernel's P."""
        u, P = (2.0 ** -8, 2.0 ** -17) if self.io == "bf16" else (2.0 ** -24, 2.0 ** -25)
        o, size = 0, self.L * self.Hq * n * self.D
        for b, N in enumerate(self.lengths):
            slots = self.live[o:o + N].long()
            o += N
            qq, got = (x[b * size:(b + 1) * size].view(self.L, self.Hq, n, self.D) for x in (q, out))
            for l in layers:
                k, v = (self.rows(w, l, slots).double().cpu().numpy() for w in ("k", "v"))
                want, A, X = qo.attend(qq[l].double().cpu().numpy(), k, v, sinks, window)
                E = ((self.D + 8) * X + 4 * (1 + X) + N + 8) * 2.0 ** -24
                tol = u * np.abs(want) + (P + 2 * E[..., None]) * A
                bad = np.abs(got[l].double().cpu().numpy() - want) > tol
                assert not bad.any(), f"session {b}, layer {l}: {int(bad.sum())} of {bad.size} out of bound"


@pytest.mark.parametrize("name,code,io", PARAMS)
def test_forms(dev, name, code, io):
    import torch
    _, L, Hq, Hkv, D, tokens, lengths, sinks, window, _ = CASES[name]
    n = tokens or 1
    s = Wide(dev, code, io, L, Hq, Hkv, D, lengths, n, seed=L + n)
    q = s.queries(n * len(lengths))
    out = s.run(q, sinks, window, decode=tokens == 0)
    assert bool(torch.isfinite(out).all())
    s.bounds(out, q, n, sinks, window, sorted({0, 1, L // 2, L - 1}))
    # every layer and head against the same call on one layer at a time: another form of the same sums
    size = L * Hq * n * D
    for l in {0, L - 1}:
        a = (1, Hq, Hkv, D, s.slots, 0)
        one = (ikv.make_pool(s.k[l:l + 1], s.v[l:l + 1], *a) if code == "bf16" else
               ikv.make_quant_pool(s.k[l:l + 1], s.v[l:l + 1], s.sc[l:l + 1], *a, io_dtype=s.io_t))
        ql = torch.cat([q[b * size:(b + 1) * size].view(L, -1)[l] for b in range(len(lengths))])
        got = torch.empty_like(ql)
        f = ikv.decode_attend_quant if tokens == 0 else ikv.attend_chunk if code == "bf16" else ikv.attend_chunk_quant
        f(one, s.sess, ql, s.live, s.nl, got, ikv.Workspace(dev), sinks=sinks, window=window)
        ol = torch.cat([out[b * size:(b + 1) * size].view(L, -1)[l] for b in range(len(lengths))])
        far = (got.float() - ol.float()).abs().max() / ol.float().abs().max()
        assert float(far) <= (2.0 ** -7 if io == "bf16" else 2.0 ** -12)


PARTS = [(8, 2, 128, 700, 1), (8, 2, 64, 90, 3), (4, 1, 128, 2100, 4)]
PARTS = [(code, io, *p) for code, io in (("int8", "bf16"), ("e4m3", "bf16"), ("bf16", "bf16"), ("int8", "f32"), ("e4m3", "f32"))
         for p in PARTS] + [(code, "bf16", 8, 1, 128, 400, 4) for code in ("int8", "e4m3")]


@pytest.mark.parametrize("code,io,Hq,Hkv,D,N,n", PARTS)
def test_weights_in_parts(dev, code, io, Hq, Hkv, D, N, n):
    """Weights half way between two bf16 numbers, values that cancel but for them."""
    import torch
    s = Wide(dev, code, io, 1, Hq, Hkv, D, [N], n, seed=N)
    q, k, v = cancelling(N, D)
    at = s.live.long()
    for x, i in ((k, 0), (v, 1)):
        t = torch.from_numpy(x).to(dev)[:, None].expand(N, Hkv, D)
        if code == "bf16":
            (s.k, s.v)[i][0, at] = t.bfloat16()
        else:
            c, sc = qo.quantise(t.cpu().numpy(), code)
            (s.k, s.v)[i].view(torch.uint8)[0, at] = torch.from_numpy(c).to(dev)
            s.sc[0, at, :, i] = torch.from_numpy(sc).to(dev)
    qq = torch.from_numpy(q).to(s.io_t).to(dev).expand(Hq * n, D).reshape(-1).contiguous()
    out = s.run(qq, decode=n == 1 and code != "bf16")
    s.bounds(out, qq, n, 0, 0, [0])

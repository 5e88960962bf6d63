"""A 4-bit cache with sessions' lists and queries, checked as tests/test_gpu_attend.py checks the 8-bit
ones."""
import numpy as np

from oracle import e2m1_oracle as eo
from oracle import quant_oracle as qo
from paper_2606_09916_amd import ikv
from test_gpu_attend import Setup
from test_gpu_quant_rows import sessions


class Four(Setup):
    def __init__(self, dev, io, L, Hq, Hkv, D, lengths, n, n_live=None, seed=1, heavy=False, shared=False):
        """shared: all sessions list slots of one cache, filled with codes as they come."""
        import torch
        self.code, self.io, self.L, self.Hq, self.Hkv, self.D, self.n, self.dev = "e2m1", io, L, Hq, Hkv, D, n, dev
        g = torch.Generator(device=dev).manual_seed(seed)
        rn = lambda *z: torch.randn(*z, generator=g, device=dev)  # noqa: E731
        total = sum(lengths)
        self.slots = max(lengths) + 9 if shared else 2 * total + 5
        if shared:
            byte = lambda lo, hi, *z: torch.randint(lo, hi, z, generator=g, device=dev, dtype=torch.uint8)  # noqa: E731
            self.k, self.v = (byte(0, 256, L, self.slots, Hkv, D // 2) for _ in range(2))
            self.sc = byte(124, 128, L, self.slots, Hkv, 2, D // 32)
            self.live = torch.cat([1 + torch.randperm(self.slots - 1, generator=g, device=dev)[:N] for N in lengths]).int()
        else:
            k = rn(L, self.slots, Hkv, D) * torch.exp(0.5 * rn(D)) * (1 + 3 * heavy * (rn(self.slots, 1, 1) > 1.5))
            v = (rn(L, self.slots, Hkv, D) + rn(D)) * torch.exp(rn(self.slots, 1, 1))
            self.sc = torch.zeros(L, self.slots, Hkv, 2, D // 32, dtype=torch.uint8, device=dev)
            self.k, self.v = (self.fill(x, i) for i, x in enumerate((k, v)))
            self.live = (1 + torch.randperm(self.slots - 1, generator=g, device=dev)[:total]).int()
        self.lengths, self.n_live = lengths, list(lengths) if n_live is None else n_live
        self.nl = torch.tensor(self.n_live, dtype=torch.int32, device=dev)
        self.sess = sessions(lengths, dev, n)
        self.ns = [x.qe - x.qs for x in self.sess.host[:len(lengths)]]
        self.io_t = torch.bfloat16 if io == "bf16" else torch.float32
        self.ws = ikv.Workspace(dev)
        self.desc()

    def fill(self, x, i):
        """The codes of rows x [L, slots, Hkv, D]; their scales go to sc as those of keys (0) or values (1)."""
        import torch
        c, s = eo.quantise(x.double().cpu().numpy())
        self.sc[..., i, :] = torch.from_numpy(s).to(self.dev)
        return torch.from_numpy(c).to(self.dev)

    def _codes(self, which, l, slots):
        import torch
        c = getattr(self, which)[l][slots].cpu().numpy()
        return torch.from_numpy(eo.values(c, self.sc[l][slots][..., "kv".index(which), :].cpu().numpy()))

    def bounds(self, out, q, n, sinks, window, layers):
        """Outputs of these layers against the oracle, weights in two bf16 parts (bf16 outputs) or three: off by
        2^-17 or 2^-25 of them."""
        u, P = (2.0 ** -8, 2.0 ** -17) if self.io == "bf16" else (2.0 ** -24, 2.0 ** -25)
        o, size = 0, self.L * self.Hq * n * self.D
        for b, N in enumerate(self.lengths):
            slots = self.live[o:o + N].long()
            o += N
            qq, got = (x[b * size:(b + 1) * size].view(self.L, self.Hq, n, self.D) for x in (q, out))
            for l in layers:
                k, v = (self.rows(w, l, slots).numpy() for w in "kv")
                want, A, X = qo.attend(qq[l].double().cpu().numpy(), k, v, sinks, window)
                E = ((self.D + 8) * X + 4 * (1 + X) + N + 8) * 2.0 ** -24
                tol = u * np.abs(want) + (P + 2 * E[..., None]) * A
                bad = np.abs(got[l].double().cpu().numpy() - want) > tol
                assert not bad.any(), f"session {b}, layer {l}: {int(bad.sum())} of {bad.size} out of bound"

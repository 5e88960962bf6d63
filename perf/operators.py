"""Workloads for the 8-bit cache and the attention that reads it: what a serving stack has
them do, through the public entry points of ``paper_2606_09916_amd.ikv``.

``listed()`` names the cases, ``draw(rng)`` gives one more of the same ranges,
``prepare(case, seed)`` makes what a caller holds on the GPU, ``run(state)`` is one pass,
``work(case)`` the bytes and operations that a pass cannot do without, and
``exact(case, seed)`` the results in 64 bits. With ``own`` false, ``run`` computes the same
in elementary torch operations.

The operators, on rows x of D channels (one per layer, slot and KV head), with
a = max(max|x|, 2^-100) over the row:
  int8   scale = a / 127, code = x / (a / 127) to the nearest whole number, ties to even;
  e4m3   scale = the smallest power of two s with 448 s >= a, code = the e4m3 value nearest
         x / s, ties to even;
  a row stands for code * scale.
Attention of token t of a session's n newest over its list of live slots (N entries, the n
newest last), own entry i = N - n + t: entry j is seen if j <= i and, where there is a
window, j < sinks or j > i - window;
  out = sum_j softmax_j(q . k_j / sqrt(D)) v_j over the entries seen.

Kinds of pass:
  round   quantise rows of a pool into the 8-bit cache, then read them back into a pool
  load    read rows of the 8-bit cache back
  decode  attention of one new token per session over the 8-bit cache
  chunk   attention of a chunk of new tokens over the 8-bit cache or a bf16 pool

Shapes are those of the repository's configurations: Qwen3-8B (36 layers, 32 query and 8 KV
heads), Qwen2.5-14B (48, 40, 8), one GPU's half of a Qwen2.5-14B tensor-parallel pair (48,
20, 4), all D = 128 in bf16, and the small float32 layers (1 or 2 layers, 8 query and 2 KV
heads, D = 64). Pages of 16 slots are dealt from a shuffle; key channels are of uneven size,
some rows are heavy, values have a mean per channel.
"""
import math

import torch

own = False

PAGE = 16
LEAST = 2.0 ** -100

QWEN3_8B = dict(L=36, Hq=32, Hkv=8, D=128, dtype="bf16")
QWEN25_14B = dict(L=48, Hq=40, Hkv=8, D=128, dtype="bf16")
QWEN25_14B_HALF = dict(L=48, Hq=20, Hkv=4, D=128, dtype="bf16")
SMALL_F32 = dict(L=1, Hq=8, Hkv=2, D=64, dtype="f32")
SMALL_F32_2 = dict(L=2, Hq=8, Hkv=2, D=64, dtype="f32")


def _case(kind, shape, **kw):
    c = dict(kind=kind, **shape, code="int8", B=1, n=1, sinks=0, window=0)
    c.update(kw)
    c.setdefault("Nmin", c["N"])         # shortest session of a batch; N is the longest
    return c


def listed():
    return [
        # a few rows of a small float32 layer: launches only
        _case("round", SMALL_F32, name="round_small_f32", N=67),
        # the newest token of each of 16 sessions, written and read back
        _case("round", QWEN3_8B, name="round_8b_16_tokens", B=16, N=1),
        # what a retention event keeps of a session, moved into the 8-bit cache and checked
        _case("round", QWEN3_8B, name="round_8b_8k", N=8192, code="e4m3"),
        # a turn's rows read back for the scorer
        _case("load", QWEN25_14B_HALF, name="load_half14b_1021", N=1021, code="e4m3"),
        # two whole histories read back for a retention event
        _case("load", QWEN3_8B, name="load_8b_2_sessions", B=2, N=8000, Nmin=5501),
        # one decode step of small float32 layers
        _case("decode", SMALL_F32_2, name="decode_small_f32", N=300),
        # one decode step after a retention event: single session, and ragged ones with a window
        _case("decode", QWEN3_8B, name="decode_8b_8k", N=8192),
        _case("decode", QWEN25_14B_HALF, name="decode_half14b_16_sessions", B=16, N=12011, Nmin=517, code="e4m3",
              sinks=4, window=4096),
        # a decode step over the longest history, nothing dropped
        _case("decode", QWEN25_14B, name="decode_14b_92k", N=92300),
        # a handful of proposed tokens checked at once
        _case("chunk", QWEN25_14B_HALF, name="chunk_half14b_3_tokens", B=4, N=2500, Nmin=700, n=3, code="e4m3"),
        # a tool's output read into a kept history
        _case("chunk", QWEN3_8B, name="chunk_8b_509_of_8k", N=8701, n=509),
        # a long prompt's chunk in the bf16 pool, window and sinks
        _case("chunk", QWEN25_14B, name="chunk_14b_1024_bf16", N=9216, n=1024, code="bf16", sinks=4, window=4096),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["round", "load", "decode", "decode", "chunk", "chunk"])
    code = rng.choice(["int8", "e4m3"])
    if rng.random() < 0.2:               # small float32 layers
        shape = rng.choice([SMALL_F32, SMALL_F32_2])
        B, hi = rng.choice([1, 2, 3]), 4096
    else:
        shape = rng.choice([QWEN3_8B, QWEN25_14B, QWEN25_14B_HALF])
        B = rng.choice([1, 1, 2, 5, 16])
        hi = {"round": 8192, "load": 12000, "decode": 49152, "chunk": 8000}[kind] // B
    N = _log_uniform(rng, 1 if kind in ("round", "load") else 40, hi)
    kw = dict(B=B, N=N, Nmin=max(1, N // rng.choice([1, 2, 4])), code=code)
    if kind in ("decode", "chunk") and rng.random() < 0.5:
        kw.update(sinks=rng.choice([0, 1, 4, 64]), window=_log_uniform(rng, 1, N))
    if kind == "chunk":
        kw["n"] = _log_uniform(rng, 1, min(kw["Nmin"], 512 // B))
        if shape["dtype"] == "bf16" and rng.random() < 0.4:
            kw["code"] = "bf16"
    return _case(kind, shape, **kw)


# ----------------------------------------------------------------------------- sizes

def _lengths(c):
    """Entries of each session's list: the first the longest, the others unevenly spread."""
    lo, hi = c["Nmin"], c["N"]
    return [hi - int(round((hi - lo) * ((b * 0.6180339887498949) % 1.0))) for b in range(c["B"])]


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def work(case):
    c, es, D, units = case, 2 if case["dtype"] == "bf16" else 4, case["D"], case["L"] * case["Hkv"]
    row = 2 * D * es if c["code"] == "bf16" else 2 * D + 8       # K and V of one entry and head
    by = fl = 0.0
    for N in _lengths(c):
        if c["kind"] in ("round", "load"):
            by += N * units * (row + 2 * D * es) + 4 * N
            by += N * units * (2 * D * es + row) + 4 * N if c["kind"] == "round" else 0
            fl += 2.0 * N * units * D * (2 if c["kind"] == "round" else 1)
            continue
        n, seen, pairs = c["n"], N, 0
        for t in range(n):
            i = N - n + t
            pairs += i + 1 if not c["window"] else min(i + 1, c["window"] + min(c["sinks"], max(0, i + 1 - c["window"])))
        if c["window"]:
            lo = max(0, N - n - c["window"] + 1)
            seen = N - lo + min(c["sinks"], lo)
        by += seen * (units * row + 4) + 2 * n * c["L"] * c["Hq"] * D * es
        fl += 4.0 * pairs * c["L"] * c["Hq"] * D
    return {"bytes": float(by), "flops": float(fl)}


# ----------------------------------------------------------------------------- inputs

def _quantise(x, code):
    """Codes and scales of rows x [..., D] (float32), in 64 bits next to the borders."""
    x = x.double()
    a = x.abs().amax(-1, keepdim=True).clamp_min(LEAST)
    if code == "int8":
        return (x * 127 / a).round().to(torch.int8), (a / 127).float()
    m, e = torch.frexp(a / 448)                      # a / 448 = m 2^e, 0.5 <= m < 1
    e = torch.where(m == 0.5, e - 1, e).long()
    s = ((e + 1023) << 52).view(torch.float64)       # 2^e, bit for bit
    return (x / s).float().to(torch.float8_e4m3fn), s.float()


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 29)
    randn = lambda *z: torch.randn(*z, generator=gen, device=dev)  # noqa: E731
    L, Hq, Hkv, D, dt, kind = c["L"], c["Hq"], c["Hkv"], c["D"], _type(c), c["kind"]
    Ns = _lengths(c)
    st = dict(case=c, Ns=Ns)

    # each session's list of slots: pages dealt from a shuffle; slot 0 is the sentinel
    pages = [-(-N // PAGE) for N in Ns]
    order = torch.randperm(sum(pages), generator=gen, device=dev)
    lists, p = [], 0
    for N, np_ in zip(Ns, pages):
        j = torch.arange(N, device=dev)
        lists.append(1 + order[p:p + np_][j // PAGE] * PAGE + j % PAGE)
        p += np_
    num_slots, total = 1 + sum(pages) * PAGE, sum(Ns)
    st.update(num_slots=num_slots, total=total, live=torch.cat(lists).to(torch.int32),
              n_live=torch.tensor(Ns, dtype=torch.int32, device=dev))

    chan, mean = torch.exp(0.4 * randn(L, 1, Hkv, D)), randn(L, 1, Hkv, D)
    size = torch.ones(num_slots, 1, 1, device=dev)
    size[torch.randperm(num_slots, generator=gen, device=dev)[:num_slots // 20]] = 3.0
    rows = lambda l: ((randn(num_slots, Hkv, D) * chan[l] * size).to(dt),  # noqa: E731
                      (randn(num_slots, Hkv, D) + mean[l]).to(dt))
    if kind == "round" or c["code"] == "bf16":        # rows of a pool
        st["k"], st["v"] = (torch.zeros(L, num_slots, Hkv, D, dtype=dt, device=dev) for _ in range(2))
        for l in range(L):
            st["k"][l], st["v"][l] = rows(l)
    if c["code"] != "bf16":                           # the 8-bit cache, written already unless the pass writes it
        ct = torch.int8 if c["code"] == "int8" else torch.float8_e4m3fn
        st["kc"], st["vc"] = (torch.zeros(L, num_slots, Hkv, D, dtype=torch.int8, device=dev).view(ct) for _ in range(2))
        st["scales"] = torch.ones(L, num_slots, Hkv, 2, device=dev)
        if kind != "round":
            for l in range(L):
                for codes, x, i in zip(("kc", "vc"), rows(l), (0, 1)):
                    q, s = _quantise(x.float(), c["code"])
                    st[codes][l].view(torch.int8).copy_(q.view(torch.int8))
                    st["scales"][l, :, :, i] = s[..., 0]
    if kind in ("round", "load"):                     # where the rows are read back to
        st["k_out"], st["v_out"] = (torch.zeros(L, total, Hkv, D, dtype=dt, device=dev) for _ in range(2))
    else:                                             # packed by session: [L][Hq][n][D]
        st["q"] = randn(len(Ns) * L * Hq * c["n"] * D).to(dt)
        st["out"] = torch.zeros_like(st["q"])
    if own:
        st.update(_handles(st))
    torch.cuda.synchronize()
    return st


def _handles(st):
    """The descriptors and the workspace that a caller of the library keeps."""
    from paper_2606_09916_amd import ikv
    c, dev, h = st["case"], st["live"].device, {}
    L, Hq, Hkv, D = c["L"], c["Hq"], c["Hkv"], c["D"]
    rows, o = [], 0
    for N in st["Ns"]:
        rows.append(dict(slot_off=o, mem_off=0, qspan_off=0, qpos_off=0, N=N, pi=0, qs=N - c["n"], qe=N, C=N,
                         radix_prefix=0, R=1, nq=0))
        o += N
    h["sess"], h["ws"] = ikv.Sessions(rows, dev), ikv.Workspace(dev)
    if "k" in st:
        h["pool"] = ikv.make_pool(st["k"], st["v"], L, Hq, Hkv, D, st["num_slots"], 0)
    if "kc" in st:
        h["qpool"] = ikv.make_quant_pool(st["kc"], st["vc"], st["scales"], L, Hq, Hkv, D, st["num_slots"], 0,
                                         io_dtype=_type(c))
    if "k_out" in st:
        h["back"] = ikv.make_pool(st["k_out"], st["v_out"], L, Hq, Hkv, D, st["total"], 0)
    return h


# ----------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    from paper_2606_09916_amd import ikv
    c = st["case"]
    if c["kind"] in ("round", "load"):
        if c["kind"] == "round":
            ikv.quant_store(st["qpool"], st["pool"], st["sess"], st["live"], st["live"], st["n_live"])
        ikv.quant_load(st["qpool"], st["back"], st["sess"], st["live"], None, st["n_live"])
        return [st["k_out"], st["v_out"]]
    if c["kind"] == "decode":
        ikv.decode_attend_quant(st["qpool"], st["sess"], st["q"], st["live"], st["n_live"], st["out"], st["ws"],
                                sinks=c["sinks"], window=c["window"])
    elif c["code"] == "bf16":
        ikv.attend_chunk(st["pool"], st["sess"], st["q"], st["live"], st["n_live"], st["out"], st["ws"],
                         sinks=c["sinks"], window=c["window"])
    else:
        ikv.attend_chunk_quant(st["qpool"], st["sess"], st["q"], st["live"], st["n_live"], st["out"], st["ws"],
                               sinks=c["sinks"], window=c["window"])
    return [st["out"]]


def _plain_rows(st, which, layers, slots):
    """float32 rows [layers, len(slots), Hkv, D] that the cache holds at these slots."""
    c = st["case"]
    if c["code"] == "bf16":
        return st[which][layers][:, slots].float()
    codes, scale = st[which + "c"][layers], st["scales"][layers][:, slots, :, 0 if which == "k" else 1]
    return codes.view(torch.int8)[:, slots].view(codes.dtype).float() * scale[..., None]


def _run_plain(st):
    c, every = st["case"], slice(None)
    slots = st["live"].long()
    if c["kind"] in ("round", "load"):
        if c["kind"] == "round":
            for which, i in (("k", 0), ("v", 1)):
                q, s = _quantise(st[which][:, slots].float(), c["code"])
                st[which + "c"].view(torch.int8)[:, slots] = q.view(torch.int8)
                st["scales"][:, slots, :, i] = s[..., 0]
        st["k_out"].copy_(_plain_rows(st, "k", every, slots))
        st["v_out"].copy_(_plain_rows(st, "v", every, slots))
        return [st["k_out"], st["v_out"]]
    L, Hq, Hkv, D, n = c["L"], c["Hq"], c["Hkv"], c["D"], c["n"]
    G, o, done = Hq // Hkv, 0, 0
    for N in st["Ns"]:
        mine = slots[o:o + N]
        o += N
        span = slice(done, done + L * Hq * n * D)
        done = span.stop
        q = st["q"][span].view(L, Hkv, G * n, D).float()
        own_i = N - n + torch.arange(n, device=q.device)[:, None]
        j = torch.arange(N, device=q.device)[None]
        hidden = j > own_i
        if c["window"]:
            hidden = hidden | ((j >= c["sinks"]) & (j <= own_i - c["window"]))
        hidden = hidden.repeat(G, 1)
        at_once = max(1, min(L, 2 ** 30 // (N * Hkv * max(D, G * n))))
        for l in range(0, L, at_once):
            layers = slice(l, l + at_once)
            k = _plain_rows(st, "k", layers, mine).permute(0, 2, 3, 1).contiguous()
            x = torch.matmul(q[layers], k).mul_(1.0 / math.sqrt(D)).masked_fill_(hidden, -math.inf)
            w = x.sub_(x.amax(-1, keepdim=True)).exp_()
            v = _plain_rows(st, "v", layers, mine).transpose(1, 2).contiguous()
            st["out"][span].view(L, Hkv, G * n, D)[layers] = torch.matmul(w, v).div_(w.sum(-1, keepdim=True))
    return [st["out"]]


# ----------------------------------------------------------------------------- 64 bits

def _stands_for(x, code):
    """What rows x (float64) stand for once quantised."""
    a = x.abs().max(-1, keepdim=True).values.clamp(min=LEAST)
    if code == "int8":
        step = a / 127
        return torch.round(x / a * 127) * step
    powers = torch.tensor([2.0 ** e for e in range(-120, 130)], dtype=torch.float64, device=x.device)
    s = powers[torch.searchsorted(powers * 448, a)]              # the first that holds a
    r = x / s
    step = powers[torch.searchsorted(powers, r.abs().clamp(min=2.0 ** -6), right=True) - 1] / 8
    return torch.round(r / step) * step * s


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    L, Hq, Hkv, D, n = c["L"], c["Hq"], c["Hkv"], c["D"], c["n"]

    def held(which, l, at):
        if c["code"] == "bf16":
            return st[which][l][at].double()
        if c["kind"] == "round":
            return _stands_for(st[which][l][at].double(), c["code"])
        codes = st[which + "c"][l].float().double()[at]
        return codes * st["scales"][l][at][:, :, "kv".index(which)].double().unsqueeze(-1)

    at = st["live"].long()
    if c["kind"] in ("round", "load"):
        return [torch.stack([held(w, l, at) for l in range(L)]) for w in "kv"]
    parts, o, done = [], 0, 0
    for N in st["Ns"]:
        q = st["q"][done:done + L * Hq * n * D].view(L, Hq, n, D).double()
        done += q.numel()
        i = torch.arange(N - n, N, device=at.device)
        j = torch.arange(N, device=at.device)
        seen = j[None, :] <= i[:, None]
        if c["window"] > 0:
            seen &= (j[None, :] < c["sinks"]) | (i[:, None] - j[None, :] < c["window"])
        out = torch.zeros_like(q)
        for l in range(L):
            k, v = held("k", l, at[o:o + N]), held("v", l, at[o:o + N])
            for h in range(Hq):
                g = h // (Hq // Hkv)
                logit = (q[l, h] @ k[:, g].T) / D ** 0.5
                top = torch.where(seen, logit, -math.inf).max(1, keepdim=True).values
                e = torch.where(seen, torch.exp(logit - top), 0.0)
                out[l, h] = (e @ v[:, g]) / e.sum(1, keepdim=True)
        o += N
        parts.append(out.reshape(-1))
    return [torch.cat(parts)]

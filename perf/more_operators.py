"""Workloads for the 4-bit cache, the attention that reads it, and the slots of new tokens:
what a serving stack has them do, through the public entry points of
``paper_2606_09916_amd.ikv``.

``listed()`` names the cases, ``draw(rng)`` gives one more of the same ranges,
``prepare(case, seed)`` makes what a caller holds on the GPU, ``run(state)`` is one pass,
``work(case)`` the bytes and operations that a pass cannot do without, and
``exact(case, seed)`` the results in 64 bits. With ``own`` false, ``run`` computes the same
in elementary torch operations.

The 4-bit cache holds a row of D channels (one per layer, slot and KV head) in blocks of 32:
a scale, a power of two, as one byte e for 2^(e - 127), and 32 codes, two a byte, the lower
channel in the lower half. A code is a sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6. With
a = max(max|x|, 2^-100) over the block:
  scale  the least power of two s with 7 s >= a, at most 2^125;
  code   the value nearest x / s, ties to the even code (0, 1, 2 or 4 of two neighbours),
         6 past 5.
Attention of token t of a session's n newest over its list of live slots (N entries, the n
newest last), own entry i = N - n + t: entry j is seen if j <= i and, where there is a
window, j < sinks or j > i - window;
  out = sum_j softmax_j(q . k_j / sqrt(D)) v_j over the entries seen.
Slots: a stack of free ones. Returning pushes the sessions' lists, in order. Taking serves
sessions in order, as long as the stack holds enough for all up to them (and a session's list
has room); the T slots of all tokens served are the topmost T, in the stack's order.

Kinds of pass:
  round   quantise rows of a pool into the 4-bit cache, then read them back into a pool
  load    read rows of the 4-bit cache back
  decode  attention of one new token per session over the 4-bit cache
  chunk   attention of a chunk of new tokens over the 4-bit cache
  slots   return the slots that a retention event freed, then take those of the new tokens
          (as many): into the slot maps, behind the live lists, and as a list for the store

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
BLOCK = 32
LEAST = 2.0 ** -100
MOST = 2.0 ** 125

QWEN3_8B = dict(L=36, Hq=32, Hkv=8, D=128, dtype="bf16")
QWEN25_14B = dict(L=48, Hq=40, Hkv=8, D=128, dtype="bf16")
QWEN25_14B_HALF = dict(L=48, Hq=20, Hkv=4, D=128, dtype="bf16")
SMALL_F32 = dict(L=1, Hq=8, Hkv=2, D=64, dtype="f32")
SMALL_F32_2 = dict(L=2, Hq=8, Hkv=2, D=64, dtype="f32")


def _case(kind, shape, **kw):
    c = dict(kind=kind, **shape, B=1, n=1, sinks=0, window=0)
    c.update(kw)
    c.setdefault("Nmin", c["N"])         # shortest session of a batch; N is the longest
    return c


def _slots(**kw):
    """N: history and new tokens of the longest session, n: its new tokens; nmin: the fewest. padded: every third
    session of the batch is idle, and the tokens of each are counted on the GPU."""
    c = dict(kind="slots", B=1, padded=False)
    c.update(kw)
    c.setdefault("nmin", c["n"])
    return c


def listed():
    return [
        # a few rows of a small float32 layer: launches only
        _case("round", SMALL_F32, name="round_small_f32", N=45),
        # what a retention event keeps of a session, moved into the 4-bit cache and checked
        _case("round", QWEN3_8B, name="round_8b_8k", N=8189),
        # two histories read back for a retention event
        _case("load", QWEN25_14B_HALF, name="load_half14b_2_sessions", B=2, N=7000, Nmin=2501),
        # one decode step of small float32 layers
        _case("decode", SMALL_F32_2, name="decode_small_f32", N=411),
        # one decode step after a retention event: single session, and ragged ones with a window
        _case("decode", QWEN3_8B, name="decode_8b_8k", N=8201),
        _case("decode", QWEN25_14B_HALF, name="decode_half14b_16_sessions", B=16, N=12007, Nmin=613, sinks=4,
              window=4096),
        # a decode step over the longest history, nothing dropped
        _case("decode", QWEN25_14B, name="decode_14b_92k", N=92300),
        # a handful of proposed tokens checked at once
        _case("chunk", QWEN25_14B_HALF, name="chunk_half14b_4_tokens", B=4, N=3100, Nmin=800, n=4),
        # a user's message read into a kept history
        _case("chunk", QWEN3_8B, name="chunk_8b_61_of_8k", N=8253, n=61),
        # a long prompt's chunk, window and sinks
        _case("chunk", QWEN25_14B, name="chunk_14b_1021_window", N=9213, n=1021, sinks=4, window=4096),
        # a decode step of a padded batch: a slot for each session that is not idle
        _slots(name="slots_64_sessions_token", B=64, N=8201, n=1, padded=True),
        # 64 whole histories admitted into a full pool
        _slots(name="slots_64_histories", B=64, N=36000, n=36000, nmin=30011),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["round", "load", "decode", "decode", "chunk", "chunk", "slots"])
    if kind == "slots":
        B = _log_uniform(rng, 1, 256)
        n = _log_uniform(rng, 1, 2000000 // B)
        return _slots(B=B, n=n, nmin=max(1, n // rng.choice([1, 2, 4])), N=n + _log_uniform(rng, 1, 1 + 2000000 // B),
                      padded=rng.random() < 0.5)
    if rng.random() < 0.2:               # small float32 layers
        shape = rng.choice([SMALL_F32, SMALL_F32_2])
        B, hi = rng.choice([1, 2, 3]), 4096
    else:
        shape = rng.choice([QWEN3_8B, QWEN25_14B, QWEN25_14B_HALF])
        B = rng.choice([1, 1, 2, 5, 16])
        hi = {"round": 8000, "load": 12000, "decode": 49152, "chunk": 8000}[kind] // B
    N = _log_uniform(rng, 1 if kind in ("round", "load") else 40, hi)
    kw = dict(B=B, N=N, Nmin=max(1, N // rng.choice([1, 2, 4])))
    if kind in ("decode", "chunk") and rng.random() < 0.5:
        kw.update(sinks=rng.choice([0, 1, 4, 64]), window=_log_uniform(rng, 1, N))
    if kind == "chunk":
        kw["n"] = _log_uniform(rng, 1, min(kw["Nmin"], 512 // B))
    return _case(kind, shape, **kw)


# ----------------------------------------------------------------------------- sizes

def _spread(lo, hi, B):
    """B lengths: the first the longest, the others unevenly spread."""
    return [hi - int(round((hi - lo) * ((b * 0.6180339887498949) % 1.0))) for b in range(B)]


def _lengths(c):
    return _spread(c["Nmin"], c["N"], c["B"])


def _new_tokens(c):
    """Of each session of a slots pass: the span's length, and how many of it are wanted."""
    n = _spread(c["nmin"], c["n"], c["B"])
    return n, [0 if c["padded"] and b % 3 == 2 else x for b, x in enumerate(n)]


def _type(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def work(case):
    c = case
    if c["kind"] == "slots":             # slots read and written by the return; read and written thrice by the take
        T = float(sum(_new_tokens(c)[1]))
        return {"bytes": 24 * T + 16.0 * c["B"], "flops": T}
    es, D, units = 2 if c["dtype"] == "bf16" else 4, c["D"], c["L"] * c["Hkv"]
    row = D + 2 * D // BLOCK             # K and V of one entry and head
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


# ----------------------------------------------------------------------------- the 4-bit rows, plainly

def _quantise(x):
    """Rows x [..., D] (float32) -> codes [..., D / 2] and scales [..., D / 32], bytes."""
    x = x.unflatten(-1, (-1, BLOCK))
    a = x.abs().amax(-1).double().clamp_min(LEAST)
    m, e = torch.frexp(a / 7)                        # a / 7 = m 2^e, 0.5 <= m < 1
    e = torch.where(m == 0.5, e - 1, e).clamp_max(125)
    r = x * torch.exp2(-e.float())[..., None]        # exact
    z = r.abs()
    code = ((z > 0.25).byte() + (z >= 0.75) + (z > 1.25) + (z >= 1.75) + (z > 2.5) + (z >= 3.5) + (z > 5) +
            (r < 0).byte() * 8).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | code[..., 1] << 4, (e + 127).byte()


def _values(codes, scales):
    """float32 rows that codes [..., D / 2] with scales [..., D / 32] stand for."""
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    x = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], -1).flatten(-2)
    s = (scales.int() << 23).view(torch.float32)
    return (x.unflatten(-1, (-1, BLOCK)) * s[..., None]).flatten(-2)


# ----------------------------------------------------------------------------- inputs

def _pages(Ns, gen, dev):
    """Each session's list of slots, pages dealt from a shuffle (slot 0 is the sentinel), and the pool's slots."""
    pages = [-(-N // PAGE) for N in Ns]
    order = torch.randperm(sum(pages), generator=gen, device=dev)
    lists, p = [], 0
    for N, np_ in zip(Ns, pages):
        j = torch.arange(N, device=dev)
        lists.append(1 + order[p:p + np_][j // PAGE] * PAGE + j % PAGE)
        p += np_
    return torch.cat(lists).to(torch.int32), 1 + sum(pages) * PAGE


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 31)
    st = _prepare_slots(c, gen, dev) if c["kind"] == "slots" else _prepare_rows(c, gen, dev)
    if own:
        st.update(_handles(st))
    torch.cuda.synchronize()
    return st


def _prepare_rows(c, gen, dev):
    randn = lambda *z: torch.randn(*z, generator=gen, device=dev)  # noqa: E731
    L, Hq, Hkv, D, dt, kind = c["L"], c["Hq"], c["Hkv"], c["D"], _type(c), c["kind"]
    Ns = _lengths(c)
    live, num_slots = _pages(Ns, gen, dev)
    st = dict(case=c, Ns=Ns, num_slots=num_slots, total=sum(Ns), live=live,
              n_live=torch.tensor(Ns, dtype=torch.int32, device=dev))
    chan, mean = torch.exp(0.4 * randn(L, 1, Hkv, D)), randn(L, 1, Hkv, D)
    size = torch.ones(num_slots, 1, 1, device=dev)
    size[torch.randperm(num_slots, generator=gen, device=dev)[:num_slots // 20]] = 3.0
    rows = lambda l: ((randn(num_slots, Hkv, D) * chan[l] * size).to(dt),  # noqa: E731
                      (randn(num_slots, Hkv, D) + mean[l]).to(dt))
    if kind == "round":                               # rows of a pool
        st["k"], st["v"] = (torch.zeros(L, num_slots, Hkv, D, dtype=dt, device=dev) for _ in range(2))
        for l in range(L):
            st["k"][l], st["v"][l] = rows(l)
    # the 4-bit cache, written already unless the pass writes it
    st["kc"], st["vc"] = (torch.zeros(L, num_slots, Hkv, D // 2, dtype=torch.uint8, device=dev) for _ in range(2))
    st["scales"] = torch.full((L, num_slots, Hkv, 2, D // BLOCK), 127, dtype=torch.uint8, device=dev)
    if kind != "round":
        for l in range(L):
            for codes, x, i in zip(("kc", "vc"), rows(l), (0, 1)):
                st[codes][l], st["scales"][l, :, :, i] = _quantise(x.float())
    if kind in ("round", "load"):                     # where the rows are read back to
        st["k_out"], st["v_out"] = (torch.zeros(L, st["total"], Hkv, D, dtype=dt, device=dev) for _ in range(2))
    else:                                             # packed by session: [L][Hq][n][D]
        st["q"] = randn(len(Ns) * L * Hq * c["n"] * D).to(dt)
        st["out"] = torch.zeros_like(st["q"])
    return st


def _prepare_slots(c, gen, dev):
    B, (spans, wanted) = c["B"], _new_tokens(c)
    Ns = [c["N"] - c["n"] + x for x in spans]         # equal histories before uneven spans
    T, total = sum(wanted), sum(Ns)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    offs = [sum(Ns[:b]) for b in range(B + 1)]
    # what the retention event freed: T slots in all, unevenly over the sessions
    cuts = sorted(torch.randint(0, T + 1, (B - 1,), generator=gen, device=dev).tolist())
    n_freed = [min(b - a, N) for a, b, N in zip([0] + cuts, cuts + [T], Ns)]
    for b in range(B):                                # what does not fit a session's list goes to others
        n_freed[b] += min(Ns[b] - n_freed[b], T - sum(n_freed))
    num_slots = 2 * total + 1
    order = 1 + torch.randperm(num_slots - 1, generator=gen, device=dev).int()
    freed, at = torch.zeros(total, dtype=torch.int32, device=dev), 0
    for b in range(B):
        freed[offs[b]:offs[b] + n_freed[b]] = order[at:at + n_freed[b]]
        at += n_freed[b]
    n_free = total // 3                               # free already; the rest of the pool is in use
    free = torch.zeros(num_slots, dtype=torch.int32, device=dev)
    free[:n_free] = order[T:T + n_free]
    hist = [(N - x) * 5 // 8 for N, x in zip(Ns, spans)]      # live before the new tokens
    zeros = lambda n: torch.zeros(n, dtype=torch.int32, device=dev)  # noqa: E731
    st = dict(case=c, Ns=Ns, spans=spans, num_slots=num_slots, n_new=ints(wanted) if c["padded"] else None,
              free=free, n_free=ints([n_free, 0]), freed=freed, n_freed=ints(n_freed), n_live=ints(hist),
              live=zeros(total), slot_maps=zeros(total), dst=zeros(total), n_all=zeros(B), n_taken=zeros(B))
    # the batch's layout, as a program keeps it: session and place of each token of a span, of each place of a list
    st["off"], st["span"], st["room"] = ints(offs[:-1]).long(), ints(spans).long(), ints(Ns).long()
    for name, n in (("token", spans), ("entry", Ns)):
        b = torch.repeat_interleave(torch.arange(B, device=dev), ints(n).long(), output_size=sum(n))
        st[name] = b, torch.arange(sum(n), device=dev) - (torch.cumsum(ints(n).long(), 0) - ints(n).long())[b]
    return st


def _handles(st):
    """The descriptors and the workspace that a caller of the library keeps."""
    from paper_2606_09916_amd import ikv
    c, dev, h = st["case"], st["live"].device, {}
    rows, o = [], 0
    for b, N in enumerate(st["Ns"]):
        n = st["spans"][b] if c["kind"] == "slots" else c["n"]
        rows.append(dict(slot_off=o, mem_off=0, qspan_off=0, qpos_off=0, N=N, pi=0, qs=N - n, qe=N, C=N,
                         radix_prefix=0, R=1, nq=0))
        o += N
    h["sess"] = ikv.Sessions(rows, dev)
    if c["kind"] == "slots":
        h["stack"] = ikv.make_free_slots(st["free"], st["n_free"], st["num_slots"], 0)
        return h
    L, Hq, Hkv, D = c["L"], c["Hq"], c["Hkv"], c["D"]
    h["ws"] = ikv.Workspace(dev)
    h["qpool"] = ikv.make_quant_pool(st["kc"], st["vc"], st["scales"], L, Hq, Hkv, D, st["num_slots"], 0,
                                     io_dtype=_type(c))
    if "k" in st:
        h["pool"] = ikv.make_pool(st["k"], st["v"], L, Hq, Hkv, D, st["num_slots"], 0)
    if "k_out" in st:
        h["back"] = ikv.make_pool(st["k_out"], st["v_out"], L, Hq, Hkv, D, st["total"], 0)
    return h


# ----------------------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _slots_out(st):
    return [st[k] for k in ("slot_maps", "live", "n_all", "dst", "n_taken", "free", "n_free")]


def _run_own(st):
    from paper_2606_09916_amd import ikv
    c = st["case"]
    if c["kind"] == "slots":
        ikv.return_slots(st["stack"], st["sess"], st["freed"], st["n_freed"])
        ikv.take_slots(st["stack"], st["sess"], st["n_taken"], slot_maps=st["slot_maps"], live=st["live"],
                       n_live=st["n_live"], n_all=st["n_all"], dst=st["dst"], n_new=st["n_new"])
        return _slots_out(st)
    if c["kind"] in ("round", "load"):
        if c["kind"] == "round":
            ikv.quant_store(st["qpool"], st["pool"], st["sess"], st["live"], st["live"], st["n_live"])
        ikv.quant_load(st["qpool"], st["back"], st["sess"], st["live"], None, st["n_live"])
        return [st["k_out"], st["v_out"]]
    call = ikv.decode_attend_quant if c["kind"] == "decode" else ikv.attend_chunk_quant
    call(st["qpool"], st["sess"], st["q"], st["live"], st["n_live"], st["out"], st["ws"], sinks=c["sinks"],
         window=c["window"])
    return [st["out"]]


def _put(buf, at, values, where):
    """buf[at] = values where it holds, and nothing elsewhere."""
    grown = torch.cat([buf, buf[:1]])
    grown[torch.where(where, at, len(buf))] = values
    buf.copy_(grown[:-1])


def _plain_slots(st):
    free, n_free, off = st["free"], st["n_free"], st["off"]
    # return
    b, k = st["entry"]
    n = torch.minimum(st["n_freed"].long().clamp_min(0), st["room"])
    _put(free, n_free[0] + (torch.cumsum(n, 0) - n)[b] + k, st["freed"][off[b] + k], k < n[b])
    have = n_free[0] + n.sum()
    # take
    b, t = st["token"]
    n = st["span"] if st["n_new"] is None else torch.minimum(st["n_new"].long().clamp_min(0), st["span"])
    n_live = torch.minimum(st["n_live"].long().clamp_min(0), st["room"])
    n = torch.where(n_live + n <= st["room"], n, 0)
    n = torch.where(torch.cumsum(n, 0) <= have, n, 0)
    before, served, left = torch.cumsum(n, 0) - n, t < n[b], have - n.sum()
    slots = free[torch.where(served, left + before[b] + t, 0)]
    _put(st["slot_maps"], (off + st["room"] - st["span"])[b] + t, slots, served)
    _put(st["live"], (off + n_live)[b] + t, slots, served)
    _put(st["dst"], off[b] + t, slots, served)
    st["n_all"].copy_(n_live + n)
    st["n_taken"].copy_(n)
    n_free[:1] = left
    return _slots_out(st)


def _plain_rows(st, which, layers, slots):
    """float32 rows [layers, len(slots), Hkv, D] that the cache holds at these slots."""
    return _values(st[which + "c"][layers][:, slots], st["scales"][layers][:, slots, :, "kv".index(which)])


def _run_plain(st):
    c = st["case"]
    if c["kind"] == "slots":
        return _plain_slots(st)
    L, Hq, Hkv, D, n = c["L"], c["Hq"], c["Hkv"], c["D"], c["n"]
    slots = st["live"].long()
    if c["kind"] in ("round", "load"):
        at_once = max(1, min(L, 2 ** 27 // (st["total"] * Hkv * D)))
        for l in range(0, L, at_once):
            layers = slice(l, l + at_once)
            for which, i in (("k", 0), ("v", 1)):
                if c["kind"] == "round":
                    q, s = _quantise(st[which][layers][:, slots].float())
                    st[which + "c"][layers, slots], st["scales"][layers, slots, :, i] = q, s
                st[which + "_out"][layers] = _plain_rows(st, which, layers, slots).to(_type(c))
        return [st["k_out"], st["v_out"]]
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

def _stands_for(x):
    """What rows x [..., D] (float64) stand for once quantised."""
    x = x.reshape(*x.shape[:-1], -1, BLOCK)
    a = x.abs().max(-1, keepdim=True).values.clamp(min=LEAST)
    powers = torch.tensor([2.0 ** e for e in range(-120, 126)], dtype=torch.float64, device=x.device)
    s = powers[torch.searchsorted(powers * 7, a).clamp(max=len(powers) - 1)]     # the first that holds a
    r = (x / s).abs()
    step = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0)).double()        # of the binade that holds r
    y = torch.minimum(torch.round(r / step) * step, torch.full_like(r, 6.0))
    return (torch.copysign(y, x) * s).flatten(-2)


def _held(codes, scales):
    """What one layer's codes [slots, Hkv, D / 2] and scales [slots, Hkv, D / 32] stand for, in float64."""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2)
    k = (c % 8).double()
    mag = torch.where(k < 2, k / 2, (1 + (k % 2) / 2) * torch.exp2(torch.floor(k / 2) - 1))
    s = torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1)
    return torch.where(c >= 8, -mag, mag) * s


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    if c["kind"] == "slots":
        return _exact_slots(st)
    L, Hq, Hkv, D, n = c["L"], c["Hq"], c["Hkv"], c["D"], c["n"]

    def held(which, l, at):
        if c["kind"] == "round":
            return _stands_for(st[which][l][at].double())
        return _held(st[which + "c"][l][at], st["scales"][l][at][:, :, "kv".index(which)])

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


def _exact_slots(st):
    h = {k: st[k].cpu().numpy() for k in ("slot_maps", "live", "n_all", "dst", "n_taken", "free", "n_free", "freed",
                                          "n_freed", "n_live")}
    stack = h["free"][:h["n_free"][0]].tolist()
    o, wanted = 0, st["spans"] if st["n_new"] is None else st["n_new"].tolist()
    for b, N in enumerate(st["Ns"]):
        stack += h["freed"][o:o + h["n_freed"][b]].tolist()
        o += N
    h["free"][:len(stack)] = stack
    served, T = [], 0
    for b, N in enumerate(st["Ns"]):
        fits = h["n_live"][b] + wanted[b] <= N and T + wanted[b] <= len(stack)
        served.append(wanted[b] if fits else 0)
        T += served[b]
    o, at = 0, len(stack) - T
    for b, (N, n) in enumerate(zip(st["Ns"], served)):
        mine, qs, nl = stack[at:at + n], o + N - st["spans"][b], o + h["n_live"][b]
        h["slot_maps"][qs:qs + n] = h["live"][nl:nl + n] = h["dst"][o:o + n] = mine
        h["n_all"][b], h["n_taken"][b] = h["n_live"][b] + n, n
        o, at = o + N, at + n
    h["n_free"][0] = len(stack) - T
    return [torch.from_numpy(h[k]) for k in ("slot_maps", "live", "n_all", "dst", "n_taken", "free", "n_free")]

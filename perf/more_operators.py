"""A cache held in 4 bits (written, read back, attended to, evicted from) and attention with a sliding window, for
timing and comparing.

The 4-bit form: blocks of 32 coordinates, value = code * 2^e with codes of one sign, two exponent and one mantissa bit
(0, 0.5, 1, 1.5, 2, 3, 4, 6) and one byte e + 127 a block.  e is the smallest with amax <= 7 * 2^e, in [-124, 125].

A case is a dict of plain values; "kind" names the operator:

  store    T new tokens of every sequence are written into its 4-bit cache, and what was written is read back (as for
           scoring, which takes plain keys);
  attend4  attention of the newest T queries over a 4-bit cache, optionally adding to every cached token's `mass` the
           weight that it was given, optionally with a window;
  evict4   the tokens that came since the last eviction are written into the 4-bit cache, then each head keeps its
           prefix, its recent window and the tokens of largest mass, and the cache is compacted in place: in order, or
           with the kept rows past the budget moved into the holes below it ("fill");
  window   attention over a bf16 or fp32 cache where a query sees the last `window` tokens up to its own, and the first
           `sinks` ones.

`own` selects the side: the framework's calls where it is true, else the same from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda"
INF = math.inf
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, name, **kw):
    c = {"name": name, "kind": kind, "dtype": "bf16", "D": 128, "T": 1, "cap": 0, "ragged": False}
    return dict(c, **kw)


def _attend4(name, **kw):
    return _case("attend4", name, **dict({"causal": False, "mass": False, "window": 0, "sinks": 0}, **kw))


def listed():
    return [
        # a decode step's token of every sequence and layer into the caches, at places of their own
        _case("store", "store step 36 layers", B=576, Hkv=8, N=4096, ragged=True),
        # a prompt's keys and values of all 36 layers
        _case("store", "store prompt 36 layers", B=36, Hkv=8, T=4096, N=4096, cap=128),
        # the smallest call: a decode step of one layer of a small fp32 model, where only latency counts
        _attend4("step tiny fp32", B=1, Hq=8, Hkv=2, D=64, N=512, dtype="fp32"),
        # a decode step of all 36 layers stacked into one call, weights collected, as the periodic driver has it
        _attend4("step 36 layers mass", B=576, Hq=32, Hkv=8, N=3584, cap=512, mass=True),
        # one sequence with a long cache: few heads, the work is split over the tokens
        _attend4("step 64k", B=1, Hq=32, Hkv=8, N=65536),
        # five drafted tokens verified at once, seven query heads per kv-head, ragged lengths in a longer allocation
        _attend4("verify ragged 16k", B=8, Hq=28, Hkv=4, T=5, N=16001, cap=383, causal=True, ragged=True),
        # prompts read in, their weights collected for the first eviction
        _attend4("prompt 4k mass", B=2, Hq=32, Hkv=8, T=4096, N=4096, causal=True, mass=True),
        # the periodic eviction of all 36 layers, 7/8 of the cache kept, kept rows left where they are
        _case("evict4", "evict 36 layers fill", B=576, Hkv=8, N=4096, W=32, budget=3584, n_prefix=4, fill=True),
        # a layer of long caches cut to an eighth, in token order
        _case("evict4", "evict 32k", B=8, Hkv=8, N=32768, W=32, budget=4096, n_prefix=4, fill=False),
        # a decode step of a layer with a window, over long caches of many sequences
        _case("window", "window step", B=32, Hq=32, Hkv=8, N=16000, cap=100, window=1024, sinks=4, ragged=True),
        # a long prompt read in by a layer with a window
        _case("window", "window prompt 16k", B=1, Hq=32, Hkv=8, T=16384, N=16384, window=4096, sinks=4),
        # chunks of long prompts against what is cached already, small heads, lengths of their own
        _case("window", "window chunk of 24k", B=2, Hq=28, Hkv=4, D=64, T=500, N=24001, cap=575, window=4096, sinks=16, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "attend4", "attend4", "attend4", "evict4", "evict4", "window", "window", "window"])
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 4, 5, 7, 8])
    c = {"kind": kind, "dtype": "fp32" if rng.random() < 0.2 else "bf16", "D": 64 if rng.random() < 0.25 else 128, "Hkv": Hkv, "cap": rng.choice([0, 0, rng.randint(1, 500)])}
    c["ragged"] = rng.random() < 0.4
    fp32 = c["dtype"] == "fp32"
    room = (1 << 24) // (4 if fp32 else 1)  # tokens of all heads: the largest listed case has 16 M
    if kind == "store":
        T = rng.choice([1, 1, rng.randint(2, 9), _log(rng, 16, 8192)])
        N = max(T, _log(rng, 64, 16384))
        B = max(1, min(_log(rng, 1, 576), room // 8 // (Hkv * T), room // (Hkv * N)))
        return dict(c, B=B, T=T, N=N)
    if kind == "evict4":
        N = _log(rng, 256, 65536)
        B = max(1, min(_log(rng, 1, 512), room // 2 // (Hkv * N)))
        W = rng.choice([1, 8, 16, 32, 64])
        budget = max(W + 5, N * 7 // 8 if rng.random() < 0.5 else N // rng.randint(2, 8))
        return dict(c, B=B, N=N, W=W, budget=budget, n_prefix=rng.choice([0, 1, 4]), fill=rng.random() < 0.5, T=1)
    c["Hq"] = Hkv * G
    form = rng.choice(["step", "step", "verify", "prompt", "chunk"])
    if form in ("step", "verify"):
        T = 1 if form == "step" else rng.randint(2, 9)
        N = _log(rng, max(1, T), 65536)
        B = max(1, min(_log(rng, 1, 512), room // 2 // (Hkv * N)))
    else:  # prompts and chunks: at most about half of the largest prompt's products
        N = _log(rng, 64, 8192) if form == "prompt" else _log(rng, 1024, 32768)
        T = N if form == "prompt" else rng.randint(17, max(18, min(N, 700)))
        B = max(1, min(_log(rng, 1, 16), (1 << 28) // (T * N * Hkv * G)))
        while B * T * N * Hkv * G > (1 << 29) // (4 if fp32 else 1):
            T, N = (T // 2, N // 2) if form == "prompt" else (max(1, T // 2), N * 3 // 4)
    N = max(T, N)
    c |= {"B": B, "T": T, "N": N, "window": 0, "sinks": 0}
    if kind == "window" or rng.random() < 0.25:
        c |= {"window": _log(rng, 16, 8192), "sinks": rng.choice([0, 1, 4, 4, 16, rng.randint(1, 200)])}
    if kind == "attend4":
        c |= {"causal": T > 9 or c["window"] > 0 or rng.random() < 0.5, "mass": c["window"] == 0 and rng.random() < 0.5}
    return c


# ---- the 4-bit form -----------------------------------------------------------------
def _codes(x):
    """Codes [..., D/2] and scale bytes [..., D/32] of values [..., D]: elementary operations, exact in 32 bits."""
    a = x.float().unflatten(-1, (-1, 32))
    m, k = torch.frexp(a.abs().amax(-1))
    e = torch.where(m <= 0.875, k - 3, k - 2)  # amax = m 2^k with m in [0.5, 1)
    e = torch.where(m == 0, -124, e).clamp_(-124, 125)
    y = torch.ldexp(a.abs(), -e.unsqueeze(-1))
    c = (y > 0.25).to(torch.uint8)
    for up, border in ((True, 0.75), (False, 1.25), (True, 1.75), (False, 2.5), (True, 3.5), (False, 5.0)):
        c += (y >= border) if up else (y > border)  # ties to the even code
    c += torch.signbit(a).to(torch.uint8) * 8
    c = c.flatten(-2)
    return c[..., 0::2] | c[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The 32-bit values of codes [..., D/2] and scale bytes [..., D/32]."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEV)
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    v = table[c.int()].unflatten(-1, (-1, 32))
    return torch.ldexp(v, scales.int().unsqueeze(-1) - 127).flatten(-2)


def _cache(shape, rows, g):
    """Codes and scale bytes of a cache; rows(b0, b1) makes the values of some sequences."""
    B, Hkv, cap, D = shape
    codes, scales = (torch.empty(B, Hkv, cap, n, dtype=torch.uint8, device=DEV) for n in (D // 2, D // 32))
    step = max(1, (1 << 26) // (Hkv * cap * D))
    for b in range(0, B, step):
        codes[b:b + step], scales[b:b + step] = _codes(rows(b, min(B, b + step)))
    return codes, scales


# ---- inputs ---------------------------------------------------------------------
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lengths(c):
    """Lengths of the sequences, evenly spread from a quarter of the longest."""
    B, N = c["B"], c["N"]
    if not c["ragged"] or B < 2:
        return [N] * B
    return torch.linspace(max(1, min(N, c["T"]), N // 4), N, B).round().int().tolist()


def _lens(c, seed):
    """The same on the GPU, in an order of the seed's own."""
    v = torch.tensor(_lengths(c), dtype=torch.int32)
    return v[torch.randperm(len(v), generator=torch.Generator().manual_seed(seed))].to(DEV) if c["ragged"] else None


def _normal(shape, g, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)


def _near(k, mean, g):
    """One key in 32, and the first two, near the mean of the queries that will come: what collects weight."""
    near = torch.rand(k.shape[:3], generator=g, device=DEV) < 1 / 32
    near[:, :, :2] = True
    return k.add_(near.unsqueeze(-1) * (0.4 * mean).to(k.dtype).unsqueeze(2))


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, Hkv, D, T, dt, cap = c["B"], c["Hkv"], c["D"], c["T"], _dtype(c), c["N"] + c["cap"]
    s = {"case": c}
    four = lambda rows: _cache((B, Hkv, cap, D), rows, g)  # noqa: E731
    anything = lambda b0, b1: _normal((b1 - b0, Hkv, cap, D), g)  # noqa: E731
    if c["kind"] == "store":
        s["K"], s["V"] = (_normal((B, Hkv, T, D), g, dt) for _ in "KV")
        # keys have a few large coordinates, each head its own
        s["K"] *= torch.exp(_normal((1, Hkv, 1, D), g)).to(dt)
        s["KC"], s["KS"] = four(anything)
        s["VC"], s["VS"] = s["KC"].clone(), s["KS"].clone()
        at = _lens(c, seed)
        s["at"] = None if at is None else (at - T).clamp_min(0)
        s["k"], s["v"] = torch.empty_like(s["K"]), torch.empty_like(s["V"])
        return s
    if c["kind"] == "evict4":
        s["KC"], s["KS"] = four(anything)
        s["VC"], s["VS"] = four(anything)
        n = min(c["N"], c["budget"])
        # what comes between evictions: new tokens, and every token's weight
        s["turns"] = max(1, min(4, (1 << 28) // max(1, B * Hkv * D * (c["N"] - n))))
        if n < c["N"]:
            s["more_K"], s["more_V"] = (_normal((s["turns"], B, Hkv, c["N"] - n, D), g, dt) for _ in "KV")
        mass = torch.empty(s["turns"], B, Hkv, c["N"], device=DEV).exponential_(1.0, generator=g)
        mass.mul_(torch.rand(mass.shape, generator=g, device=DEV) > 0.03)  # tokens that nothing attended to: equal masses
        s["more_mass"], s["mass"] = mass, torch.zeros(B, Hkv, cap, device=DEV)
        s["turn"] = 0
        s["kept"] = torch.empty(B, Hkv, n, dtype=torch.int32, device=DEV)
        return s
    G = c["Hq"] // Hkv
    mean = _normal((B, Hkv, D), g)
    s["q"] = (1.2 * _normal((B, Hkv, G, T, D), g) + 0.8 * mean[:, :, None, None]).to(dt).reshape(B, c["Hq"], T, D)
    if c["kind"] == "attend4":
        s["KC"], s["KS"] = four(lambda b0, b1: _near(anything(b0, b1), mean[b0:b1], g))
        s["VC"], s["VS"] = four(anything)
    else:
        s["K"] = _near(_normal((B, Hkv, cap, D), g, dt), mean, g)
        s["V"] = _normal((B, Hkv, cap, D), g, dt)
    s["lens"] = _lens(c, seed)
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(B, c["Hq"], T, device=DEV)
    s["mass"] = torch.rand(B, Hkv, cap, generator=g, device=DEV) if c.get("mass") else None
    return s


# ---- the plain forms --------------------------------------------------------------
def _place(c, s, at):
    """Sequence and token indices of T rows from position at on (or from at[b] on)."""
    first = at.long().view(-1, 1) if isinstance(at, torch.Tensor) else torch.full((c["B"], 1), at, device=DEV)
    return torch.arange(c["B"], device=DEV).view(-1, 1), first


def _plain_store(c, s, K, V, at):
    b, first = _place(c, s, at)
    rows = first + torch.arange(K.shape[2], device=DEV)
    for x, codes, scales in ((K, s["KC"], s["KS"]), (V, s["VC"], s["VS"])):
        n, e = _codes(x)
        codes.transpose(1, 2)[b, rows] = n.transpose(1, 2)
        scales.transpose(1, 2)[b, rows] = e.transpose(1, 2)


def _plain_load(c, s, at):
    b, first = _place(c, s, at)
    rows = first + torch.arange(c["T"], device=DEV)
    for x, codes, scales in ((s["k"], s["KC"], s["KS"]), (s["v"], s["VC"], s["VS"])):
        x.copy_(_values(codes.transpose(1, 2)[b, rows], scales.transpose(1, 2)[b, rows]).transpose(1, 2))


def _softmax(l, V):
    """Weights [..., R, N], outputs and normalisers of logits l, -inf where a row does not see."""
    m = l.amax(-1, keepdim=True).clamp_min(-1e30)
    e = torch.exp(l - m)
    z = e.sum(-1, keepdim=True)
    w = e / z.clamp_min(1e-38)
    return w, torch.matmul(w, V), m + torch.log(z)


def _plain_attend4(c, s):
    B, Hkv, D, T, N = c["B"], c["Hkv"], c["D"], c["T"], c["N"]
    G = c["Hq"] // Hkv
    K, V = (_values(s[x + "C"][:, :, :N], s[x + "S"][:, :, :N]) for x in "KV")
    n = s["lens"].long().view(-1, 1, 1) if s["lens"] is not None else torch.full((1, 1, 1), N, device=DEV)
    j, p = torch.arange(N, device=DEV), n - T + torch.arange(T, device=DEV).view(T, 1)
    seen = (j < n) & ((j <= p) if c["causal"] else (p >= p))
    if c["window"]:
        seen = seen & ((j > p - c["window"]) | (j < c["sinks"]))
    l = torch.matmul(s["q"].float().view(B, Hkv, G * T, D), K.transpose(-1, -2).contiguous()) / math.sqrt(D)
    l = l.view(B, Hkv, G, T, N).masked_fill_(~seen[:, None, None], -INF).view(B, Hkv, G * T, N)
    if s["lens"] is not None:  # what lies behind a sequence is not read
        V = V.masked_fill((j >= n.view(B, 1, 1)).unsqueeze(-1), 0.0)
    w, out, lse = _softmax(l, V)
    s["out"].copy_(out.view(s["out"].shape))
    s["lse"].copy_(lse.view(s["lse"].shape))
    if c["mass"]:
        s["mass"][:, :, :N] += w.sum(2)


def _plain_window(c, s):
    """Blocks of queries against the tokens that any of them sees: the first ones and a stretch up to their own."""
    B, Hkv, D, T, N = c["B"], c["Hkv"], c["D"], c["T"], c["N"]
    G, W, S = c["Hq"] // Hkv, c["window"], min(c["sinks"], N)
    n = s["lens"].long().view(-1, 1) if s["lens"] is not None else torch.full((B, 1), N, device=DEV)
    q = s["q"].float().view(B, Hkv, G, T, D)
    out, lse = s["out"].view(B, Hkv, G, T, D), s["lse"].view(B, Hkv, G, T)
    step = max(16, min(512, (1 << 30) // (B * c["Hq"] * (W + S + 512))))
    for t0 in range(0, T, step):
        t1 = min(T, t0 + step)
        near = n - T + t0 + 1 - W + torch.arange(min(W - 1 + t1 - t0, N + t1 - t0), device=DEV)  # [B, stretch]
        near = near + (n - T + t1 - 1 - near[:, -1:])  # its last token is the last query's
        j = torch.cat([torch.arange(S, device=DEV).expand(B, S), near], 1)
        there = torch.cat([(j[:, :S] < n), (near >= S) & (near < n)], 1)  # each token once
        at = j.clamp(0, N - 1)
        p = n - T + torch.arange(t0, t1, device=DEV)  # [B, queries]
        seen = (there & (j >= 0)).unsqueeze(1) & (j.unsqueeze(1) <= p.unsqueeze(2)) & ((j.unsqueeze(1) > p.unsqueeze(2) - W) | (j < S).unsqueeze(1))
        b = torch.arange(B, device=DEV).view(-1, 1)
        K, V = (s[x].transpose(1, 2)[b, at].transpose(1, 2).float() for x in "KV")  # [B, Hkv, some, D]
        if s["lens"] is not None:
            V = V.masked_fill((at >= n).view(B, 1, -1, 1), 0.0)
        l = torch.matmul(q[:, :, :, t0:t1].reshape(B, Hkv, -1, D), K.transpose(-1, -2).contiguous()) / math.sqrt(D)
        l = l.view(B, Hkv, G, t1 - t0, -1).masked_fill_(~seen[:, None, None], -INF).view(B, Hkv, G * (t1 - t0), -1)
        _, o, e = _softmax(l, V)
        out[:, :, :, t0:t1] = o.view(B, Hkv, G, t1 - t0, D).to(out.dtype)
        lse[:, :, :, t0:t1] = e.view(B, Hkv, G, t1 - t0)


def _plain_evict(c, s):
    N, W, n = c["N"], c["W"], min(c["N"], c["budget"])
    if N <= n:
        s["kept"].copy_(torch.arange(n, device=DEV, dtype=torch.int32).expand(s["kept"].shape))
        return
    m = s["mass"][:, :, :N].clone()
    m[:, :, :c["n_prefix"]] = INF
    m[:, :, N - W:] = INF
    kept = m.sort(dim=-1, descending=True, stable=True).indices[:, :, :n].sort(dim=-1).values
    if c["fill"]:
        at = torch.arange(n, device=DEV)
        stays = torch.zeros(m.shape, dtype=torch.bool, device=DEV).scatter_(2, kept, True)[:, :, :n]
        past = stays.sum(-1, keepdim=True) + (~stays).cumsum(-1) - 1  # the hole's turn among the kept rows from n on
        kept = torch.where(stays, at, kept.gather(2, past.clamp_max(n - 1)))
    for x in ("KC", "KS", "VC", "VS"):
        r = _words(s[x])
        r[:, :, :n] = r.gather(2, kept.unsqueeze(-1).expand(-1, -1, -1, r.shape[-1]))
    s["mass"][:, :, :n] = s["mass"].gather(2, kept)
    s["mass"][:, :, n:N] = 0.0
    s["kept"].copy_(kept)


def _words(t):
    """Rows as the widest whole numbers that fit: they are moved, not computed."""
    n = t.shape[-1]
    return t.view(torch.int64 if n % 8 == 0 else torch.int32 if n % 4 == 0 else torch.int16)


# ---- the framework's calls ----------------------------------------------------------
def _own(c, s):
    """The binding; dims, cache and workspaces are kept from call to call, as a decoding loop does."""
    import paper_2609_04971_amd as bkv
    if "d" not in s:
        s["d"] = bkv.dims(B=c["B"], Hq=c.get("Hq", c["Hkv"]), Hkv=c["Hkv"], D=c["D"], N=c["N"], N_cap=c["N"] + c["cap"], W=c.get("W", 0), C=0,
                          budget=c.get("budget", 1), n_prefix=c.get("n_prefix", 0), dtype=c["dtype"])
        if "KC" in s:
            s["cache"] = bkv.MxCache(s["KC"], s["KS"], s["VC"], s["VS"])
        if "q" in s:
            s["ws"] = bkv.attend_workspace(s["d"], T=c["T"], mass=bool(c.get("mass")))
        elif c["kind"] == "evict4":
            s["ws"] = bkv.mass_workspace(s["d"])
    return bkv


# ---- one pass ---------------------------------------------------------------------
def run(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "store":
        at = s["at"] if s["at"] is not None else c["N"] - c["T"]
        if own:
            bkv = _own(c, s)
            bkv.store_mx(s["d"], s["K"], s["V"], s["cache"], at)
            bkv.load_mx(s["d"], s["cache"], s["k"], s["v"], at)
        else:
            _plain_store(c, s, s["K"], s["V"], at)
            _plain_load(c, s, at)
        return {"k": s["k"], "v": s["v"]}
    if kind == "evict4":
        t, n = s["turn"] % s["turns"], min(c["N"], c["budget"])
        s["turn"] += 1
        s["mass"][:, :, :c["N"]] = s["more_mass"][t]
        if own:
            bkv = _own(c, s)
            if n < c["N"]:
                bkv.store_mx(s["d"], s["more_K"][t], s["more_V"][t], s["cache"], n)
            bkv.evict_mass_mx(s["d"], s["cache"], s["mass"], s["ws"], kept=s["kept"], fill=c["fill"])
        else:
            if n < c["N"]:
                _plain_store(c, s, s["more_K"][t], s["more_V"][t], n)
            _plain_evict(c, s)
        # rows and weights are moved, not computed: all of their bits
        return {"KC": s["KC"].view(torch.int32), "KS": s["KS"], "VC": s["VC"].view(torch.int32), "VS": s["VS"], "mass": s["mass"].view(torch.int32), "kept": s["kept"]}
    if not own:
        (_plain_attend4 if kind == "attend4" else _plain_window)(c, s)
    elif kind == "attend4":
        bkv = _own(c, s)
        bkv.attend_mx(s["d"], s["q"], s["cache"], s["out"], s["ws"], lens=s["lens"], lse=s["lse"], mass=s["mass"], causal=c["causal"],
                    window=c["window"], sinks=c["sinks"])
    else:
        bkv = _own(c, s)
        bkv.attend_window(s["d"], s["q"], s["K"], s["V"], s["out"], s["ws"], c["window"], sinks=c["sinks"], lens=s["lens"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"], "mass": s["mass"]}


# ---- what a pass cannot do without -----------------------------------------------
def work(case):
    c = case
    es, D, Hkv, B, N = (2 if c["dtype"] == "bf16" else 4), c["D"], c["Hkv"], c["B"], c["N"]
    four = D // 2 + D // 32  # bytes of a row in 4 bits
    if c["kind"] == "store":  # the rows in, the 4-bit rows out, those in again, the values out
        return {"bytes": 4 * B * Hkv * c["T"] * (D * es + four), "flops": 0}
    if c["kind"] == "evict4":
        P, n = B * Hkv, min(c["budget"], N)
        moved = 0 if N <= n else min(n, N - n) if c["fill"] else n  # rows that change place: at most the ones past the budget, or nearly all
        return {"bytes": 2 * P * (N - n) * (D * es + four) + P * (8 * N + 4 * N + 4 * n + 4 * N) + 4 * P * moved * four, "flops": 0}
    T, Hq, W, S = c["T"], c["Hq"], c["window"], c["sinks"]
    seen = pairs = 0
    for n in _lengths(c):
        first = max(0, n - T + 1 - W) if W else 0  # the first token that is in any query's window
        seen += n - first + min(S, first)
        if W:
            full = lambda p: p * (p + 1) // 2 if p > 0 else 0  # noqa: E731  pairs of queries at positions below p
            p0, p1 = max(0, n - T), n
            beyond = max(0, p1 - max(p0, W))  # queries that do not see back to the start
            pairs += full(min(p1, W)) - full(min(p0, W)) + beyond * W + sum(min(S, p + 1 - W) for p in range(max(p0, W), min(p1, W + S))) + S * max(0, p1 - max(p0, W + S))
        else:
            pairs += n * T - (T * (T - 1) // 2 if c["causal"] else 0)
    row = four if c["kind"] == "attend4" else D * es
    return {"bytes": 2 * seen * Hkv * row + 2 * B * Hq * T * D * es + 4 * B * Hq * T + (8 * seen * Hkv if c.get("mass") else 0), "flops": 4 * Hq * max(0, pairs) * D}


# ---- the same in 64 bits --------------------------------------------------------------
def _nearest(x):
    """Values of x [..., D] in the 4-bit form, in 64 bits: rounded in units of half a code's own binade."""
    a = x.double().unflatten(-1, (-1, 32))
    top = a.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 7.0)).clamp(-124, 125)
    e = torch.where((top <= 7.0 * 2.0 ** (e - 1)) & (e > -124), e - 1, torch.where((top > 7.0 * 2.0 ** e) & (e < 125), e + 1, e))
    y = a / 2.0 ** e
    unit = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return ((torch.round(y / unit) * unit).clamp(-6, 6) * 2.0 ** e).flatten(-2)


def _looked_up(codes, scales):
    level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    v = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=DEV)
    v[..., 0::2] = level[(codes & 7).long()] * (1.0 - 2.0 * (codes >> 3 & 1))
    v[..., 1::2] = level[(codes >> 4 & 7).long()] * (1.0 - 2.0 * (codes >> 7))
    return v * torch.exp2(scales.double() - 127.0).repeat_interleave(32, -1)


def exact(case, seed):
    """Head by head, from softmax's definition with the normaliser as a logarithm; stored values from the form's definition."""
    c = dict(case)
    if c["kind"] == "evict4":
        return None  # indices and moved rows only
    s = prepare(c, seed)
    if c["kind"] == "store":
        return {"k": _nearest(s["K"]), "v": _nearest(s["V"])}
    B, Hkv, D, T, N, W, S = c["B"], c["Hkv"], c["D"], c["T"], c["N"], c["window"], c["sinks"]
    G = c["Hq"] // Hkv
    out, lse = torch.zeros(B, Hkv, G, T, D, dtype=torch.float64, device=DEV), torch.empty(B, Hkv, G, T, dtype=torch.float64, device=DEV)
    mass = s["mass"].double() if c.get("mass") else None
    lens = s["lens"].tolist() if s["lens"] is not None else [N] * B
    causal = c.get("causal", True)
    for b in range(B):
        n = lens[b]
        for h in range(Hkv):
            y = s["q"][b, h * G:(h + 1) * G].double()
            if c["kind"] == "attend4":
                k, v = (_looked_up(s[x + "C"][b, h, :n], s[x + "S"][b, h, :n]) for x in "KV")
            else:
                k, v = s["K"][b, h, :n].double(), s["V"][b, h, :n].double()
            for t0 in range(0, T, 1024):
                t = torch.arange(t0, min(T, t0 + 1024), device=DEV).view(-1, 1)
                last = n - T + t if causal else torch.full_like(t, n - 1)  # the last token that each query sees
                j = torch.arange(n, device=DEV)
                if W:
                    j = j[(j < S) | (j > n - T + t0 - W)]
                hidden = j > last
                if W:
                    hidden = hidden | ((j <= last - W) & (j >= S))
                l = (torch.matmul(y[:, t0:t0 + 1024], k[j].T.contiguous()) / math.sqrt(D)).masked_fill_(hidden, -INF)
                norm = torch.logsumexp(l, dim=-1)
                lse[b, h, :, t0:t0 + 1024] = norm
                w = torch.exp(l - norm.clamp_min(-1e300).unsqueeze(-1))
                out[b, h, :, t0:t0 + 1024] = torch.matmul(w, v[j])
                if mass is not None:
                    mass[b, h, j] += w.sum((0, 1))
    return {"out": out.view(s["out"].shape), "lse": lse.view(s["lse"].shape), "mass": mass}

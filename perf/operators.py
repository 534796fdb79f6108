"""Attention over the eviction library's caches and eviction by the attention weight that a token has had, for timing and comparing.

A case is a dict of plain values; "kind" names the operator:

  attend  attention of the newest T queries of every sequence over its cache (T = 1: a decode step; a few: drafted
          tokens being verified; many: a prompt or a chunk of one), optionally adding to every cached token's `mass`
          the weight that it was given;
  shared  the same where the sequences of a group share a long prefix, held once (several answers to one prompt); the
          layers of a model are groups of one call;
  evict   the tokens that came since the last eviction are written, then each head keeps its prefix, its recent window
          and the tokens of largest mass, and K, V and mass are compacted in place: in order, or with the kept rows past
          the budget moved into the holes below it ("fill").

`own` selects the side: the framework's calls where it is true, else the same from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda"
INF = math.inf


def _attend(name, **kw):
    c = {"name": name, "kind": "attend", "dtype": "bf16", "D": 128, "T": 1, "cap": 0, "causal": False, "ragged": False, "mass": False}
    return dict(c, **kw)


def _shared(name, **kw):
    return dict(_attend(name, groups=1, P=0, P_ragged=False), kind="shared", **kw)


def _evict(name, **kw):
    return dict({"name": name, "kind": "evict", "dtype": "bf16", "D": 128, "cap": 0, "n_prefix": 4, "fill": False}, **kw)


def listed():
    return [
        # the smallest call: a decode step of one layer of a small fp32 model, where only latency counts
        _attend("step tiny fp32", B=1, Hq=8, Hkv=2, D=64, N=512, dtype="fp32"),
        # the ordinary call: a decode step of one layer of 16 sequences at an eviction budget of 4096, weights collected
        _attend("step 4k mass", B=16, Hq=32, Hkv=8, N=4224, mass=True),
        # the same step for all 36 layers stacked into one call, as the periodic driver has it
        _attend("step 36 layers mass", B=576, Hq=32, Hkv=8, N=3584, cap=512, mass=True),
        # one sequence with a long cache: few heads, the work is split over the tokens
        _attend("step 64k", B=1, Hq=32, Hkv=8, N=65536),
        # five drafted tokens verified at once, seven query heads per kv-head, ragged lengths in a longer allocation
        _attend("verify ragged 16k", B=8, Hq=28, Hkv=4, T=5, N=16001, cap=383, causal=True, ragged=True),
        # prompts read in, their weights collected for the first eviction
        _attend("prompt 4k mass", B=2, Hq=32, Hkv=8, T=4096, N=4096, causal=True, mass=True),
        # a chunk of a long prompt against what is cached already, small heads
        _attend("chunk of 24k", B=1, Hq=28, Hkv=4, D=64, T=500, N=24001, cap=575, causal=True),
        # four samples of one short prompt
        _shared("shared 4 samples", B=4, Hq=32, Hkv=8, P=700, N=61, cap=67),
        # 64 samples of one long prompt, ragged answers, weights of the answers' tokens collected
        _shared("shared 64 samples 16k", B=64, Hq=32, Hkv=8, P=16384, N=2048, ragged=True, mass=True),
        # all 36 layers of 8 samples each: 36 groups
        _shared("shared 36 layers", B=288, Hq=32, Hkv=8, groups=36, P=4000, N=896, cap=128, mass=True),
        # the periodic eviction of all 36 layers, 7/8 of the cache kept, kept rows left where they are
        _evict("evict 36 layers fill", B=576, Hkv=8, N=4096, W=32, budget=3584, fill=True),
        # a layer of long caches cut to an eighth, in token order
        _evict("evict 32k", B=8, Hkv=8, N=32768, W=32, budget=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "verify", "prompt", "chunk", "shared", "shared", "evict", "evict"])
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 4, 5, 7, 8])
    c = {"dtype": "fp32" if rng.random() < 0.2 else "bf16", "D": 64 if rng.random() < 0.25 else 128, "Hkv": Hkv, "cap": rng.choice([0, 0, rng.randint(1, 500)])}
    room = (1 << 25) // (4 if c["dtype"] == "fp32" else 1)  # tokens of all heads: the largest listed case has 16 M
    if kind == "evict":
        N = _log(rng, 256, 65536)
        B = max(1, min(_log(rng, 1, 512), room // 4 // (Hkv * N)))
        W = rng.choice([1, 8, 16, 32, 64])
        budget = max(W + 5, N * 7 // 8 if rng.random() < 0.5 else N // rng.randint(2, 8))
        return dict(c, kind=kind, B=B, N=N, W=W, budget=budget, n_prefix=rng.choice([0, 1, 4]), fill=rng.random() < 0.5)
    c |= {"Hq": Hkv * G, "ragged": rng.random() < 0.4, "mass": rng.random() < 0.5, "kind": "attend", "T": 1, "causal": rng.random() < 0.7}
    if kind == "shared":
        groups = rng.choice([1, 1, 2, _log(rng, 1, 36)])
        S, P, N = _log(rng, 1, 64), _log(rng, 64, 32768), _log(rng, 1, 4096)
        S = max(1, min(S, room // 4 // (Hkv * G * groups * max(1, P // 16))))
        T = rng.choice([1, 1, 1, 2, 3])
        return dict(c, kind="shared", B=groups * S, groups=groups, P=P, P_ragged=groups > 1 and rng.random() < 0.5, T=T, N=max(T, min(N, room // 4 // (groups * S * Hkv))))
    if kind in ("step", "verify"):
        T = 1 if kind == "step" else rng.randint(2, 9)
        N = _log(rng, max(1, T), 65536)
        B = max(1, min(_log(rng, 1, 512), room // 4 // (Hkv * N)))
        return dict(c, B=B, T=T, N=N)
    # prompts and chunks: at most about a quarter of the largest prompt's products
    N = _log(rng, 64, 8192) if kind == "prompt" else _log(rng, 1024, 32768)
    T = N if kind == "prompt" else rng.randint(17, max(18, min(N, 700)))
    B = max(1, min(_log(rng, 1, 16), (1 << 28) // (T * N * Hkv * G)))
    while B * T * N * Hkv * G > (1 << 29) // (4 if c["dtype"] == "fp32" else 1):
        T, N = (T // 2, N // 2) if kind == "prompt" else (max(1, T // 2), N * 3 // 4)
    return dict(c, B=B, T=T, N=max(T, N), causal=True)


# ---- inputs ---------------------------------------------------------------------
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _lengths(n, N, low, g):
    """n lengths from `low` to N, evenly spread, in an order of the seed's own."""
    v = torch.linspace(low, N, n).round().int() if n > 1 else torch.tensor([N], dtype=torch.int32)
    return v[torch.randperm(n, generator=g)].to(DEV)


def _lens(c, g):
    return _lengths(c["B"], c["N"], max(1, c["N"] // 4), g) if c.get("ragged") else None


def _visible(c):
    """Cached tokens of all sequences, per kv-head."""
    if not c.get("ragged") or c["B"] < 2:
        return c["B"] * c["N"]
    return int(torch.linspace(max(1, c["N"] // 4), c["N"], c["B"]).round().sum())


def _keys(shape, mean, dtype, g):
    """Keys around 0, one in 32 of them near the mean of the queries that will come: what collects weight."""
    k = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)
    near = torch.rand(shape[:3], generator=g, device=DEV) < 1 / 32
    near[:, :, :2] = True
    return k.add_(near.unsqueeze(-1) * (0.4 * mean).to(dtype).unsqueeze(2))


def prepare(case, seed):
    c = dict(case)
    g, h = torch.Generator(device=DEV).manual_seed(seed), torch.Generator().manual_seed(seed)
    B, Hkv, D, dt, cap = c["B"], c["Hkv"], c["D"], _dtype(c), c["N"] + c["cap"]
    s = {"case": c}
    if c["kind"] == "evict":
        s["K"], s["V"] = (torch.empty(B, Hkv, cap, D, dtype=dt, device=DEV).normal_(generator=g) for _ in "KV")
        mass = torch.empty(B, Hkv, cap, device=DEV).exponential_(1.0, generator=g)
        mass.mul_(torch.rand(mass.shape, generator=g, device=DEV) > 0.03)  # tokens that nothing attended to: equal masses
        s["mass"] = mass
        new = c["N"] - min(c["N"], c["budget"])
        s["turns"] = max(1, min(16, (1 << 28) // max(1, B * Hkv * D * new)))  # tokens to come
        if new:
            s["more_K"], s["more_V"] = (torch.empty(s["turns"], B, Hkv, new, D, dtype=dt, device=DEV).normal_(generator=g) for _ in "KV")
            s["more_mass"] = torch.empty(s["turns"], B, Hkv, new, device=DEV).exponential_(1.5, generator=g)
        s["turn"] = 0
        s["kept"] = torch.empty(B, Hkv, min(c["N"], c["budget"]), dtype=torch.int32, device=DEV)
        return s
    G = c["Hq"] // Hkv
    groups = c.get("groups", B)
    S = B // groups
    mean = torch.randn(groups, Hkv, D, generator=g, device=DEV)
    own_mean = mean.repeat_interleave(S, 0)
    s["q"] = (1.2 * torch.randn(B, Hkv, G, c["T"], D, generator=g, device=DEV) + 0.8 * own_mean[:, :, None, None]).to(dt).reshape(B, c["Hq"], c["T"], D)
    s["K"] = _keys((B, Hkv, cap, D), own_mean, dt, g)
    s["V"] = torch.empty(B, Hkv, cap, D, dtype=dt, device=DEV).normal_(generator=g)
    s["lens"] = _lens(c, h)
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(B, c["Hq"], c["T"], device=DEV)
    s["mass"] = torch.rand(B, Hkv, cap, generator=g, device=DEV) if c["mass"] else None
    if c["kind"] == "shared":
        s["PK"] = _keys((groups, Hkv, c["P"], D), mean, dt, g)
        s["PV"] = torch.empty(groups, Hkv, c["P"], D, dtype=dt, device=DEV).normal_(generator=g)
        s["p_lens"] = _lengths(groups, c["P"], c["P"] // 2, h) if c["P_ragged"] else None
    return s


# ---- the plain forms --------------------------------------------------------------
def _seen(c, s):
    """[B or 1, 1, T, N] truth values: which of the cache's tokens each query sees."""
    T, N = c["T"], c["N"]
    n = s["lens"].long().view(-1, 1, 1, 1) if s["lens"] is not None else torch.full((1, 1, 1, 1), N, device=DEV)
    j, t = torch.arange(N, device=DEV), torch.arange(T, device=DEV).view(T, 1)
    return (j < n) & ((j <= n - T + t) if c["causal"] else (t >= 0))


def _logits(q, K, scale):
    """[B, Hkv, R, N] of queries [B, Hkv, R, D] and keys [B, Hkv, N, D]."""
    return torch.matmul(q, K.float().transpose(-1, -2).contiguous()) * scale


def _plain_attend(c, s):
    B, Hkv, D, T, N = c["B"], c["Hkv"], c["D"], c["T"], c["N"]
    G, scale = c["Hq"] // Hkv, 1.0 / math.sqrt(D)
    q = s["q"].float().view(B, Hkv, G * T, D)
    seen = _seen(c, s).unsqueeze(1)  # [B or 1, 1, 1, T, N]
    l = _logits(q, s["K"][:, :, :N], scale).view(B, Hkv, G, T, N).masked_fill(~seen, -INF)
    parts = [l]
    if c["kind"] == "shared":  # the rows of a group against its prefix, at once
        groups, P = c["groups"], c["P"]
        S = B // groups
        rows = q.view(groups, S, Hkv, G * T, D).transpose(1, 2).reshape(groups, Hkv, S * G * T, D)
        lp = _logits(rows, s["PK"], scale)
        if s["p_lens"] is not None:
            lp = lp.masked_fill(torch.arange(P, device=DEV) >= s["p_lens"].long().view(groups, 1, 1, 1), -INF)
        parts = [lp.view(groups, Hkv, S, G, T, P).transpose(1, 2).reshape(B, Hkv, G, T, P), l]
    m = torch.stack([x.amax(-1) for x in parts]).amax(0).unsqueeze(-1).clamp_min(-1e30)
    e = [torch.exp(x - m) for x in parts]
    z = sum(x.sum(-1, keepdim=True) for x in e)
    w = [x / z.clamp_min(1e-38) for x in e]
    own_v = s["V"][:, :, :N].float()
    if s["lens"] is not None:  # what lies behind a sequence is not read
        own_v = own_v.masked_fill(torch.arange(N, device=DEV).view(1, 1, N, 1) >= s["lens"].view(B, 1, 1, 1), 0.0)
    out = torch.matmul(w[-1].view(B, Hkv, G * T, N), own_v)
    if c["kind"] == "shared":
        wp = w[0].reshape(groups, S, Hkv, G * T, P).transpose(1, 2).reshape(groups, Hkv, S * G * T, P)
        out = out + torch.matmul(wp, s["PV"].float()).view(groups, Hkv, S, G * T, D).transpose(1, 2).reshape(B, Hkv, G * T, D)
    s["out"].copy_(out.view(s["out"].shape))
    s["lse"].copy_((m + torch.log(z)).view(s["lse"].shape))
    if c["mass"]:
        s["mass"][:, :, :N] += w[-1].sum((2, 3))


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
    rows = kept.unsqueeze(-1).expand(-1, -1, -1, c["D"])
    for k in "KV":
        s[k][:, :, :n] = s[k].gather(2, rows)
    s["mass"][:, :, :n] = s["mass"].gather(2, kept)
    s["mass"][:, :, n:N] = 0.0
    s["kept"].copy_(kept)


# ---- one pass ---------------------------------------------------------------------
def _own_dims(c):
    import paper_2609_04971_amd as bkv
    return bkv.dims(B=c["B"], Hq=c.get("Hq", c["Hkv"]), Hkv=c["Hkv"], D=c["D"], N=c["N"], N_cap=c["N"] + c["cap"], W=c.get("W", 0), C=0,
                    budget=c.get("budget", 1), n_prefix=c.get("n_prefix", 0), dtype=c["dtype"])


def _own_attend(c, s):
    import paper_2609_04971_amd as bkv
    groups = c.get("groups", 0)
    if "ws" not in s:  # kept from call to call, as a decoding loop does
        s["d"] = _own_dims(c)
        s["ws"] = bkv.attend_workspace(s["d"], T=c["T"], mass=c["mass"], groups=groups, P_cap=c.get("P", 0))
    kw = {"lens": s["lens"], "lse": s["lse"], "mass": s["mass"], "causal": c["causal"]}
    if groups:
        bkv.attend_shared(s["d"], s["q"], s["PK"], s["PV"], s["K"], s["V"], s["out"], s["ws"], p_lens=s["p_lens"], **kw)
    else:
        bkv.attend(s["d"], s["q"], s["K"], s["V"], s["out"], s["ws"], **kw)


def _own_evict(c, s):
    import paper_2609_04971_amd as bkv
    if "ws" not in s:
        s["d"] = _own_dims(c)
        s["ws"] = bkv.mass_workspace(s["d"])
    bkv.evict_mass(s["d"], s["K"], s["V"], s["mass"], s["ws"], kept=s["kept"], fill=c["fill"])


def _bits(t):
    """The same memory as whole numbers: rows are moved, not computed."""
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


def _write_rows(c, s):
    """The tokens that came since the last eviction, and their weight."""
    n, N = min(c["N"], c["budget"]), c["N"]
    if n < N:
        t = s["turn"] % s["turns"]
        s["turn"] += 1
        for k in ("K", "V", "mass"):
            s[k][:, :, n:N] = s["more_" + k][t]


def run(s):
    c = s["case"]
    if c["kind"] == "evict":
        _write_rows(c, s)
        (_own_evict if own else _plain_evict)(c, s)
        return {"K": _bits(s["K"]), "V": _bits(s["V"]), "mass": _bits(s["mass"]), "kept": s["kept"]}
    (_own_attend if own else _plain_attend)(c, s)
    return {"out": s["out"], "lse": s["lse"], "mass": s["mass"]}


# ---- what a pass cannot do without -----------------------------------------------
def work(case):
    c = case
    es, D, Hkv = (2 if c["dtype"] == "bf16" else 4), c["D"], c["Hkv"]
    if c["kind"] == "evict":
        P, N, n = c["B"] * Hkv, c["N"], min(c["budget"], c["N"])
        moved = min(n, N - n) if c["fill"] else n  # rows that change place: at most the ones past the budget, or nearly all
        written = 2 * P * (N - n) * (2 * D * es + 4)  # the tokens that came, in and into the cache
        return {"bytes": written + P * (4 * N + 4 * n + 4 * N) + 2 * 2 * P * (moved if N > n else 0) * D * es, "flops": 0}
    T, N, B, Hq = c["T"], c["N"], c["B"], c["Hq"]
    seen = _visible(c)
    pairs = seen * T - (B * T * (T - 1) // 2 if c["causal"] else 0)  # (query, token) of one query head
    flops = 4 * Hq * pairs * D
    nbytes = 2 * seen * Hkv * D * es + 2 * B * Hq * T * D * es + 4 * B * Hq * T + (8 * seen * Hkv if c["mass"] else 0)
    if c["kind"] == "shared":
        keys = c["groups"] * c["P"] * (3 if c["P_ragged"] else 4) // 4
        flops += 4 * Hq * (B // c["groups"]) * T * keys * D
        nbytes += 2 * keys * Hkv * D * es
    return {"bytes": nbytes, "flops": max(0, flops)}


# ---- the same in 64 bits --------------------------------------------------------------
def exact(case, seed):
    """Head by head, from softmax's definition with the normaliser as a logarithm."""
    c = dict(case)
    if c["kind"] == "evict":
        return None  # indices and moved rows only
    s = prepare(c, seed)
    B, Hkv, D, T, N = c["B"], c["Hkv"], c["D"], c["T"], c["N"]
    G, groups = c["Hq"] // Hkv, c.get("groups", B)
    t = torch.arange(T, device=DEV).repeat(G)
    out, lse = torch.zeros(B, Hkv, G * T, D, dtype=torch.float64, device=DEV), torch.empty(B, Hkv, G * T, dtype=torch.float64, device=DEV)
    mass = s["mass"].double() if c["mass"] else None
    lens = s["lens"].tolist() if s["lens"] is not None else [N] * B
    p_lens = s["p_lens"].tolist() if s.get("p_lens") is not None else [c.get("P", 0)] * groups
    for b in range(B):
        n, p = lens[b], p_lens[b * groups // B] if c["kind"] == "shared" else 0
        last = (n - T + t if c["causal"] else torch.full_like(t, n)).view(-1, 1)  # the last token that each row sees
        hidden = torch.cat([torch.zeros(G * T, p, dtype=torch.bool, device=DEV), torch.arange(n, device=DEV) > last], dim=1)
        for h in range(Hkv):
            y = s["q"][b, h * G:(h + 1) * G].reshape(G * T, D).double()
            k, v = s["K"][b, h, :n].double(), s["V"][b, h, :n].double()
            if p:
                a = b * groups // B
                k, v = torch.cat([s["PK"][a, h, :p].double(), k]), torch.cat([s["PV"][a, h, :p].double(), v])
            l = (y @ k.T / math.sqrt(D)).masked_fill_(hidden, -INF)
            norm = torch.logsumexp(l, dim=1)
            lse[b, h] = norm
            w = torch.exp(l - norm.clamp_min(-1e300).unsqueeze(1))
            out[b, h] = w @ v
            if mass is not None:
                mass[b, h, :n] += w[:, p:].sum(0)
    return {"out": out.view(s["out"].shape), "lse": lse.view(s["lse"].shape), "mass": mass}

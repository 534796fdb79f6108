"""Inputs, calls and the 64-bit reference of attention with a window and of attention
over a 4-bit cache.  attend_ref.check holds their bounds: a 4-bit cache's values are
exact in every type that the products take, so the arithmetic is a plain cache's."""
import math

import torch

import attend_bounds
import attend_ref
import mx_ref
import paper_2609_04971_amd as bkv
from gpu_util import say

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def reference(q, K, V, N, causal=False, lens=None, scale=None, window=0, sinks=0):
    """What attend_ref.reference gives, of rows that see their windows where window is not 0; K, V [B,Hkv,cap,D]."""
    if not window:
        return attend_ref.reference(q, K, V, N, causal=causal, lens=lens, scale=scale)
    B, Hq, T, D = q.shape
    Hkv, dev = K.shape[1], q.device
    G, scale = Hq // Hkv, scale or 1.0 / math.sqrt(D)
    out, abs_v = (torch.zeros(B, Hq, T, D, dtype=torch.float64, device=dev) for _ in "ov")
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=dev)
    dl = torch.zeros(B, Hkv, dtype=torch.float64, device=dev)
    for b in range(B):
        n = N if lens is None else min(max(int(lens[b]), 0), N)
        if n == 0:
            continue
        j, p = torch.arange(n, device=dev), n - T + torch.arange(T, device=dev).unsqueeze(1)
        hidden = (j > p) | ((j <= p - window) & (j >= sinks))
        none = hidden.all(-1)
        for h in range(Hkv):
            y, k, v = q[b, h * G:(h + 1) * G].double(), K[b, h, :n].double(), V[b, h, :n].double()
            l = torch.matmul(y, k.T.contiguous()) * scale
            dl[b, h] = (torch.matmul(y.abs(), k.abs().T.contiguous()) * scale).max() * (D + 4) * attend_ref.U32
            l = l.masked_fill(hidden, -math.inf)
            w = torch.softmax(l, -1).masked_fill(none.unsqueeze(-1), 0.0)
            rows = slice(h * G, (h + 1) * G)
            out[b, rows], abs_v[b, rows] = torch.matmul(w, v), torch.matmul(w, v.abs())
            lse[b, rows] = torch.logsumexp(l, -1)
    return {"out": out, "abs_v": abs_v, "lse": lse, "dl": dl, "mass": None}


def make(B, Hkv, G, D, T, N, cap, dtype, seed, mx, q_scale=1.0, lens=None, spread=False):
    """Inputs on the GPU.  Behind a sequence lies NaN, in a 4-bit cache bytes that stand for it.  spread: values whose
    outputs show every row (attend_bounds)."""
    g = torch.Generator().manual_seed(seed)
    x = {"q": (q_scale * torch.randn(B, Hkv * G, T, D, generator=g)).to(DT[dtype]), "mass": torch.rand(B, Hkv, cap, generator=g)}
    K, V = (torch.randn(B, Hkv, cap, D, generator=g).to(DT[dtype]) for _ in "KV")
    if spread:
        attend_bounds.spread_rows(V, seed=seed)
    if mx:
        cache = [t for p in (K, V) for t in mx_ref.quantise(p)]
    for b in range(B):
        n = N if lens is None else min(max(lens[b], 0), N)
        for t in cache if mx else (K, V):
            t[b, :, n:] = 255 if mx else float("nan")
    if mx:
        x["cache"] = bkv.MxCache(*(t.cuda() for t in cache))
        x["K"], x["V"] = mx_ref.values(*x["cache"][:2]), mx_ref.values(*x["cache"][2:])
    else:
        x["K"], x["V"] = K, V
    x = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in x.items()}
    x["lens"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    return x


def call(d, x, T, causal=True, scale=0.0, with_mass=False, with_lse=True, ws=None, window=0, sinks=0):
    out = torch.full_like(x["q"], float("nan"))
    lse = torch.full(x["q"].shape[:3], float("nan"), device="cuda") if with_lse else None
    mass = x["mass"].clone() if with_mass else None
    ws = bkv.attend_workspace(d, T, with_mass) if ws is None else ws
    if "cache" in x:
        bkv.attend_mx(d, x["q"], x["cache"], out, ws, lens=x["lens"], lse=lse, mass=mass, scale=scale, causal=causal, window=window,
                      sinks=sinks)
    else:
        bkv.attend_window(d, x["q"], x["K"], x["V"], out, ws, window, sinks=sinks, lens=x["lens"], lse=lse, scale=scale)
    torch.cuda.synchronize()
    return out, lse, mass


def run_case(B, Hkv, G, D, T, N, cap, dtype, mx, causal=True, lens=None, q_scale=1.0, scale=0.0, window=0, sinks=0, spread=False):
    say(f"B{B} Hkv{Hkv} G{G} D{D} T{T} N{N}/{cap} {dtype} mx={mx} causal={causal} lens={lens} window={window}+{sinks}")
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, N_cap=cap, W=0, C=0, budget=1, dtype=dtype)
    x = make(B, Hkv, G, D, T, N, cap, dtype, N + T, mx, q_scale, lens, spread)
    with_mass = mx and not window
    ws = bkv.attend_workspace(d, T, with_mass)
    ws.fill_(0xff)  # nothing in it is read before it is written
    kw = {"causal": causal, "scale": scale, "window": window, "sinks": sinks}
    out, lse, mass = call(d, x, T, with_mass=with_mass, ws=ws, **kw)
    ref = reference(x["q"], x["K"], x["V"], N, causal, x["lens"], scale, window, sinks)
    in_type = not (spread and attend_bounds.two_terms(d, T))
    worst = attend_ref.check(ref, out, lse, mass, x["mass"], N, weights_in_type=in_type)
    # the outputs do not depend on which of them are asked for
    out2, lse2, _ = call(d, x, T, **kw)
    assert torch.equal(out2, out) and torch.equal(lse2, lse)
    out3, _, mass3 = call(d, x, T, with_mass=with_mass, with_lse=False, **kw)
    assert torch.equal(out3, out) and (mass is None or torch.equal(mass3, mass))
    say(f"  worst {worst:.3f} of the bound")
    return x, out, lse, mass

"""64-bit reference of the attention over a cache and of the eviction by mass,
and the error bounds that go with the kernels' arithmetic."""
import math

import torch

U32 = 2.0 ** -24  # half a step of fp32


def reference(q, K, V, N, causal=False, lens=None, scale=None, PK=None, PV=None, P=0, p_lens=None, groups=1):
    """q [B,Hq,T,D], K, V [B,Hkv,cap,D], PK, PV [groups,Hkv,cap,D]: a dict of
    out [B,Hq,T,D], lse [B,Hq,T], mass [B,Hkv,N], and for bounds abs_v (the
    weighted mean of |v|) and dl (the largest error of a logit in fp32:
    D products and sums of one rounding each, and the scale's)."""
    B, Hq, T, D = q.shape
    Hkv = K.shape[1]
    G = Hq // Hkv
    dev = q.device
    scale = 1.0 / math.sqrt(D) if not scale else scale
    out = torch.zeros(B, Hq, T, D, dtype=torch.float64, device=dev)
    abs_v = torch.zeros_like(out)
    lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device=dev)
    mass = torch.zeros(B, Hkv, N, dtype=torch.float64, device=dev)
    dl = torch.zeros(B, Hkv, dtype=torch.float64, device=dev)
    for b in range(B):
        n = N if lens is None else min(max(int(lens[b]), 0), N)
        a = b * groups // B
        p = 0 if PK is None else (P if p_lens is None else min(max(int(p_lens[a]), 0), P))
        for h in range(Hkv):
            y = q[b, h * G:(h + 1) * G].double()  # [G, T, D]
            k, v = K[b, h, :n].double(), V[b, h, :n].double()
            if p:
                k, v = torch.cat([PK[a, h, :p].double(), k]), torch.cat([PV[a, h, :p].double(), v])
            if p + n == 0:
                continue
            l = torch.matmul(y, k.T.contiguous()) * scale
            dl[b, h] = (torch.matmul(y.abs(), k.abs().T.contiguous()) * scale).max() * (D + 4) * U32
            if causal:
                j, t = torch.arange(n, device=dev), torch.arange(T, device=dev).unsqueeze(1)
                l[:, :, p:] = l[:, :, p:].masked_fill(j > n - T + t, -math.inf)
            m = l.amax(-1, keepdim=True).clamp_min(-1e300)
            e = torch.exp(l - m)
            z = e.sum(-1, keepdim=True)
            w = torch.where(z > 0, e / z.clamp_min(1e-300), torch.zeros_like(e))
            out[b, h * G:(h + 1) * G] = torch.matmul(w, v)
            abs_v[b, h * G:(h + 1) * G] = torch.matmul(w, v.abs())
            lse[b, h * G:(h + 1) * G] = torch.where(z > 0, m + torch.log(z), torch.full_like(z, -math.inf)).squeeze(-1)
            mass[b, h, :n] = w[:, :, p:].sum((0, 1))
    return {"out": out, "abs_v": abs_v, "lse": lse, "mass": mass, "dl": dl}


def check(ref, out, lse, mass, mass_before, N, weights_in_type=True):
    """Bounds, per element, from the arithmetic:
      lse   the logits' error dl, a sum of at most 2^12 sequential additions
            (U32 each; longer sums are split), exp2 and log2 to 2 steps, and
            the roundings of m, l log2(e) and the result, each relative to |lse|;
      out   the same error of every weight twice (numerator and normaliser),
            the weights' rounding to the cache's type where they enter a
            matrix product in it, both against the weighted mean of |v|, and
            the result's own rounding;
      mass  every weight's error, and a rounding of the sum for every row."""
    B, Hq, T, D = out.shape
    Hkv = ref["dl"].shape[1]
    G = Hq // Hkv
    dl = ref["dl"].repeat_interleave(G, 1)[:, :, None]
    r = ref["lse"]
    empty = torch.isneginf(r)
    assert torch.equal(torch.isneginf(lse), empty), "rows that see nothing"
    assert not out[empty].float().any(), "out of a row that sees nothing"
    sums = 4096 * U32
    size = torch.where(empty, torch.zeros_like(r), r.abs())
    e_l = dl + sums + 8 * U32 * (1 + size)
    err = torch.where(empty, torch.zeros_like(r), (lse.double() - r).abs())
    assert bool((err <= e_l).all()), f"lse off by {float((err / e_l).max()):.3g} bounds"
    half = torch.finfo(out.dtype).eps / 2
    e_w = 2 * e_l.unsqueeze(-1) + (half if weights_in_type else 0.0)
    bound = half * ref["out"].abs() + e_w * (1 + half) * ref["abs_v"] + 1e-30
    err = (out.double() - ref["out"]).abs()
    assert bool((err <= bound).all()), f"out off by {float((err / bound).max()):.3g} bounds"
    worst = float((err / bound).max()) if err.numel() else 0.0
    if mass is not None:
        e = e_l.view(B, Hkv, G * T).amax(-1, keepdim=True) * 2
        want = mass_before[:, :, :N].double() + ref["mass"]
        bound = ref["mass"] * (e + (G * T + 4) * U32) + 2 * U32 * want.abs() + 1e-30
        err = (mass[:, :, :N].double() - want).abs()
        assert bool((err <= bound).all()), f"mass off by {float((err / bound).max()):.3g} bounds"
        assert torch.equal(mass[:, :, N:], mass_before[:, :, N:]), "mass behind the cache"
    return worst


def evict(K, V, mass, N, budget, W, n_prefix, fill):
    """(K, V, mass, kept) after the eviction, of one-dimensional lists of heads
    [P, cap, ...] on the host."""
    K, V, mass = K.clone(), V.clone(), mass.clone()
    Pn, n = K.shape[0], min(budget, N)
    kept = torch.arange(n, dtype=torch.int32).repeat(Pn, 1)
    if N <= budget:
        return K, V, mass, kept
    for h in range(Pn):
        m = mass[h, :N].tolist()
        middle = sorted(range(n_prefix, N - W), key=lambda j: (-m[j], j))[:budget - n_prefix - W]
        keep = sorted([*range(n_prefix), *middle, *range(N - W, N)])
        if fill:
            inside = set(j for j in keep if j < n)
            past = iter(j for j in keep if j >= n)
            keep = [j if j in inside else next(past) for j in range(n)]
        idx = torch.tensor(keep)
        K[h, :n], V[h, :n], mass[h, :n] = K[h, idx], V[h, idx], mass[h, idx]
        mass[h, n:N] = 0.0
        kept[h] = idx.int()
    return K, V, mass, kept

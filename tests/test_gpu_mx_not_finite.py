"""Infinities and NaNs on their way through a 4-bit cache: their block is stored as the byte
that stands for NaNs, read back as NaNs, and shows in the attention of its head."""
import math

import pytest
import torch

import mx_ref
import paper_2609_04971_amd as bkv
from attend_more import call, make
from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
KINDS = {"nan": [math.nan], "-nan": [-math.nan], "inf": [math.inf], "-inf": [-math.inf], "both": [math.inf, math.nan], "all": [math.nan] * 32}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", list(KINDS))
def test_stored_and_read_back(kind, D, dtype):
    say(f"{kind} D{D} {dtype}")
    B, Hkv, T = 2, 3, 40
    d = bkv.dims(B=B, Hq=Hkv, Hkv=Hkv, D=D, N=0, N_cap=T, W=0, C=0, budget=1, dtype=dtype)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(B, Hkv, T, D, generator=g).to(DT[dtype]) for _ in "kv")
    if dtype == "fp32":  # the smallest and the largest payloads of a NaN
        k[1, 2, 39, 40] = torch.tensor(0x7F800001, dtype=torch.int32).view(torch.float32)
        v[1, 2, 39, 40] = torch.tensor(-1, dtype=torch.int32).view(torch.float32)
    x = torch.tensor(KINDS[kind])
    for t, at in ((k, 0), (v, 1)):  # each place of a block, in blocks that come first and last
        for p in range(33 - len(x)):
            t[at, p % Hkv, p, D - 32 * (1 + p % 2):][p:p + len(x)] = x.to(t.dtype)
    c = bkv.mx_cache(d)
    bkv.store_mx(d, k.cuda(), v.cuda(), c)
    k2, v2 = torch.empty_like(k).cuda(), torch.empty_like(v).cuda()
    bkv.load_mx(d, c, k2, v2)
    for y, codes, scales, back in ((k, c.K, c.KS, k2), (v, c.V, c.VS, v2)):
        bad = ~y.isfinite().unflatten(-1, (-1, 32)).all(-1)
        assert int(bad.sum()) == 33 - len(x) + (dtype == "fp32")
        n, e = mx_ref.quantise(torch.where(bad.repeat_interleave(32, -1), torch.zeros(()).to(y.dtype), y))
        e[bad] = 255
        assert torch.equal(codes.cpu(), n) and torch.equal(scales.cpu(), e)
        want = mx_ref.values(n, torch.where(bad, 127, e))
        want[bad.repeat_interleave(32, -1)] = math.nan
        assert torch.equal(back.cpu().double().nan_to_num(1e300), want.nan_to_num(1e300))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 6, 10, 16, 40])  # one to four row tiles, tiles
def test_shows_in_the_attention_of_its_head(T, D, dtype):
    say(f"T{T} D{D} {dtype}")
    N, G = 300, 4
    d = bkv.dims(B=2, Hq=2 * G, Hkv=2, D=D, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = make(2, 2, G, D, T, N, N, dtype, 3, True)
    row = torch.ones(2, 2, 1, D, dtype=DT[dtype], device="cuda")

    def with_row(side, row):  # the case with a token's key or value of one head taken from `row`
        y = dict(x, cache=bkv.MxCache(*(t.clone() for t in x["cache"])))
        one = bkv.MxCache(*(t[:, :, 150:151].contiguous() for t in y["cache"]))
        bkv.store_mx(d.replace(N=0, N_cap=1), row if side == "K" else None, row if side == "V" else None, one)
        for t, s in zip(y["cache"], one):
            t[1, 0, 150] = s[1, 0, 0]
        return call(d, y, T, causal=False, with_mass=True)

    bad = row.clone()
    bad[1, 0, 0, D - 1] = math.nan
    for side in "KV":
        want = with_row(side, row)
        out, lse, mass = with_row(side, bad)
        for got, ref, axis in ((out, want[0], G), (lse, want[1], G), (mass, want[2], 1)):
            assert ref.isfinite().all()
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1, axis:], ref[1, axis:])
        if side == "K":
            assert out[1, :G].isnan().all() and lse[1, :G].isnan().all() and mass[1, 0].isnan().all()
        else:
            assert out[1, :G, :, D - 32:].isnan().all() and torch.equal(out[1, :G, :, :D - 32], want[0][1, :G, :, :D - 32])
            assert torch.equal(lse, want[1]) and torch.equal(mass, want[2])

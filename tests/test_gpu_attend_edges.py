"""Edges of the attention over the cache that the sweep of sizes and layouts
does not reach: values near fp32's range, ragged prompts, and bounds tight
enough that a single misplaced or missing row of V shows."""
import pytest
import torch

import attend_bounds
import attend_ref
import paper_2609_04971_amd as bkv
from gpu_util import say
from test_gpu_attend import call, make, ref_of

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _rising(B, Hkv, G, D, T, N, dtype, rise, v_max, seed):
    """One key in 64 has a logit `rise` above all others', from the second tile
    on; values of size v_max."""
    x = make(B, Hkv, G, D, T, N, N, dtype, seed)
    x["q"].zero_()
    x["q"][..., 0] = 8.0
    x["K"].zero_()
    x["K"][:, :, 70::64, 0] = rise / 8.0  # scale 1
    g = torch.Generator().manual_seed(seed)
    x["V"] = (v_max * (0.5 + 0.5 * torch.rand(B, Hkv, N, D, generator=g))).to(DT[dtype]).cuda()
    return x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("rise", [0.0, 4.0, 6.9, 16.5])
@pytest.mark.parametrize("N", [64, 1000, 9000])
def test_values_near_the_range_of_fp32(N, rise, T, dtype):
    """bkv.h: |v| (keys + 128) up to 2^122 gives finite results.  The output is
    a weighted mean of values, so it is bounded as any other's."""
    v_max = 2.0 ** 122 / (N + 128)
    say(f"N{N} T{T} rise {rise} {dtype} values {v_max:.3g}")
    x = _rising(2, 2, 4, 128, T, N, dtype, rise, v_max, seed=N)
    d = bkv.dims(B=2, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1, dtype=dtype)
    out, lse, mass = call(d, x, T, scale=1.0)
    assert out.isfinite().all()
    attend_ref.check(ref_of(x, N, scale=1.0), out, lse, mass, x["mass"], N)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 40])
def test_arrays_that_touch(T, dtype):
    """Everything in one allocation, each array at the last one's end."""
    B, Hkv, G, D, N = 2, 2, 4, 64, 300
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = make(B, Hkv, G, D, T, N, N, dtype, seed=4, lens=[300, 77])
    want = call(d, x, T)
    parts = [x["q"], x["K"], x["V"], x["mass"], want[0], want[1], x["lens"].repeat(32), bkv.attend_workspace(d, T, True)]  # whole vectors
    store = torch.zeros(sum(p.nbytes for p in parts), dtype=torch.uint8, device="cuda")
    cut = []
    for p, raw in zip(parts, store.split([p.nbytes for p in parts])):
        cut.append(raw.view(p.dtype).view(p.shape))
        cut[-1].copy_(p)
    q, K, V, mass, out, lse, lens, ws = cut
    out.zero_(), lse.zero_()
    bkv.attend(d, q, K, V, out, ws, lens=lens[:B], lse=lse, mass=mass)
    assert all(torch.equal(a, b) for a, b in zip((out, lse, mass), want))
    for bad in (dict(out=q), dict(lse=mass.view(-1)[1:1 + lse.numel()].view(lse.shape)), dict(ws=K.view(-1).view(torch.uint8))):
        kw = dict(out=out, lse=lse, ws=ws) | bad
        with pytest.raises(bkv.BkvError) as e:
            bkv.attend(d, q, K, V, kw["out"], kw["ws"], lens=lens[:B], lse=kw["lse"], mass=mass)
        assert e.value.status in (bkv.ERR_INVALID, bkv.ERR_WORKSPACE)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,Hkv,G,T,cap", [(350, 3, 4, 1, 700), (520, 2, 8, 2, 900), (520, 2, 5, 1, 4096), (6, 2, 4, 1, 120)])
def test_nothing_is_written_behind_the_workspace(B, Hkv, G, T, cap, dtype):
    """Weights of heads that are never split, whose logits stay in LDS, and of some whose do not."""
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=64, N=cap, W=0, C=0, budget=1, dtype=dtype)
    n = int(bkv.lib().bkv_attend_workspace_bytes(d, T, 1, 0, 0))
    store = torch.full((n + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    for N in (cap, cap // 3):
        say(f"B{B} Hkv{Hkv} G{G} T{T} N{N}/{cap} {dtype}, workspace of {n} bytes")
        x = make(B, Hkv, G, 64, T, N, cap, dtype, seed=N)
        got = call(d.replace(N=N), x, T, causal=True, ws=store[:n])
        attend_ref.check(ref_of(x, N, True), *got, x["mass"], N)
        assert (store[n:] == 0xAB).all()


def spread(B, Hkv, G, D, T, N, cap, dtype, causal=False, lens=None, groups=0, P=0, P_cap=0, p_lens=None, tiled_prefix=False, seed=0):
    """A call whose outputs show every row of V: attend_bounds."""
    say(f"B{B} Hkv{Hkv} G{G} D{D} T{T} N{N}/{cap} {dtype} causal={causal} lens={lens} groups={groups} P={P} {p_lens}")
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, N_cap=cap, W=0, C=0, budget=1, dtype=dtype)
    x = make(B, Hkv, G, D, T, N, cap, dtype, seed=N + T + seed, lens=lens, groups=groups, P=P, P_cap=P_cap, p_lens=p_lens)
    attend_bounds.spread_rows(x["V"], first=P, seed=seed)
    for b in range(B):
        x["V"][b, :, N if lens is None else min(max(lens[b], 0), N):] = float("nan")
    if groups:
        attend_bounds.spread_rows(x["PV"], seed=seed + 1)
        for a in range(groups):
            x["PV"][a, :, P if p_lens is None else min(max(p_lens[a], 0), P):] = float("nan")
    ws = bkv.attend_workspace(d, T, True, groups, P_cap)
    ws.fill_(0xff)
    out, lse, mass = call(d, x, T, causal, P=P, ws=ws)
    worst = attend_bounds.check(d, T, ref_of(x, N, causal, P=P), out, lse, mass, x["mass"], N, tiled_prefix)
    say(f"  worst {worst:.3f} of the bound")
    return ws


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (3, 7), (8, 4), (9, 4), (60, 2), (130, 4)])
@pytest.mark.parametrize("N", [17, 128, 700, 1111, 4097, 5000])
def test_every_row_of_v_counts(N, T, G, D, dtype):
    # one split and several, both kernels, whole tiles and pieces of one
    spread(1, 2, G, D, T, N, N + N % 3, dtype, causal=T <= N)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kw", [
    dict(B=4, Hkv=2, G=4, D=128, T=1, N=61, cap=64, groups=1, P=700, P_cap=700),
    dict(B=6, Hkv=2, G=2, D=64, T=2, N=100, cap=128, groups=3, P=333, P_cap=400, causal=True, lens=[0, 1, 2, 99, 100, 50], p_lens=[333, 0, 17]),
    dict(B=64, Hkv=4, G=4, D=128, T=1, N=9, cap=9, groups=2, P=2000, P_cap=2048, p_lens=[2000, 129], tiled_prefix=False),
    dict(B=64, Hkv=4, G=4, D=128, T=1, N=9, cap=9, groups=2, P=4200, P_cap=4200, p_lens=[4200, 129], tiled_prefix=True),
    dict(B=16, Hkv=8, G=4, D=128, T=1, N=300, cap=300, groups=1, P=9000, P_cap=9001, lens=[300 - 20 * i for i in range(16)], tiled_prefix=True),
    dict(B=8, Hkv=8, G=4, D=64, T=1, N=3000, cap=3100, lens=[3000, 1, 2999, 0, 64, 1500, 128, 129]),
])
def test_every_row_of_v_counts_of_prefixes_and_ragged_batches(kw, dtype):
    spread(dtype=dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,T,lens,splits,parts", [
    (300, 300, [300, 75, 1, 0], False, True),          # prompts padded to the longest
    (1500, 600, [1500, 599, 130, 400], True, True),    # lengths below the queries': their first rows see nothing
    (1500, 600, [601, 1499, 2 ** 31 - 1, -5], True, True),
    (4000, 500, [4000, 2100, 501, 64], True, True),    # chunks, a fifth of the keys and less
    (700, 130, [700, 129, 131, 333], False, True),
    (2000, 64, [2000, 64, 63, 1025], True, False),
])
def test_ragged_prompts(N, T, lens, splits, parts, D, dtype):
    ws = spread(4, 2, 4, D, T, N, N + 3, dtype, causal=True, lens=lens)
    # partials are the workspace's first region, the parts' sums its last: the fill is gone where they were taken (whether
    # the other prompts are split depends on D)
    if splits and dtype == "bf16":
        assert (ws[:4096] != 0xff).any()
    if parts:
        assert (ws[-(1 << 20):] != 0xff).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kw", [
    dict(B=3, Hkv=2, G=3, D=128, T=400, N=400, cap=400, lens=[400, 33, 256]),                  # not causal
    dict(B=2, Hkv=1, G=7, D=64, T=290, N=1300, cap=1301, causal=True, lens=[1300, 288]),
    dict(B=3, Hkv=1, G=1, D=128, T=1030, N=1030, cap=1030, causal=True, lens=[1030, 515, 2]),  # one head, many queries
    dict(B=9, Hkv=2, G=4, D=128, T=256, N=256, cap=256, causal=True, lens=[256, 0, 1, 63, 64, 65, 127, 128, 255]),
    dict(B=4, Hkv=2, G=4, D=128, T=150, N=900, cap=900, causal=True, lens=[900, 149, 0, 450], groups=2, P=700, P_cap=701,
         p_lens=[700, 63], tiled_prefix=True),
    dict(B=4, Hkv=1, G=4, D=64, T=200, N=200, cap=200, causal=True, lens=[200, 199, 1, 0], groups=1, P=2000, P_cap=2000, tiled_prefix=True),
])
def test_ragged_prompts_of_other_layouts(kw, dtype):
    spread(dtype=dtype, **kw)


@pytest.mark.parametrize("groups", [0, 2])
def test_arrays_of_no_tokens_meet_nothing(groups):
    """With N (and P) 0 nothing of the cache, the prefix or the masses is touched, wherever they lie."""
    B, H, T, D, cap = 2, 2, 8, 64, 2
    store = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    out = store[:B * H * T * D].view(B, H, T, D).fill_(1.0)
    K = store[512:512 + B * H * cap * D].view(B, H, cap, D)  # within out
    mass = store[256:256 + 2 * B * H * cap].view(torch.float32).view(B, H, cap)
    q = torch.randn(B, H, T, D, device="cuda").bfloat16()
    d = bkv.dims(B=B, Hq=H, Hkv=H, D=D, N=0, N_cap=cap, W=0, C=0, budget=1)
    ws = bkv.attend_workspace(d, T, True, groups, cap if groups else 0)
    if groups:
        bkv.attend_shared(d, q, K, K, K, K, out, ws, P=0, mass=mass)
    else:
        bkv.attend(d, q, K, K, out, ws, mass=mass)
    assert not out.float().any()

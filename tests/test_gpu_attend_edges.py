"""Edges of the attention over the cache that the sweep of sizes and layouts
does not reach: values near fp32's range, ragged prompts, and bounds tight
enough that a single misplaced or missing row of V shows."""
import pytest
import torch

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

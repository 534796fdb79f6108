"""Rows into the 4-bit cache and out of it (bkv_store_mx, bkv_load_mx) against the
64-bit reference, bit for bit: types, ties and powers of two, positions of every
sequence's own, rows that fall outside, one side alone, streams and graphs."""
import pytest
import torch

import mx_ref
import paper_2609_04971_amd as bkv
from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make(B, Hkv, D, cap, dtype, seed=0, T=1, spread=3.0):
    d = bkv.dims(B=B, Hq=Hkv, Hkv=Hkv, D=D, N=0, N_cap=cap, W=0, C=0, budget=1, dtype=dtype)
    g = torch.Generator().manual_seed(seed)
    k, v = ((torch.randn(B, Hkv, T, D, generator=g) * torch.exp(spread * torch.randn(B, Hkv, T, D, generator=g))).to(DT[dtype])
            for _ in "kv")
    c = bkv.MxCache(*(torch.randint(0, 256, (B, Hkv, cap, n), generator=g, dtype=torch.uint8) for n in (D // 2, D // 32) * 2))
    return d, k, v, c


def gpu(c):
    return bkv.MxCache(*(t.cuda() for t in c))


def expected(k, v, c, at):
    """The cache after the rows are stored, on the CPU."""
    want = bkv.MxCache(*(t.clone() for t in c))
    cap = c.K.shape[2]
    for x, codes, scales in ((k, want.K, want.KS), (v, want.V, want.VS)):
        if x is None:
            continue
        n, e = mx_ref.quantise(x)
        for b in range(x.shape[0]):
            for t in range(x.shape[2]):
                p = at[b] + t
                if 0 <= p < cap:
                    codes[b, :, p], scales[b, :, p] = n[b, :, t], e[b, :, t]
    return want


def same(a, b):
    return all(torch.equal(x.cpu(), y.cpu()) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,Hkv,T,cap,first", [(1, 1, 1, 1, 0), (3, 2, 1, 7, 6), (2, 3, 5, 9, 4), (2, 2, 130, 131, 0), (1, 8, 33, 64, 31)])
def test_store_and_load(dtype, D, B, Hkv, T, cap, first):
    say(f"{dtype} D{D} B{B} Hkv{Hkv} T{T} cap{cap} first{first}")
    d, k, v, c = make(B, Hkv, D, cap, dtype, T=T)
    x = gpu(c)
    bkv.store_mx(d, k.cuda(), v.cuda(), x, first)
    assert same(x, expected(k, v, c, [first] * B))
    k2, v2 = torch.full_like(k, 7).cuda(), torch.full_like(v, 7).cuda()
    bkv.load_mx(d, x, k2, v2, first)
    for y, codes, scales in ((k2, x.K, x.KS), (v2, x.V, x.VS)):
        assert torch.equal(y.double(), mx_ref.values(codes, scales)[:, :, first:first + T])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_border(dtype):
    # ties, their neighbours and saturation at powers of two from the least to the most
    b = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], dtype=torch.float64)
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    mags = torch.cat([b, b * (1 - step), b * (1 + step), torch.zeros(1, dtype=torch.float64)])
    rows = []
    for e in list(range(-149, -118)) + [-1, 0, 1, 30] + list(range(120, 126)):
        for top in (3.52, 4.0, 6.0, 7.0, 7.03125):
            r = torch.zeros(64, dtype=torch.float64)
            r[:28], r[28:31] = mags, torch.tensor([top, -top, -0.0])
            r[32:60], r[60] = -mags, top
            rows.append(r * 2.0 ** e)
    x = torch.stack(rows).view(1, 1, -1, 64)
    x = x.clamp(-3.38e38, 3.38e38).to(DT[dtype])
    d, _, _, c = make(1, 1, 64, x.shape[2], dtype)
    y = gpu(c)
    bkv.store_mx(d, x.cuda(), x.cuda(), y)
    assert same(y, expected(x, x, c, [0]))


def test_zeros_and_signs():
    d, k, v, c = make(1, 1, 128, 4, "fp32", T=4)
    k[0, 0, 0] = 0.0
    k[0, 0, 1] = -0.0
    k[0, 0, 2, 5:] = 0.0
    y = gpu(c)
    bkv.store_mx(d, k.cuda(), v.cuda(), y)
    assert same(y, expected(k, v, c, [0]))
    assert y.KS[0, 0, 0].tolist() == [3] * 4 and int(y.K[0, 0, 0].sum()) == 0


def test_what_is_not_finite_stays_in_its_block():
    d, k, v, c = make(1, 2, 128, 3, "bf16", T=3)
    k[0, 1, 1, 40] = float("inf")
    k[0, 1, 1, 41] = float("nan")
    y = gpu(c)
    bkv.store_mx(d, k.cuda(), v.cuda(), y)
    k[0, 1, 1, 32:64] = 0
    want = expected(k, v, c, [0])
    got = [t.cpu() for t in y]
    got[0][0, 1, 1, 16:32], got[1][0, 1, 1, 1] = want.K[0, 1, 1, 16:32], want.KS[0, 1, 1, 1]
    assert same(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 6])
def test_positions_of_each_sequence(dtype, T):
    # before the start, across it, inside, across the end, far outside both ways
    at = [-T - 3, -1, 0, 5, 17 - T, 17, 18, -2 ** 31, 2 ** 31 - 1]
    d, k, v, c = make(len(at), 2, 64, 17, dtype, T=T)
    x, p = gpu(c), torch.tensor(at, dtype=torch.int32, device="cuda")
    bkv.store_mx(d, k.cuda(), v.cuda(), x, p)
    assert same(x, expected(k, v, c, at))
    k2, v2 = torch.full_like(k, 7).cuda(), torch.full_like(v, 7).cuda()
    bkv.load_mx(d, x, k2, v2, p)
    for y, codes, scales in ((k2, x.K, x.KS), (v2, x.V, x.VS)):
        want = torch.full_like(k, 7).double().cuda()
        val = mx_ref.values(codes, scales)
        for b in range(len(at)):
            for t in range(T):
                if 0 <= at[b] + t < 17:
                    want[b, :, t] = val[b, :, at[b] + t]
        assert torch.equal(y.double(), want)


def test_one_side_alone():
    d, k, v, c = make(2, 2, 128, 9, "bf16", T=4)
    x = gpu(c)
    bkv.store_mx(d, k.cuda(), None, x, 2)
    assert same(x, expected(k, None, c, [2, 2]))
    bkv.store_mx(d, None, v.cuda(), x, 3)
    assert same(x, expected(None, v, expected(k, None, c, [2, 2]), [3, 3]))
    v2 = torch.empty_like(v).cuda()
    bkv.load_mx(d, x, None, v2, 3)
    assert torch.equal(v2.double(), mx_ref.values(x.V, x.VS)[:, :, 3:7])


def test_prompt_past_2_31_coordinates_and_blocks_in_turns():
    # 2^24 + 8 rows of 128: past 2^31 coordinates, and more workgroups than a launch takes at once
    T = (1 << 24) + 8
    d = bkv.dims(B=1, Hq=1, Hkv=1, D=128, N=0, N_cap=T, W=0, C=0, budget=1)
    k = torch.empty(1, 1, T, 128, dtype=torch.bfloat16, device="cuda")
    for i in range(0, T, 1 << 20):
        k[:, :, i:i + (1 << 20)].normal_(generator=torch.Generator(device="cuda").manual_seed(i))
    x = bkv.mx_cache(d)
    bkv.store_mx(d, k, None, x)
    for i in (0, 1 << 20, (1 << 24) - 5, T - 3):
        n, e = mx_ref.quantise(k[:, :, i:i + 3].cpu())
        assert torch.equal(x.K[:, :, i:i + 3].cpu(), n) and torch.equal(x.KS[:, :, i:i + 3].cpu(), e)
    k2 = torch.empty_like(k)
    bkv.load_mx(d, x, k2, None)
    for i in range(0, T, 1 << 22):
        assert torch.equal(k2[:, :, i:i + (1 << 22)].float(), mx_ref.values(x.K[:, :, i:i + (1 << 22)], x.KS[:, :, i:i + (1 << 22)]).float())


def test_stream_and_graph():
    d, k, v, c = make(4, 2, 128, 50, "bf16", T=3)
    kg, vg, x = k.cuda(), v.cuda(), gpu(c)
    at = torch.zeros(4, dtype=torch.int32, device="cuda")
    k2, v2 = torch.zeros_like(kg), torch.zeros_like(vg)

    def step():
        bkv.store_mx(d, kg, vg, x, at)
        bkv.load_mx(d, x, k2, v2, at)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    want = expected(k, v, c, [0] * 4)
    for i in range(4):  # tokens of their own at places of their own, on every replay
        p = [i, 3 * i, 47 - i, 20]
        k, v = torch.randn(k.shape).to(k.dtype), torch.randn(v.shape).to(v.dtype)
        kg.copy_(k)
        vg.copy_(v)
        at.copy_(torch.tensor(p, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want = expected(k, v, want, p)
        assert same(x, want)
        for b in range(4):
            assert torch.equal(k2[b].cpu().double(), mx_ref.values(want.K, want.KS)[b, :, p[b]:p[b] + 3])


def test_binding_refuses():
    d, k, v, c = make(2, 2, 128, 9, "bf16", T=4)
    x, k, v = gpu(c), k.cuda(), v.cuda()
    with pytest.raises(bkv.BkvError):
        bkv.store_mx(d, k, v, x, 6)
    for bad in (k.float(), k[:1].contiguous(), k.transpose(2, 3), k[0]):
        with pytest.raises(ValueError):
            bkv.store_mx(d, bad, v, x)
    with pytest.raises(ValueError):
        bkv.store_mx(d, k, v, tuple(x))
    with pytest.raises(ValueError):
        bkv.store_mx(d, k, v, x._replace(KS=x.K))
    with pytest.raises(ValueError):
        bkv.load_mx(d, x, k, v, torch.zeros(2, dtype=torch.int64, device="cuda"))

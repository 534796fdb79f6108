"""Attention over a 4-bit cache (bkv_attend_mx) against the 64-bit reference: types,
head layouts, lengths from none to long, ragged and empty rows, what lies behind a
sequence, the weights' sums, windows, streams, graphs and offsets past 32 bits."""
import math

import pytest
import torch

import attend_ref
import mx_ref
import paper_2609_04971_amd as bkv
from attend_more import call, make, reference, run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (1, 7), (2, 8), (5, 4), (9, 7), (40, 3)])
@pytest.mark.parametrize("N", [1, 2, 31, 33, 129, 700])
def test_attend(dtype, D, T, G, N):
    run_case(2, 2, G, D, T, N, N + N % 3, dtype, True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,N", [(1, 5000), (3, 4097), (17, 1023), (130, 130), (300, 1111), (257, 256)])
@pytest.mark.parametrize("causal", [False, True])
def test_attend_longer(dtype, D, T, N, causal):
    run_case(1, 2, 4, D, T, N, N + 5, dtype, True, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (3, 7), (8, 4), (9, 4), (60, 2), (130, 4)])
@pytest.mark.parametrize("N", [17, 128, 1111, 5000])
def test_every_row_of_v_counts(N, T, G, D, dtype):
    run_case(1, 2, G, D, T, N, N + N % 3, dtype, True, causal=T <= N, spread=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 4, 50])
def test_ragged_lengths_and_rows_that_see_nothing(dtype, T):
    for window, sinks in ((0, 0), (70, 3)):
        run_case(8, 2, 4, 64, T, 500, 517, dtype, True, lens=[-7, 0, 1, 3, 33, 499, 500, 2 ** 31 - 1], window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kw", [
    dict(B=3, Hkv=1, G=71, D=64, T=1, N=1234, cap=1234, lens=[1234, 0, 777]),    # one kv-head for all
    dict(B=2, Hkv=1, G=128, D=128, T=1, N=2500, cap=2501),
    dict(B=3, Hkv=2, G=6, D=64, T=33, N=2100, cap=2100, lens=[2100, 40, 1999]),
    dict(B=2, Hkv=3, G=1, D=128, T=200, N=3100, cap=3100, lens=[199, 3100]),
    dict(B=9, Hkv=5, G=3, D=64, T=11, N=333, cap=340, lens=[333, 1, 0, 64, 65, 128, 5, 11, 12]),
    dict(B=16, Hkv=8, G=8, D=128, T=4, N=900, cap=901),
    dict(B=300, Hkv=2, G=2, D=64, T=1, N=65, cap=66),
    dict(B=3, Hkv=2, G=8, D=128, T=3, N=3000, cap=3000, lens=[3000, 100, 1777]),  # two row tiles, split
    dict(B=2, Hkv=1, G=6, D=128, T=7, N=4000, cap=4001, lens=[4000, 1333]),       # three
    dict(B=2, Hkv=1, G=9, D=64, T=7, N=4000, cap=4001, lens=[4000, 77]),          # four
    dict(B=2, Hkv=2, G=24, D=128, T=1, N=2000, cap=2000, lens=[1999, 0]),
    dict(B=64, Hkv=4, G=8, D=128, T=2, N=1500, cap=1503),                        # logits that LDS does not hold
    dict(B=4, Hkv=2, G=4, D=128, T=600, N=1500, cap=1500, lens=[1500, 599, 130, 400]),
])
def test_head_layouts_and_ragged_batches(dtype, kw):
    run_case(dtype=dtype, mx=True, **kw)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 33), (8, 5), (8, 8), (5, 13), (1, 65), (12, 8), (1, 96), (1, 97)])
def test_weights_of_rows_about_the_registers(G, T, D):
    run_case(3, 2, G, D, T, 1100, 1103, "bf16", True, lens=[1100, T - 2, 1025])
    run_case(2, 1, G, D, T, 130, 130, "bf16", True, causal=False, lens=[33, 130])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 40])
def test_large_logits_and_scale(dtype, T):
    run_case(2, 2, 4, 128, T, 900, 900, dtype, True, causal=False, q_scale=40.0)  # one key takes nearly all
    run_case(2, 2, 4, 128, T, 900, 900, dtype, True, scale=0.37)
    run_case(2, 2, 4, 128, T, 900, 900, dtype, True, causal=False, scale=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,G", [(1, 4), (6, 5), (50, 3), (300, 2)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 4), (128, 70), (2000, 200)])
def test_windows(dtype, T, G, window, sinks):
    run_case(2, 2, G, 128, T, 1700, 1701, dtype, True, window=window, sinks=sinks)
    run_case(2, 2, G, 64, T, 1700, 1701, dtype, True, window=window, sinks=sinks, lens=[1699, 40])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 4), (40, 2)])
def test_as_a_plain_cache_of_the_same_values(dtype, D, T, G):
    """Bits of attend() over a bf16 cache that holds the same values: both bounds at once."""
    d = bkv.dims(B=2, Hq=2 * G, Hkv=2, D=D, N=700, N_cap=701, W=0, C=0, budget=1, dtype=dtype)
    x = make(2, 2, G, D, T, 700, 701, dtype, 3, True)
    out, lse, mass = call(d, x, T, with_mass=True)
    K, V = (x[k].nan_to_num().to(x["q"].dtype) for k in "KV")
    o, e, m = torch.empty_like(out), torch.empty_like(lse), x["mass"].clone()
    bkv.attend(d, x["q"], K, V, o, bkv.attend_workspace(d, T, True), lse=e, mass=m, causal=True)
    ref = reference(x["q"], K, V, 700, True)
    attend_ref.check(ref, out, lse, mass, x["mass"], 700)
    attend_ref.check(ref, o, e, m, x["mass"], 700)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 40])
def test_powers_of_two_at_both_ends(dtype, T):
    """Blocks of the smallest and the largest scales: keys of 2^-124 beside some of 1, values from
    2^-100 to 6 2^110."""
    N = 300
    d = bkv.dims(B=1, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = make(1, 2, 4, 128, T, N, N, dtype, 5, True)
    c = x["cache"]
    c.KS[:, :, ::3] = 3
    c.KS[:, :, 1::3, 1] = 20
    c.VS[:, :, :, 0] = 127 + 110
    c.VS[:, :, :, 2] = 27
    x["K"], x["V"] = mx_ref.values(c.K, c.KS), mx_ref.values(c.V, c.VS)
    out, lse, mass = call(d, x, T, with_mass=True)
    assert out.isfinite().all()
    attend_ref.check(reference(x["q"], x["K"], x["V"], N, True), out, lse, mass, x["mass"], N)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,G", [(1, 4), (6, 4), (10, 4), (40, 4)])
@pytest.mark.parametrize("first,step", [(0, 0), (5, 1), (70, 1), (70, 64)])
@pytest.mark.parametrize("rise", [0.0, 4.0, 4.5, 6.5, 16.0])
@pytest.mark.parametrize("N", [64, 1000, 9000])
def test_values_near_the_range_of_fp32(N, rise, first, step, T, G, dtype):
    """bkv.h: |v| (keys + 128) up to 2^122 gives finite results, however the weights rise as the keys go by."""
    d = bkv.dims(B=1, Hq=2 * G, Hkv=2, D=128, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = make(1, 2, G, 128, T, N, N, dtype, N, True)
    c = x["cache"]
    x["q"].zero_()
    x["q"][..., 0] = 2.0 * rise  # half of it is the logit, scale 1
    c.K.zero_()
    if step:
        c.K[:, :, first::step, 0] = 1
    c.KS.fill_(127)
    c.VS.fill_(127 + int(math.log2(2.0 ** 122 / (N + 128) / 6)))
    c.V.random_(0, 256, generator=torch.Generator(device="cuda").manual_seed(N))
    c.V.bitwise_and_(0x77)  # positive: their sums are the largest
    x["K"], x["V"] = mx_ref.values(c.K, c.KS), mx_ref.values(c.V, c.VS)
    out, lse, mass = call(d, x, T, causal=False, scale=1.0, with_mass=True)
    assert out.isfinite().all()
    attend_ref.check(reference(x["q"], x["K"], x["V"], N, scale=1.0), out, lse, mass, x["mass"], N)


@pytest.mark.parametrize("T,G", [(1, 4), (6, 4), (10, 4), (40, 4)])
def test_small_fp32_queries_and_large_keys(T, G):
    """Queries near fp32's smallest normal values: their lower terms are below bf16's."""
    d = bkv.dims(B=1, Hq=2 * G, Hkv=2, D=128, N=500, W=0, C=0, budget=1, dtype="fp32")
    x = make(1, 2, G, 128, T, 500, 500, "fp32", 6, True)
    x["q"] *= 2.0 ** -118
    x["cache"].KS[:, :, :500] += 116
    x["K"] = mx_ref.values(x["cache"].K, x["cache"].KS)
    out, lse, mass = call(d, x, T, causal=False, with_mass=True)
    attend_ref.check(reference(x["q"], x["K"], x["V"], 500), out, lse, mass, x["mass"], 500)


def test_a_nan_stays_in_its_head():
    for T in (1, 40):
        d = bkv.dims(B=2, Hq=8, Hkv=2, D=128, N=300, W=0, C=0, budget=1)
        x = make(2, 2, 4, 128, T, 300, 300, "bf16", 3, True)
        want = call(d, x, T, with_mass=True)
        y = dict(x, cache=x["cache"]._replace(KS=x["cache"].KS.clone()))
        y["cache"].KS[1, 0, 150, 2] = 255
        out, lse, mass = call(d, y, T, with_mass=True)
        for got, ref, axis in ((out, want[0], 4), (lse, want[1], 4), (mass, want[2], 1)):
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1, axis:], ref[1, axis:])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_tokens_at_all(dtype):
    run_case(2, 2, 2, 128, 3, 0, 8, dtype, True)
    run_case(2, 2, 2, 128, 3, 0, 8, dtype, True, window=5, sinks=2)


@pytest.mark.parametrize("T", [1, 40])
def test_side_stream_and_captured_graph(T):
    N = 600
    d = bkv.dims(B=4, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1)
    x = make(4, 2, 4, 128, T, N, N, "bf16", 9, True)
    want = call(d, x, T, with_mass=True)
    ws = bkv.attend_workspace(d, T, True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = call(d, x, T, with_mass=True, ws=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out, lse, mass = torch.empty_like(x["q"]), torch.empty_like(want[1]), x["mass"].clone()
    graphs = []
    for _ in range(2):  # two graphs of one workspace, replayed in turn on one stream
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            bkv.attend_mx(d, x["q"], x["cache"], out, ws, lse=lse, mass=mass, causal=True)
        graphs.append(g)
    for i in range(4):
        x["q"].mul_(0.9)
        x["cache"].VS[:, :, i::4] = 120 + i
        mass.copy_(x["mass"])
        out.fill_(float("nan"))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = (out.clone(), lse.clone(), mass.clone())
        want = call(d, x, T, with_mass=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), f"replay {i}"


def test_two_streams_at_once():
    N, T = 6000, 1
    d = bkv.dims(B=1, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1)
    x = [make(1, 2, 4, 128, T, N, N, "bf16", s, True) for s in (1, 2)]
    want = [call(d, y, T) for y in x]
    ws = [bkv.attend_workspace(d, T) for _ in x]
    outs = [[(torch.empty_like(y["q"]), torch.empty_like(want[0][1])) for _ in range(10)] for y in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    for i in range(10):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                bkv.attend_mx(d, x[k]["q"], x[k]["cache"], outs[k][i][0], ws[k], lse=outs[k][i][1], causal=True)
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for got in outs[k] for a, b in zip(got, want[k]))


@pytest.mark.parametrize("T", [1, 40])
def test_heads_and_one_head_past_32_bits_of_bytes(T):
    # 80 heads of 2^20 allocated rows, 5.4 GB of codes; one head of 2^26 + 77 tokens, 4.3 GB
    for Hkv, N, cap in ((80, 300, 1 << 20), (1, (1 << 26) + 77, (1 << 26) + 77)):
        if T > 1 and Hkv == 1:
            continue  # the 64-bit reference would take 20 GB for every few rows
        d = bkv.dims(B=1, Hq=Hkv, Hkv=Hkv, D=128, N=N, N_cap=cap, W=0, C=0, budget=1)
        g = torch.Generator(device="cuda").manual_seed(1)
        c = bkv.mx_cache(d)
        for t, lo, hi in ((c.K, 0, 256), (c.KS, 126, 128), (c.V, 0, 256), (c.VS, 126, 128)):
            t[:, :, :N].random_(lo, hi, generator=g)
        q = torch.randn(1, Hkv, T, 128, generator=g, device="cuda").bfloat16()
        x = {"q": q, "cache": c, "lens": None}
        out, lse, _ = call(d, x, T, causal=False)
        n = min(N, 400)
        if Hkv > 1:
            K, V = mx_ref.values(c.K[:, :, :N], c.KS[:, :, :N]), mx_ref.values(c.V[:, :, :N], c.VS[:, :, :N])
            attend_ref.check(reference(q, K, V, N), out, lse, None, None, N)
            continue
        # in pieces, joined in 64 bits
        m, z, o = -float("inf"), 0.0, torch.zeros(128, dtype=torch.float64, device="cuda")
        a = torch.zeros_like(o)
        for i in range(0, N, 1 << 22):
            K, V = (mx_ref.values(p[0, 0, i:i + (1 << 22)], s[0, 0, i:i + (1 << 22)]) for p, s in ((c.K, c.KS), (c.V, c.VS)))
            l = torch.mv(K, q[0, 0, 0].double()) / 128 ** 0.5
            top = max(m, float(l.max()))
            f, w = torch.exp(torch.tensor(m - top, dtype=torch.float64)).item(), torch.exp(l - top)
            z, o, a, m = z * f + float(w.sum()), o * f + torch.mv(V.T.contiguous(), w), a * f + torch.mv(V.abs().T.contiguous(), w), top
        half = 2.0 ** -9 * 2  # the result's rounding and the weights' (two terms): bf16 half step 2^-8 and less
        e_l = 2.0 ** -24 * (4096 + 132 * 6 * 128)
        assert abs(float(lse) - (m + torch.log(torch.tensor(z, dtype=torch.float64)).item())) <= e_l
        assert bool(((out[0, 0, 0].double() - o / z).abs() <= half * (o / z).abs() + (2 * e_l + half) * a / z).all()), n


def test_refusals_of_the_binding():
    d = bkv.dims(B=2, Hq=4, Hkv=2, D=128, N=32, N_cap=40, W=0, C=0, budget=1)
    x = make(2, 2, 2, 128, 1, 32, 40, "bf16", 1, True)
    ws, out, c = bkv.attend_workspace(d, 1, True), torch.empty_like(x["q"]), x["cache"]
    for kw in (dict(cache=c._replace(K=c.K[:, :, :39])), dict(cache=c._replace(VS=c.VS.float())), dict(cache=tuple(c)), dict(q=x["q"][:1]),
               dict(out=out.float()), dict(lens=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(mass=x["mass"][:, :, :32])):
        a = dict(q=x["q"], cache=c, out=out, ws=ws) | kw
        with pytest.raises(ValueError):
            bkv.attend_mx(d, a.pop("q"), a.pop("cache"), a.pop("out"), a.pop("ws"), **a)
    for kw in (dict(window=-1), dict(window=5, sinks=-1), dict(window=5, mass=x["mass"].clone()), dict(ws=ws[:0], mass=x["mass"].clone())):
        with pytest.raises(bkv.BkvError):
            bkv.attend_mx(d, x["q"], c, out, kw.pop("ws", ws), **kw)

"""Attention over the cache (bkv_attend, bkv_attend_shared) against the 64-bit
reference: types, head layouts, lengths from none to long, ragged and empty
rows, what lies behind a sequence, streams, graphs and offsets past 32 bits."""
import pytest
import torch

import attend_ref
import paper_2609_04971_amd as bkv
from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make(B, Hkv, G, D, T, N, cap, dtype, seed, q_scale=1.0, lens=None, groups=0, P=0, P_cap=0, p_lens=None):
    """Inputs on the GPU; what lies behind a sequence or prefix is NaN."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(DT[dtype])  # noqa: E731
    x = {"q": (q_scale * torch.randn(B, Hkv * G, T, D, generator=g)).to(DT[dtype]), "K": r(B, Hkv, cap, D), "V": r(B, Hkv, cap, D),
         "mass": torch.rand(B, Hkv, cap, generator=g)}
    for b in range(B):
        n = N if lens is None else min(max(lens[b], 0), N)
        x["K"][b, :, n:] = float("nan")
        x["V"][b, :, n:] = float("nan")
    if groups:
        x["PK"], x["PV"] = r(groups, Hkv, P_cap, D), r(groups, Hkv, P_cap, D)
        for a in range(groups):
            n = P if p_lens is None else min(max(p_lens[a], 0), P)
            x["PK"][a, :, n:] = float("nan")
            x["PV"][a, :, n:] = float("nan")
    x = {k: v.cuda() for k, v in x.items()}
    x["lens"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    x["p_lens"] = None if p_lens is None else torch.tensor(p_lens, dtype=torch.int32, device="cuda")
    return x


def call(d, x, T, causal=False, scale=0.0, with_mass=True, with_lse=True, P=None, ws=None, out=None):
    mass = x["mass"].clone() if with_mass else None
    out = torch.full_like(x["q"], float("nan")) if out is None else out
    lse = torch.full(x["q"].shape[:3], float("nan"), device="cuda") if with_lse else None
    kw = {"lens": x["lens"], "lse": lse, "mass": mass, "scale": scale, "causal": causal}
    if "PK" in x:
        ws = bkv.attend_workspace(d, T, with_mass, x["PK"].shape[0], x["PK"].shape[2]) if ws is None else ws
        bkv.attend_shared(d, x["q"], x["PK"], x["PV"], x["K"], x["V"], out, ws, P=P, p_lens=x["p_lens"], **kw)
    else:
        ws = bkv.attend_workspace(d, T, with_mass) if ws is None else ws
        bkv.attend(d, x["q"], x["K"], x["V"], out, ws, **kw)
    torch.cuda.synchronize()
    return out, lse, mass


def ref_of(x, N, causal=False, scale=None, P=0):
    kw = {}
    if "PK" in x:
        kw = {"PK": x["PK"], "PV": x["PV"], "P": P, "p_lens": x["p_lens"], "groups": x["PK"].shape[0]}
    return attend_ref.reference(x["q"], x["K"], x["V"], N, causal=causal, lens=x["lens"], scale=scale, **kw)


def run_case(B, Hkv, G, D, T, N, cap, dtype, causal=False, lens=None, q_scale=1.0, scale=0.0, groups=0, P=0, P_cap=0, p_lens=None):
    say(f"B{B} Hkv{Hkv} G{G} D{D} T{T} N{N} cap{cap} {dtype} causal={causal} lens={lens} groups={groups} P={P}/{P_cap} {p_lens}")
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, N_cap=cap, W=0, C=0, budget=1, dtype=dtype)
    x = make(B, Hkv, G, D, T, N, cap, dtype, seed=N + T, q_scale=q_scale, lens=lens, groups=groups, P=P, P_cap=P_cap, p_lens=p_lens)
    out, lse, mass = call(d, x, T, causal, scale, P=P)
    ref = ref_of(x, N, causal, scale, P)
    worst = attend_ref.check(ref, out, lse, mass, x["mass"], N)
    # the outputs do not depend on which of them are asked for
    out2, lse2, _ = call(d, x, T, causal, scale, with_mass=False, P=P)
    assert torch.equal(out2, out) and torch.equal(lse2, lse)
    out3, _, mass3 = call(d, x, T, causal, scale, with_lse=False, P=P)
    assert torch.equal(out3, out) and torch.equal(mass3, mass)
    say(f"  worst {worst:.3f} of the bound")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,G", [(1, 1), (1, 4), (1, 7), (2, 8), (5, 4), (9, 7), (40, 3)])
@pytest.mark.parametrize("N", [1, 2, 31, 33, 129, 700])
def test_attend(dtype, D, T, G, N):
    run_case(2, 2, G, D, T, N, N + N % 3, dtype, causal=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N", [(1, 5000), (3, 4097), (17, 1023), (130, 130), (300, 1111), (257, 256)])
@pytest.mark.parametrize("causal", [False, True])
def test_attend_longer(dtype, T, N, causal):
    run_case(1, 2, 4, 128, T, N, N + 5, dtype, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 4, 50])
def test_ragged_lengths_and_rows_that_see_nothing(dtype, T):
    # lengths below 0, of 0, shorter than T (the first queries see nothing), past N
    run_case(8, 2, 4, 64, T, 500, 517, dtype, causal=True, lens=[-7, 0, 1, 3, 33, 499, 500, 2 ** 31 - 1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_kept_logits_that_do_not_fit_lds(dtype):
    run_case(2, 2, 8, 128, 4, 20000, 20000, dtype, causal=True)   # several splits
    run_case(64, 4, 8, 128, 2, 1500, 1503, dtype)                 # one


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N", [(1, 300), (1, 3000), (40, 300), (40, 3000)])
def test_a_nan_stays_in_its_head(dtype, T, N):
    d = bkv.dims(B=2, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = make(2, 2, 4, 128, T, N, N, dtype, seed=3)
    want = call(d, x, T)
    for k in "KV":
        y = dict(x, **{k: x[k].clone()})
        y[k][1, 0, N // 2, 5] = float("nan")
        out, lse, mass = call(d, y, T)
        for got, ref, axis in ((out, want[0], 4), (lse, want[1], 4), (mass, want[2], 1)):
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1, axis:], ref[1, axis:])  # the other heads
        if k == "K":
            assert out[1, :4].isnan().all() and lse[1, :4].isnan().all() and mass[1, 0].isnan().all()
        else:
            assert out[1, :4, :, 5].isnan().all() and torch.equal(lse, want[1]) and torch.equal(mass, want[2])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_tokens_at_all(dtype):
    run_case(2, 2, 2, 128, 3, 0, 8, dtype)
    d = bkv.dims(B=2, Hq=4, Hkv=2, D=128, N=0, N_cap=8, W=0, C=0, budget=1, dtype=dtype)
    out = torch.full((2, 4, 0, 128), 1.0, dtype=DT[dtype], device="cuda")
    bkv.attend(d, out, torch.empty(2, 2, 8, 128, dtype=DT[dtype], device="cuda"), torch.empty(2, 2, 8, 128, dtype=DT[dtype], device="cuda"),
               out.clone(), bkv.attend_workspace(d, 0))  # no queries


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 40])
def test_large_logits_and_scale(dtype, T):
    run_case(2, 2, 4, 128, T, 900, 900, dtype, q_scale=40.0)              # one key takes nearly all
    run_case(2, 2, 4, 128, T, 900, 900, dtype, scale=0.37, causal=True)
    run_case(2, 2, 4, 128, T, 900, 900, dtype, scale=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kw", [
    dict(B=4, Hkv=2, G=4, D=128, T=1, N=61, cap=64, groups=1, P=700, P_cap=700),
    dict(B=6, Hkv=2, G=2, D=64, T=2, N=100, cap=128, groups=3, P=333, P_cap=400, causal=True, lens=[0, 1, 2, 99, 100, 50], p_lens=[333, 0, 17]),
    dict(B=24, Hkv=1, G=7, D=128, T=1, N=37, cap=37, groups=2, P=1500, P_cap=1501, p_lens=[1500, 1]),
    dict(B=40, Hkv=2, G=4, D=128, T=1, N=130, cap=130, groups=1, P=2049, P_cap=2049),
    dict(B=2, Hkv=2, G=4, D=64, T=70, N=70, cap=70, groups=2, P=129, P_cap=129, causal=True),
    dict(B=4, Hkv=2, G=4, D=128, T=1, N=0, cap=4, groups=2, P=90, P_cap=90),
    dict(B=4, Hkv=2, G=4, D=128, T=1, N=77, cap=77, groups=2, P=0, P_cap=5),
    dict(B=4, Hkv=2, G=4, D=128, T=2, N=0, cap=4, groups=4, P=0, P_cap=5),
    dict(B=3, Hkv=1, G=1, D=128, T=1, N=1, cap=1, groups=3, P=1, P_cap=1),
    dict(B=33, Hkv=1, G=8, D=64, T=3, N=9, cap=9, groups=1, P=260, P_cap=300, causal=True),
    dict(B=64, Hkv=4, G=4, D=128, T=1, N=9, cap=9, groups=2, P=2000, P_cap=2048, p_lens=[2000, 129]),  # rows in blocks, streamed
    dict(B=64, Hkv=4, G=4, D=128, T=1, N=9, cap=9, groups=2, P=4200, P_cap=4200, p_lens=[4200, 129]),  # and in tiles
    dict(B=20, Hkv=2, G=5, D=64, T=4, N=300, cap=300, groups=4, P=100, P_cap=5000, causal=True, lens=[i * 16 for i in range(20)]),
])
def test_shared(dtype, kw):
    run_case(dtype=dtype, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_shared_is_attend_over_the_joined_cache(dtype):
    B, Hkv, G, D, P, N = 4, 2, 4, 128, 150, 60
    x = make(B, Hkv, G, D, 2, N, N, dtype, seed=5, groups=2, P=P, P_cap=P)
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, W=0, C=0, budget=1, dtype=dtype)
    out, lse, mass = call(d, x, 2, causal=True)
    y = dict(x, K=torch.cat([x["PK"].repeat_interleave(2, 0), x["K"]], 2), V=torch.cat([x["PV"].repeat_interleave(2, 0), x["V"]], 2),
             mass=torch.cat([torch.zeros(B, Hkv, P, device="cuda"), x["mass"]], 2))
    del y["PK"], y["PV"]
    full, flse, fmass = call(bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N + P, W=0, C=0, budget=1, dtype=dtype), y, 2, causal=True)
    ref = ref_of(x, N, True, P=P)
    attend_ref.check(ref, out, lse, mass, x["mass"], N)
    attend_ref.check(ref, full, flse, fmass[:, :, P:], x["mass"], N)


def test_one_workspace_serves_every_length_and_calls_repeat():
    B, Hkv, G, D, cap = 2, 2, 4, 128, 3000
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=cap, W=0, C=0, budget=1)
    ws = bkv.attend_workspace(d, 2, True)
    ws.fill_(0xff)  # NaN everywhere: nothing in it is read before it is written
    for N in (cap, 1, 700, 33, 2999):
        x = make(B, Hkv, G, D, 2, N, cap, "bf16", seed=N)
        dn = d.replace(N=N)
        out, lse, mass = call(dn, x, 2, causal=True, ws=ws)
        attend_ref.check(ref_of(x, N, True), out, lse, mass, x["mass"], N)
        again = call(dn, x, 2, causal=True, ws=ws)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse) and torch.equal(again[2], mass)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kw", [
    dict(B=3, Hkv=1, G=71, D=64, T=1, N=1234, cap=1234, lens=[1234, 0, 777]),    # one kv-head for all
    dict(B=2, Hkv=1, G=128, D=128, T=1, N=2500, cap=2501),
    dict(B=1, Hkv=1, G=33, D=128, T=1, N=4000, cap=4000),
    dict(B=3, Hkv=2, G=6, D=64, T=33, N=2100, cap=2100, causal=True, lens=[2100, 40, 1999]),
    dict(B=2, Hkv=3, G=1, D=128, T=200, N=3100, cap=3100, causal=True, lens=[199, 3100]),
    dict(B=9, Hkv=5, G=3, D=64, T=11, N=333, cap=340, causal=True, lens=[333, 1, 0, 64, 65, 128, 5, 11, 12]),
    dict(B=16, Hkv=8, G=8, D=128, T=4, N=900, cap=901, causal=True),
    dict(B=300, Hkv=2, G=2, D=64, T=1, N=65, cap=66),
    dict(B=4, Hkv=2, G=5, D=64, T=3, N=700, cap=700, causal=True, lens=[700, 2, 350, 0], groups=2, P=5000, P_cap=5003, p_lens=[4999, 64]),
    dict(B=8, Hkv=1, G=8, D=64, T=9, N=300, cap=300, causal=True, lens=[300, 9, 8, 299, 0, 1, 64, 65], groups=1, P=3001, P_cap=3001),
])
def test_head_layouts_and_ragged_batches(dtype, kw):
    run_case(dtype=dtype, **kw)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,T", [(1, 33), (8, 5), (8, 8), (5, 13), (1, 65), (12, 8), (1, 96), (1, 97)])
def test_weights_of_rows_about_the_registers(G, T, D):
    run_case(3, 2, G, D, T, 1100, 1103, "bf16", causal=True, lens=[1100, T - 2, 1025])
    run_case(2, 1, G, D, T, 130, 130, "bf16", lens=[33, 130])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 60])
def test_two_streams_at_once(dtype, T):
    """Calls in flight together, each with a workspace of its own."""
    N = 6000
    d = bkv.dims(B=1, Hq=8, Hkv=2, D=128, N=N, W=0, C=0, budget=1, dtype=dtype)
    x = [make(1, 2, 4, 128, T, N, N, dtype, seed=s) for s in (1, 2)]
    want = [call(d, y, T, causal=True) for y in x]
    ws = [bkv.attend_workspace(d, T, True) for _ in x]
    outs = [[(torch.empty_like(y["q"]), torch.empty_like(want[0][1]), y["mass"].clone()) for _ in range(10)] for y in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    for i in range(10):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                out, lse, mass = outs[k][i]
                bkv.attend(d, x[k]["q"], x[k]["K"], x[k]["V"], out, ws[k], lse=lse, mass=mass, causal=True)
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(a, b) for got in outs[k] for a, b in zip(got, want[k]))


@pytest.mark.parametrize("T,groups", [(1, 0), (40, 0), (1, 2)])
def test_side_stream_and_captured_graph(T, groups):
    B, Hkv, G, D, N = 4, 2, 4, 128, 600
    P = 300 if groups else 0
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, W=0, C=0, budget=1)
    x = make(B, Hkv, G, D, T, N, N, "bf16", seed=9, groups=groups, P=P, P_cap=P)
    want = call(d, x, T, causal=True)
    ws = bkv.attend_workspace(d, T, True, groups, P)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = call(d, x, T, causal=True, ws=ws)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out, lse, mass = torch.empty_like(x["q"]), torch.empty_like(want[1]), x["mass"].clone()
    kw = {"lse": lse, "mass": mass, "causal": True}
    graphs = []
    for _ in range(2):  # two graphs of one workspace, replayed in turn on one stream
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            if groups:
                bkv.attend_shared(d, x["q"], x["PK"], x["PV"], x["K"], x["V"], out, ws, **kw)
            else:
                bkv.attend(d, x["q"], x["K"], x["V"], out, ws, **kw)
        graphs.append(g)
    for i in range(4):
        x["q"].mul_(0.9)
        mass.copy_(x["mass"])
        out.fill_(float("nan"))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = (out.clone(), lse.clone(), mass.clone())
        want = call(d, x, T, causal=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), f"replay {i}"


@pytest.mark.parametrize("T", [1, 20])
def test_heads_past_32_bits_of_bytes(T):
    # 20 heads of 1 M allocated rows: 5 GB of keys; the last head lies past 2^32 bytes
    B, Hkv, G, D, N, cap = 1, 20, 2, 128, 300, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(1)
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=N, N_cap=cap, W=0, C=0, budget=1)
    x = {k: torch.zeros(B, Hkv, cap, D, dtype=torch.bfloat16, device="cuda") for k in "KV"}
    for k in "KV":
        x[k][:, :, :N] = torch.randn(B, Hkv, N, D, generator=g, device="cuda").bfloat16()
    x["q"] = torch.randn(B, Hkv * G, T, D, generator=g, device="cuda").bfloat16()
    x["mass"], x["lens"] = torch.zeros(B, Hkv, cap, device="cuda"), None
    out, lse, mass = call(d, x, T)
    attend_ref.check(ref_of(x, N), out, lse, mass, x["mass"], N)


def test_one_head_past_32_bits_of_bytes():
    # 17 M tokens of one head: 4.3 GB of keys
    N, D = (1 << 24) + 77, 128
    g = torch.Generator(device="cuda").manual_seed(2)
    d = bkv.dims(B=1, Hq=2, Hkv=1, D=D, N=N, W=0, C=0, budget=1)
    x = {k: torch.empty(1, 1, N, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for k in "KV"}
    x["q"] = torch.randn(1, 2, 1, D, generator=g, device="cuda").bfloat16()
    x["K"][0, 0, -3:] = 3 * x["q"][0, 0, 0]  # the last tokens take the weight
    x["mass"], x["lens"] = torch.zeros(1, 1, N, device="cuda"), None
    out, lse, mass = call(d, x, 1)
    attend_ref.check(ref_of(x, N), out, lse, mass, x["mass"], N)


def test_refusals_of_the_binding():
    d = bkv.dims(B=2, Hq=4, Hkv=2, D=128, N=32, N_cap=40, W=0, C=0, budget=1)
    x = make(2, 2, 2, 128, 1, 32, 40, "bf16", seed=1)
    ws, out = bkv.attend_workspace(d, 1, True), torch.empty_like(x["q"])
    wide = torch.empty(2, 2, 40, 256, dtype=torch.bfloat16, device="cuda")[..., ::2]
    for kw in (dict(K=wide), dict(V=x["V"].float()), dict(K=x["K"][:, :, :39]), dict(q=x["q"][:1]), dict(out=out.float()),
               dict(lens=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(mass=x["mass"][:, :, :32])):
        a = dict(q=x["q"], K=x["K"], V=x["V"], out=out, ws=ws) | kw
        with pytest.raises(ValueError):
            bkv.attend(d, a.pop("q"), a.pop("K"), a.pop("V"), a.pop("out"), a.pop("ws"), **a)
    big = bkv.dims(B=2, Hq=4, Hkv=2, D=128, N=40, N_cap=40, W=0, C=0, budget=1)
    with pytest.raises(bkv.BkvError):
        bkv.attend(big, x["q"], x["K"], x["V"], out, ws[:16], mass=x["mass"].clone())

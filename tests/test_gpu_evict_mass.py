"""Eviction by accumulated weight (bkv_evict_mass): kept indices, K, V and
mass bit for bit against the plain rule, both layouts; and a run of attention
and eviction together, as a decoding loop has them."""
import pytest
import torch

import attend_ref
import paper_2609_04971_amd as bkv
from gpu_util import host, say

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def masses(kind, P, cap, g):
    m = torch.empty(P, cap).exponential_(generator=g)
    if kind == "sinks":  # a few tokens hold nearly all, many have nothing
        m = torch.where(torch.rand(P, cap, generator=g) < 0.01, 5000 * m, 1e-6 * m)
        m[torch.rand(P, cap, generator=g) < 0.3] = 0.0
    elif kind == "equal":
        m = torch.full((P, cap), 0.25)
    elif kind == "zeros":
        m = torch.zeros(P, cap)
        m[:, ::3] = -0.0
    elif kind == "few values":
        m = torch.randint(0, 5, (P, cap), generator=g).float()
    elif kind == "near":  # neighbouring bit patterns
        m = (torch.full((P, cap), 1.0).view(torch.int32) + torch.randint(0, 3000, (P, cap), generator=g, dtype=torch.int32)).view(torch.float32)
    elif kind == "signs":
        m = torch.randn(P, cap, generator=g) * 10 ** torch.randint(-30, 30, (P, cap), generator=g).float()
    elif kind == "infinite":
        m[torch.rand(P, cap, generator=g) < 0.1] = float("inf")
        m[torch.rand(P, cap, generator=g) < 0.1] = float("-inf")
    return m


def bits(t):
    return host(t).contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def run_case(B, Hkv, D, N, cap, budget, W, n_prefix, dtype, kind, fill, kept=True):
    say(f"B{B} Hkv{Hkv} D{D} N{N}/{cap} budget {budget} W{W} prefix {n_prefix} {dtype} {kind} fill={fill}")
    P = B * Hkv
    g = torch.Generator().manual_seed(N + budget)
    m = masses(kind, P, cap, g)
    if dtype == "bf16":  # any bits: rows are copied
        K, V = (torch.randint(-32768, 32768, (P, cap, D), generator=g, dtype=torch.int16).view(torch.bfloat16) for _ in "KV")
    else:
        K, V = (torch.randint(-2 ** 31, 2 ** 31 - 1, (P, cap, D), generator=g, dtype=torch.int32).view(torch.float32) for _ in "KV")
    d = bkv.dims(B=B, Hq=Hkv, Hkv=Hkv, D=D, N=N, N_cap=cap, W=W, C=0, budget=budget, n_prefix=n_prefix, dtype=dtype)
    ws = bkv.mass_workspace(d)
    Kd, Vd, md = K.cuda().view(B, Hkv, cap, D), V.cuda().view(B, Hkv, cap, D), m.cuda().view(B, Hkv, cap)
    kd = torch.full((B, Hkv, d.n_keep), -1, dtype=torch.int32, device="cuda") if kept else None
    bkv.evict_mass(d, Kd, Vd, md, ws, kept=kd, fill=fill)
    torch.cuda.synchronize()
    assert bkv.device_status(ws) == bkv.OK
    Kr, Vr, mr, kr = attend_ref.evict(K, V, m, N, budget, W, n_prefix, fill)
    if kept:
        assert torch.equal(host(kd).view(P, -1), kr)
    for got, want in ((Kd, Kr), (Vd, Vr), (md, mr)):
        assert torch.equal(bits(got).view(want.shape), bits(want))


KINDS = ["exponential", "sinks", "equal", "zeros", "few values", "near", "signs", "infinite"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("fill", [False, True])
def test_kinds_of_masses(kind, fill):
    run_case(2, 2, 64, 1500, 1531, 700, 16, 4, "bf16", kind, fill)


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("N,cap,budget,W,n_prefix", [
    (2, 2, 1, 0, 0), (2, 2, 1, 1, 0), (65, 65, 64, 8, 0), (100, 130, 12, 8, 4),  # forced rows only
    (100, 100, 13, 8, 4), (500, 500, 499, 0, 0), (500, 501, 1, 0, 0), (1024, 1024, 896, 32, 4), (4096, 4096, 3584, 32, 4),
    (4097, 4100, 2000, 5, 1), (9000, 9000, 8999, 1, 0), (16385, 16385, 3000, 64, 0)])
def test_sizes(N, cap, budget, W, n_prefix, fill):
    for dtype, D in (("bf16", 128), ("fp32", 64), ("fp32", 128), ("bf16", 64)):
        run_case(1, 2, D, N, cap, budget, W, n_prefix, dtype, "sinks" if N % 2 else "exponential", fill)


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("N", [32768, 32769, 40000, 70001])
@pytest.mark.parametrize("kind", ["sinks", "few values"])
def test_long_heads(N, kind, fill):
    run_case(1, 2, 64, N, N + 3, N // 3, 32, 4, "bf16", kind, fill)


def test_many_heads_no_indices_asked_for():
    for fill in (False, True):
        run_case(40, 8, 64, 600, 600, 525, 16, 2, "bf16", "exponential", fill, kept=False)


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("Hkv,N,budget", [(255, 700, 600), (256, 700, 600), (256, 5000, 4600), (256, 5000, 2400), (256, 8193, 8000),
                                          (383, 4097, 3900), (384, 4097, 3900), (384, 8192, 7500), (384, 5000, 2400)])
def test_heads_around_the_many(Hkv, N, budget, fill):
    # one workgroup moves a head's rows itself from 256 heads on (384 of more than 4096 tokens), up to 8192 tokens and 2048 moves
    run_case(1, Hkv, 64, N, N + 1, budget, 8, 1, "bf16", "exponential", fill)


@pytest.mark.parametrize("fill", [False, True])
def test_within_the_budget_nothing_changes(fill):
    run_case(2, 2, 64, 100, 128, 100, 8, 2, "bf16", "exponential", fill)
    run_case(2, 2, 64, 50, 128, 100, 8, 2, "bf16", "exponential", fill)


@pytest.mark.parametrize("fill", [False, True])
def test_nan_masses_keep_an_exact_count(fill):
    d = bkv.dims(B=1, Hq=2, Hkv=2, D=64, N=800, W=8, C=0, budget=300, n_prefix=2)
    m = torch.rand(1, 2, 800, device="cuda")
    m[:, :, 5:700:3] = float("nan")
    K = torch.zeros(1, 2, 800, 64, dtype=torch.bfloat16, device="cuda")
    kept = torch.full((1, 2, 300), -1, dtype=torch.int32, device="cuda")
    bkv.evict_mass(d, K, K.clone(), m, bkv.mass_workspace(d), kept=kept, fill=fill)
    k = host(kept).sort(-1).values
    assert (k.diff(dim=-1) > 0).all() and int(k.min()) >= 0 and int(k.max()) < 800


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("kind", ["any bits", "top NaNs", "bottom NaNs"])
@pytest.mark.parametrize("Hkv,N", [(2, 800), (2, 9000), (300, 800)])
def test_masses_of_any_bits(kind, Hkv, N, fill):
    """NaNs rank by their bits: the keys' range reaches both ends of 32 bits."""
    g = torch.Generator().manual_seed(N)
    b = torch.randint(-2 ** 31, 2 ** 31, (1, Hkv, N), generator=g, dtype=torch.int64)
    if kind != "any bits":
        b = 1 + torch.randint(0, 2 ** 30, (1, Hkv, N), generator=g)   # positive, none of them 0
        b[..., ::3] = 0x7fffffff - torch.randint(0, 2 ** 18, b[..., ::3].shape, generator=g)
        b[..., 1], b[..., 6] = 1, 0x7fffffff
        if kind == "bottom NaNs":
            b -= 2 ** 31
    u = b & 0xffffffff
    key = torch.where(u >= 2 ** 31, 0xffffffff - u, u + 2 ** 31)
    key[u == 2 ** 31] = 2 ** 31                                      # -0
    budget = {"any bits": N // 3, "top NaNs": N // 6, "bottom NaNs": N - N // 6}[kind]
    d = bkv.dims(B=1, Hq=Hkv, Hkv=Hkv, D=64, N=N, W=8, C=0, budget=budget, n_prefix=2)
    key[..., :2] = key[..., N - 8:] = 2 ** 40
    want = key[0].sort(dim=-1, descending=True, stable=True).indices[:, :budget].sort(dim=-1).values
    K = torch.arange(N).float().view(1, 1, N, 1).expand(1, Hkv, N, 64).bfloat16().cuda()
    kept = torch.full((1, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    ws = bkv.mass_workspace(d)
    bkv.evict_mass(d, K, K.clone(), b.to(torch.int32).view(torch.float32).cuda(), ws, kept=kept, fill=fill)
    assert bkv.device_status(ws) == bkv.OK
    assert torch.equal(host(kept)[0].long().sort(dim=-1).values, want)


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("Hkv", [2, 300])
def test_a_workspace_stamped_for_other_dims_moves_nothing(fill, Hkv):
    d = bkv.dims(B=1, Hq=Hkv, Hkv=Hkv, D=64, N=700, W=8, C=0, budget=300, n_prefix=2)
    g = torch.Generator(device="cuda").manual_seed(8)
    K, V = (torch.randn(1, Hkv, 700, 64, generator=g, device="cuda").bfloat16() for _ in "KV")
    m = torch.rand(1, Hkv, 700, generator=g, device="cuda")
    kept = torch.full((1, Hkv, 300), -1, dtype=torch.int32, device="cuda")
    before = [t.clone() for t in (K, V, m, kept)]
    ws = bkv.mass_workspace(d)
    bkv.workspace_init(d.replace(budget=299), ws)
    bkv.evict_mass(d, K, V, m, ws, kept=kept, fill=fill)
    assert bkv.device_status(ws) == bkv.ERR_DEVICE
    assert all(torch.equal(a, b) for a, b in zip((K, V, m, kept), before))
    ws.zero_()  # never initialised
    bkv.evict_mass(d, K, V, m, ws, kept=kept, fill=fill)
    assert bkv.device_status(ws) == bkv.ERR_WORKSPACE
    assert all(torch.equal(a, b) for a, b in zip((K, V, m, kept), before))
    bkv.workspace_init(d, ws)
    bkv.evict_mass(d, K, V, m, ws, kept=kept, fill=fill)
    assert bkv.device_status(ws) == bkv.OK and not torch.equal(kept, before[3])


@pytest.mark.parametrize("fill", [False, True])
def test_captured_graph(fill):
    d = bkv.dims(B=2, Hq=4, Hkv=2, D=128, N=900, W=8, C=0, budget=600, n_prefix=2)
    g = torch.Generator(device="cuda").manual_seed(3)
    K0, V0 = (torch.randn(2, 2, 900, 128, generator=g, device="cuda").bfloat16() for _ in "KV")
    K, V, m = K0.clone(), V0.clone(), torch.zeros(2, 2, 900, device="cuda")
    kept, ws = torch.empty(2, 2, 600, dtype=torch.int32, device="cuda"), bkv.mass_workspace(d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bkv.evict_mass(d, K, V, m, ws, kept=kept, fill=fill)
    for i in range(4):
        m0 = torch.rand(2, 2, 900, generator=g, device="cuda")
        K.copy_(K0), V.copy_(V0), m.copy_(m0)
        graph.replay()
        torch.cuda.synchronize()
        Ke, Ve, me, ke = K0.clone(), V0.clone(), m0.clone(), torch.empty_like(kept)
        bkv.evict_mass(d, Ke, Ve, me, bkv.mass_workspace(d), kept=ke, fill=fill)
        for a, b in ((K, Ke), (V, Ve), (m, me), (kept, ke)):
            assert torch.equal(a, b), f"replay {i}"


@pytest.mark.parametrize("N,budget", [(700, 652), (700, 650), (4096, 3904), (4096, 3903), (4097, 4000), (4096, 100)])
def test_few_moves_of_few_heads(N, budget):
    """Both sides of the bytes that the selecting workgroup moves itself."""
    for dtype, D in (("bf16", 128), ("fp32", 128), ("bf16", 64)):
        run_case(1, 3, D, N, N + 3, budget, 16, 4, dtype, "sinks", True)


@pytest.mark.parametrize("fill", [False, True])
def test_two_streams_at_once(fill):
    d = bkv.dims(B=1, Hq=2, Hkv=2, D=128, N=5000, W=8, C=0, budget=3000, n_prefix=2)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = [[torch.randn(1, 2, 5000, 128, generator=g, device="cuda").bfloat16() for _ in "KV"]
         + [torch.rand(1, 2, 5000, generator=g, device="cuda"), torch.empty(1, 2, 3000, dtype=torch.int32, device="cuda")]
         for _ in range(16)]
    want = [[t.clone() for t in y] for y in x]
    for K, V, m, kept in want:
        bkv.evict_mass(d, K, V, m, bkv.mass_workspace(d), kept=kept, fill=fill)
    ws, streams = [bkv.mass_workspace(d) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i, (K, V, m, kept) in enumerate(x):
        with torch.cuda.stream(streams[i % 2]):
            bkv.evict_mass(d, K, V, m, ws[i % 2], kept=kept, fill=fill)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got, ref in zip(x, want) for a, b in zip(got, ref))


@pytest.mark.parametrize("compaction", ["order", "fill"])
def test_attention_and_eviction_together(compaction):
    """Two layers of two sequences decode past their budget twice: the weights
    collected step by step decide what stays, and the attention that follows
    reads what was kept."""
    LB, Hq, Hkv, D, cap, budget, W, steps = 4, 8, 2, 128, 192, 160, 8, 80  # full after 42 steps, then every 32
    g = torch.Generator().manual_seed(11)
    K, V = torch.zeros(LB, Hkv, cap, D, dtype=torch.bfloat16), torch.zeros(LB, Hkv, cap, D, dtype=torch.bfloat16)
    r = lambda *s: torch.randn(*s, generator=g).bfloat16()  # noqa: E731
    T0 = 150
    K[:, :, :T0], V[:, :, :T0], qp = r(LB, Hkv, T0, D), r(LB, Hkv, T0, D), r(LB, Hq, T0, D)
    d = bkv.dims(B=LB, Hq=Hq, Hkv=Hkv, D=D, N=T0, N_cap=cap, W=W, C=0, budget=budget, n_prefix=2)
    Kd, Vd, md = K.cuda(), V.cuda(), torch.zeros(LB, Hkv, cap, device="cuda")
    ws_p, ws, we = bkv.attend_workspace(d, T0, True), bkv.attend_workspace(d, 1, True), bkv.mass_workspace(d)
    lse, out = torch.empty(LB, Hq, T0, device="cuda"), torch.empty(LB, Hq, T0, D, dtype=torch.bfloat16, device="cuda")
    bkv.attend(d, qp.cuda(), Kd, Vd, out, ws_p, lse=lse, mass=md, causal=True)
    ref = attend_ref.reference(qp, K, V, T0, causal=True)
    attend_ref.check(ref, host(out), host(lse), host(md), torch.zeros(LB, Hkv, cap), T0)
    out, lse = torch.empty(LB, Hq, 1, D, dtype=torch.bfloat16, device="cuda"), torch.empty(LB, Hq, 1, device="cuda")
    kept = torch.empty(LB, Hkv, budget, dtype=torch.int32, device="cuda")
    N, evictions = T0, 0
    for _ in range(steps):
        k, v, q = r(LB, Hkv, D), r(LB, Hkv, D), r(LB, Hq, 1, D)
        bkv.append_rows([(Kd, N, k.cuda()), (Vd, N, v.cuda())])
        N += 1
        before = host(md)
        bkv.attend(d.replace(N=N), q.cuda(), Kd, Vd, out, ws, lse=lse, mass=md)
        ref = attend_ref.reference(q, host(Kd), host(Vd), N)
        attend_ref.check(ref, host(out), host(lse), host(md), before, N)
        if N == cap:
            pre = [host(t).view(LB * Hkv, cap, *t.shape[3:]) for t in (Kd, Vd, md)]
            bkv.evict_mass(d.replace(N=N), Kd, Vd, md, we, kept=kept, fill=compaction == "fill")
            Kr, Vr, mr, kr = attend_ref.evict(*pre, N, budget, W, 2, compaction == "fill")
            assert torch.equal(host(kept).view(-1, budget), kr)
            for a, b in ((Kd, Kr), (Vd, Vr), (md, mr)):
                assert torch.equal(bits(a).view(b.shape), bits(b))
            N, evictions = budget, evictions + 1
    assert evictions == 2

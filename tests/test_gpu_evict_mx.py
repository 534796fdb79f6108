"""Eviction of a 4-bit cache: by accumulated weight (bkv_evict_mass_mx) and from a
kept list (bkv_compact_mx), bit for bit against the plain rule; the whole of it as
a decoding loop has it: rows stored, attended to with their weights, evicted."""
import pytest
import torch

import attend_ref
import mx_ref
import paper_2609_04971_amd as bkv
from attend_more import reference
from gpu_util import host, say
from test_gpu_evict_mass import KINDS, masses

pytestmark = pytest.mark.gpu


def make(B, Hkv, D, N, cap, budget, W, n_prefix, seed):
    d = bkv.dims(B=B, Hq=Hkv, Hkv=Hkv, D=D, N=N, N_cap=cap, W=W, C=0, budget=budget, n_prefix=n_prefix)
    g = torch.Generator().manual_seed(seed)
    c = bkv.MxCache(*(torch.randint(0, 256, (B, Hkv, cap, n), generator=g, dtype=torch.uint8) for n in (D // 2, D // 32) * 2))
    return d, c, g


def joined(c):
    """Codes and bytes of a row side by side, heads in one dimension."""
    return [torch.cat([a, b], -1).flatten(0, 1) for a, b in ((c.K, c.KS), (c.V, c.VS))]


def run_case(B, Hkv, D, N, cap, budget, W, n_prefix, kind, fill, kept=True):
    say(f"B{B} Hkv{Hkv} D{D} N{N}/{cap} budget {budget} W{W} prefix {n_prefix} {kind} fill={fill}")
    d, c, g = make(B, Hkv, D, N, cap, budget, W, n_prefix, N + budget)
    m = masses(kind, B * Hkv, cap, g)
    ws, x, md = bkv.mass_workspace(d), bkv.MxCache(*(t.cuda() for t in c)), m.cuda().view(B, Hkv, cap)
    kd = torch.full((B, Hkv, d.n_keep), -1, dtype=torch.int32, device="cuda") if kept else None
    bkv.evict_mass_mx(d, x, md, ws, kept=kd, fill=fill)
    torch.cuda.synchronize()
    assert bkv.device_status(ws) == bkv.OK
    Kr, Vr, mr, kr = attend_ref.evict(*joined(c), m, N, budget, W, n_prefix, fill)
    Kg, Vg = joined(bkv.MxCache(*(host(t) for t in x)))
    assert torch.equal(Kg, Kr) and torch.equal(Vg, Vr)
    assert torch.equal(host(md).view(mr.shape).view(torch.int32), mr.view(torch.int32))
    if kept:
        assert torch.equal(host(kd).view(B * Hkv, -1), kr)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("fill", [False, True])
def test_kinds_of_masses(kind, fill):
    run_case(2, 2, 64, 1500, 1531, 700, 16, 4, kind, fill)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("N,cap,budget,W,n_prefix", [
    (1, 1, 1, 0, 0), (2, 2, 1, 0, 0), (2, 2, 1, 1, 0), (65, 65, 64, 8, 0), (100, 130, 12, 8, 4), (100, 100, 200, 8, 4), (100, 100, 13, 8, 4),
    (500, 500, 499, 0, 0), (500, 501, 1, 0, 0), (1024, 1024, 896, 32, 4), (4096, 4096, 3584, 32, 4), (4097, 4101, 2000, 5, 1),
    (9000, 9000, 8999, 1, 0), (16385, 16385, 3000, 64, 0), (33000, 33001, 28000, 8, 2)])
def test_sizes(N, cap, budget, W, n_prefix, fill, D):
    run_case(1, 3, D, N, cap, budget, W, n_prefix, "sinks" if N % 2 else "exponential", fill)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("B,N,budget", [(150, 600, 500), (150, 5000, 2600), (200, 5000, 4700), (90, 3000, 1500)])
def test_many_heads(B, N, budget, fill, D):
    # the selecting workgroup moves the rows itself, or another launch does
    run_case(B, 2, D, N, N + 3, budget, 4, 1, "sinks", fill, kept=False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,cap,budget", [(1, 1, 1), (50, 53, 50), (200, 200, 3), (1000, 1001, 875), (3000, 3000, 129), (777, 900, 1000)])
def test_compact(N, cap, budget, D):
    say(f"D{D} N{N}/{cap} budget {budget}")
    d, c, g = make(3, 2, D, N, cap, budget, 0, 0, N)
    n = min(N, budget)
    kept = torch.stack([torch.randperm(N, generator=g)[:n].sort().values for _ in range(6)]).int()
    ws, x = bkv.workspace(d, bkv.OP_COMPACT), bkv.MxCache(*(t.cuda() for t in c))
    for turn in range(2):  # the workspace as the call before has left it
        want = [t.clone() for t in joined(c)]
        for t in want:
            t[:, :n] = t.gather(1, kept.long().unsqueeze(-1).expand(-1, -1, t.shape[-1]))
        bkv.compact_mx(d, x, kept.cuda().view(3, 2, n), ws)
        assert bkv.device_status(ws) == bkv.OK
        c = bkv.MxCache(*(host(t) for t in x))
        assert all(torch.equal(a, b) for a, b in zip(joined(c), want))


def test_bad_indices_move_nothing():
    d, c, _ = make(2, 2, 128, 600, 600, 400, 0, 0, 1)
    ws, x = bkv.workspace(d, bkv.OP_COMPACT), bkv.MxCache(*(t.cuda() for t in c))
    kept = torch.arange(100, 500, dtype=torch.int32).repeat(2, 2, 1)
    kept[1, 0, 130:] = torch.arange(600, 870)  # past the cache from the second segment on
    kept[1, 1, 399] = -1
    bkv.compact_mx(d, x, kept.cuda(), ws)
    assert bkv.device_status(ws) == bkv.ERR_DEVICE
    got = [host(t) for t in x]
    for t, was in zip(got, c):
        assert torch.equal(t[0, :, :400], was[0, :, 100:500]) and torch.equal(t[:, :, 400:], was[:, :, 400:])


def test_a_workspace_that_is_not_initialised():
    d, c, g = make(2, 2, 128, 600, 600, 400, 0, 0, 1)
    x, m = bkv.MxCache(*(t.cuda() for t in c)), torch.rand(2, 2, 600, generator=g).cuda()
    for fill in (False, True):
        ws = torch.zeros_like(bkv.mass_workspace(d))
        before = m.clone()
        bkv.evict_mass_mx(d, x, m, ws, fill=fill)
        assert bkv.device_status(ws) == bkv.ERR_WORKSPACE
        assert all(torch.equal(host(a), b) for a, b in zip(x, c)) and torch.equal(m, before)


@pytest.mark.parametrize("fill", [False, True])
def test_graph(fill):
    d, c, g = make(3, 2, 128, 700, 701, 500, 8, 2, 3)
    x, ws = bkv.MxCache(*(t.cuda() for t in c)), bkv.mass_workspace(d)
    m, kept = torch.zeros(3, 2, 701, device="cuda"), torch.zeros(3, 2, 500, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bkv.evict_mass_mx(d, x, m, ws, kept=kept, fill=fill)
    for i in range(4):
        mh = torch.rand(6, 701, generator=g)
        m.copy_(mh.view(3, 2, 701))
        was = joined(bkv.MxCache(*(host(t) for t in x)))
        graph.replay()
        torch.cuda.synchronize()
        Kr, Vr, mr, kr = attend_ref.evict(*was, mh, 700, 500, 8, 2, fill)
        Kg, Vg = joined(bkv.MxCache(*(host(t) for t in x)))
        assert torch.equal(Kg, Kr) and torch.equal(Vg, Vr) and torch.equal(host(kept).view(6, -1), kr)


@pytest.mark.parametrize("fill", [False, True])
def test_late_heads_past_32_bits_of_bytes(fill):
    # 80 heads of 2^20 rows: 5.4 GB of codes
    d = bkv.dims(B=1, Hq=80, Hkv=80, D=128, N=3000, N_cap=1 << 20, W=4, C=0, budget=2500, n_prefix=1)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = bkv.mx_cache(d)
    for t in x:
        t[:, :, :3000].random_(0, 256, generator=g)
    m = torch.zeros(1, 80, 1 << 20, device="cuda")
    m[:, :, :3000] = torch.rand(1, 80, 3000, generator=g, device="cuda")
    was, mh = [t[:, 76:, :3000].cpu() for t in x], m[:, 76:, :3000].cpu()
    ws = bkv.mass_workspace(d)
    bkv.evict_mass_mx(d, x, m, ws, fill=fill)
    assert bkv.device_status(ws) == bkv.OK
    Kr, Vr, mr, _ = attend_ref.evict(*joined(bkv.MxCache(*was)), mh[0], 3000, 2500, 4, 1, fill)
    Kg, Vg = joined(bkv.MxCache(*(t[:, 76:, :3000].cpu() for t in x)))
    assert torch.equal(Kg, Kr) and torch.equal(Vg, Vr) and torch.equal(m[0, 76:, :3000].cpu(), mr)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fill", [False, True])
def test_stored_attended_to_and_evicted(dtype, fill):
    """A prompt and 100 steps at a budget of 200 of 256, every result against 64 bits."""
    B, Hkv, G, D, cap, budget = 2, 2, 4, 128, 256, 200
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(1)
    d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=cap, W=8, C=0, budget=budget, n_prefix=2, dtype=dtype)
    c, mass, ews = bkv.mx_cache(d), torch.zeros(B, Hkv, cap, device="cuda"), bkv.mass_workspace(d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    N = 0
    for T in [180] + [1] * 100:
        k, v, q = r(B, Hkv, T, D), r(B, Hkv, T, D), r(B, Hkv * G, T, D)
        bkv.store_mx(d, k, v, c, N)
        N += T
        out, lse, before = torch.empty_like(q), torch.empty(B, Hkv * G, T, device="cuda"), mass.clone()
        bkv.attend_mx(d.replace(N=N), q, c, out, bkv.attend_workspace(d, T, True), lse=lse, mass=mass, causal=True)
        n, e = mx_ref.quantise(k.cpu())
        assert torch.equal(c.K[:, :, N - T:N].cpu(), n) and torch.equal(c.KS[:, :, N - T:N].cpu(), e)
        attend_ref.check(reference(q, mx_ref.values(c.K, c.KS), mx_ref.values(c.V, c.VS), N, True), out, lse, mass, before, N)
        if N == cap:
            was, mh = joined(bkv.MxCache(*(host(t) for t in c))), host(mass).view(B * Hkv, cap)
            bkv.evict_mass_mx(d, c, mass, ews, fill=fill)
            Kr, Vr, mr, _ = attend_ref.evict(*was, mh, cap, budget, 8, 2, fill)
            Kg, Vg = joined(bkv.MxCache(*(host(t) for t in c)))
            assert torch.equal(Kg, Kr) and torch.equal(Vg, Vr) and torch.equal(host(mass).view(B * Hkv, cap), mr)
            N = budget
    assert bkv.device_status(ews) == bkv.OK


def test_refusals_of_the_binding():
    d, c, g = make(2, 2, 128, 600, 600, 400, 0, 0, 1)
    x, m, ws = bkv.MxCache(*(t.cuda() for t in c)), torch.rand(2, 2, 600).cuda(), bkv.mass_workspace(d)
    kept = torch.zeros(2, 2, 400, dtype=torch.int32, device="cuda")
    for bad in (x._replace(K=x.K[:, :, :599]), x._replace(VS=x.V), tuple(x)):
        with pytest.raises(ValueError):
            bkv.evict_mass_mx(d, bad, m, ws)
        with pytest.raises(ValueError):
            bkv.compact_mx(d, bad, kept, ws)
    with pytest.raises(ValueError):
        bkv.evict_mass_mx(d, x, m[:, :, :599], ws)
    with pytest.raises(ValueError):
        bkv.compact_mx(d, x, kept[:, :, :300], ws)
    with pytest.raises(bkv.BkvError):
        bkv.evict_mass_mx(d, x._replace(V=x.K), m, ws)
    with pytest.raises(bkv.BkvError):
        bkv.evict_mass_mx(d, x, m, ws[:64])

"""Edges of the eviction by accumulated weight: one array for K and V, and
rows past 2^32 bytes."""
import pytest
import torch

import attend_ref
import paper_2609_04971_amd as bkv
from gpu_util import host, say
from test_gpu_evict_mass import bits, masses

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("Hkv,N,budget", [(2, 700, 600), (2, 9000, 4000), (300, 700, 300)])
def test_one_array_for_keys_and_values(Hkv, N, budget, fill):
    say(f"one array: {Hkv} heads, {N} -> {budget}, fill={fill}")
    g = torch.Generator().manual_seed(N)
    K = torch.randn(Hkv, N, 64, generator=g).bfloat16()
    m = masses("sinks", Hkv, N, g)
    d = bkv.dims(B=1, Hq=Hkv, Hkv=Hkv, D=64, N=N, W=8, C=0, budget=budget, n_prefix=2)
    Kd, md, ws = K.cuda().unsqueeze(0), m.cuda().unsqueeze(0), bkv.mass_workspace(d)
    kept = torch.empty(1, Hkv, budget, dtype=torch.int32, device="cuda")
    bkv.evict_mass(d, Kd, Kd, md, ws, kept=kept, fill=fill)
    assert bkv.device_status(ws) == bkv.OK
    Kr, _, mr, kr = attend_ref.evict(K, K, m, N, budget, 8, 2, fill)
    assert torch.equal(host(kept)[0], kr) and torch.equal(bits(Kd)[0], bits(Kr)) and torch.equal(bits(md)[0], bits(mr))


def _by_sorting(K, V, mass, N, budget, W, n_prefix, fill):
    """(K, V rows below the budget, mass, kept) of one head [cap, ...], on the GPU."""
    m = mass[:N].clone()
    m[:n_prefix] = m[N - W:] = float("inf")
    kept = m.sort(descending=True, stable=True).indices[:budget].sort().values
    if fill:
        stays, past = kept[kept < budget], kept[kept >= budget]
        at = torch.arange(budget, device=K.device)
        hole = torch.ones(budget, dtype=torch.bool, device=K.device)
        hole[stays] = False
        at[hole] = past
        kept = at
    after = torch.cat([mass[kept], torch.zeros(N - budget, device=K.device), mass[N:]])
    return K[kept], V[kept], after, kept.int()


def _past_32_bits(Hkv, N, cap, budget, fill, heads):
    say(f"{Hkv} heads of {N}/{cap} -> {budget}, fill={fill}: {Hkv * cap * 256 / 2 ** 32:.2f} x 2^32 bytes")
    g = torch.Generator(device="cuda").manual_seed(N)
    K, V = (torch.zeros(1, Hkv, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in "KV")
    for x in (K, V):
        for h in range(Hkv):
            x[0, h, :N].normal_(generator=g)
    mass = torch.empty(1, Hkv, cap, device="cuda").exponential_(generator=g)
    mass[mass < 0.3] = 0.0
    want = {h: _by_sorting(K[0, h], V[0, h], mass[0, h], N, budget, 16, 4, fill) for h in heads}
    behind = {h: [x[0, h, budget:budget + 100].clone() for x in (K, V)] for h in heads}
    d = bkv.dims(B=1, Hq=Hkv, Hkv=Hkv, D=128, N=N, N_cap=cap, W=16, C=0, budget=budget, n_prefix=4)
    ws, kept = bkv.mass_workspace(d), torch.empty(1, Hkv, budget, dtype=torch.int32, device="cuda")
    bkv.evict_mass(d, K, V, mass, ws, kept=kept, fill=fill)
    assert bkv.device_status(ws) == bkv.OK
    for h in heads:
        Kr, Vr, mr, kr = want[h]
        assert torch.equal(kept[0, h], kr)
        assert torch.equal(K[0, h, :budget], Kr) and torch.equal(V[0, h, :budget], Vr) and torch.equal(mass[0, h], mr)
        assert all(torch.equal(x[0, h, budget:budget + 100], y) for x, y in zip((K, V), behind[h]))


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("N,budget", [(3000, 2000), (9000, 5000), (40000, 30000)])
def test_heads_past_32_bits_of_bytes(N, budget, fill):
    # 20 heads of 1 M allocated rows of 256 bytes: 5 GB each of K and V; the last heads lie past 2^32 bytes
    _past_32_bits(20, N, 1 << 20, budget, fill, (0, 15, 16, 19))


def test_one_head_past_32_bits_of_bytes():
    # 17 M tokens of one head: rows past 2^32 bytes move into the holes below
    N = (1 << 24) + 5000
    _past_32_bits(1, N, N + 3, N - 3000, True, (0,))


@pytest.mark.parametrize("fill", [False, True])
@pytest.mark.parametrize("Hkv,N,budget", [(2, 700, 600), (3, 5000, 2400), (300, 700, 300)])
def test_keys_and_values_in_turns(Hkv, N, budget, fill):
    """One array of 2 N rows a head, its keys first and its values behind them."""
    say(f"in turns: {Hkv} heads, {N} -> {budget}, fill={fill}")
    g = torch.Generator().manual_seed(N)
    KV = torch.randn(Hkv, 2 * N, 64, generator=g).bfloat16()
    m = masses("sinks", Hkv, 2 * N, g)
    d = bkv.dims(B=1, Hq=Hkv, Hkv=Hkv, D=64, N=N, N_cap=2 * N, W=8, C=0, budget=budget, n_prefix=2)
    KVd, md, ws = KV.cuda(), m.cuda(), bkv.mass_workspace(d)
    kept = torch.empty(1, Hkv, budget, dtype=torch.int32, device="cuda")
    call = lambda off: bkv.lib().bkv_evict_mass(d, int(fill), KVd.data_ptr(), KVd.data_ptr() + off * 128, md.data_ptr(),  # noqa: E731
                                                kept.data_ptr(), ws.data_ptr(), ws.nbytes, torch.cuda.current_stream().cuda_stream)
    for off in (1, N - 1, N + 1):
        assert call(off) == bkv.ERR_INVALID
    assert call(N) == bkv.OK and bkv.device_status(ws) == bkv.OK
    Kr, Vr, mr, kr = attend_ref.evict(KV[:, :N], KV[:, N:], m, N, budget, 8, 2, fill)
    assert torch.equal(host(kept)[0], kr) and torch.equal(bits(KVd), bits(torch.cat([Kr, Vr], 1))) and torch.equal(bits(md), bits(mr))

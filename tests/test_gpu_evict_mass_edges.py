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

"""The periodic driver with attention: every step's output against the 64-bit
reference on the cache that the step saw, the masses of mode "mass" step by
step and its evictions bit for bit, and samples that share a prefix."""
import pytest
import torch

import attend_ref
from gpu_util import host, say
from paper_2609_04971_amd import diagnostics, synth
from paper_2609_04971_amd.driver import PeriodicEviction

pytestmark = pytest.mark.gpu

LAYERS, B, HQ, HKV, D, B_MAX, NR, T0, STEPS = 2, 2, 8, 2, 64, 64, 4, 50, 24  # evictions after 14 and 22 steps
LB = LAYERS * B


def rope(t):
    c, s = synth.rope_table(D, t)
    return c.cuda(), s.cuda()


@pytest.mark.parametrize("mode,compaction,prefix", [("mass", "order", 0), ("mass", "fill", 0), ("mass", "fill", 70),
                                                    ("beacon", "order", 0), ("rpc", "fill", 33), ("ns", "order", 0),
                                                    ("initial", "order", 5)])
def test_steps(mode, compaction, prefix):
    say(f"driver {mode} {compaction} prefix {prefix}")
    g = torch.Generator().manual_seed(21)
    r = lambda *s: torch.randn(*s, generator=g).bfloat16()  # noqa: E731
    drv = PeriodicEviction(LAYERS, B, HQ, HKV, D, B_MAX, rope, n_beacon=4, n_recent=NR, n_prefix=2, mode=mode, compaction=compaction,
                           attention=True, record=True)
    pre = {}
    if prefix:
        pre = {"PK": r(LAYERS, HKV, prefix, D), "PV": r(LAYERS, HKV, prefix, D), "P": prefix, "groups": LAYERS}
        drv.share_prefix(pre["PK"].cuda(), pre["PV"].cuda())
    K, V, q = r(LB, HKV, T0, D), r(LB, HKV, T0, D), r(LB, HQ, T0, D)
    out = drv.prefill(K.cuda(), V.cuda(), q.cuda(), q_rope=q.cuda())
    ref = attend_ref.reference(q, K, V, T0, causal=True, **pre)
    zero = torch.zeros(LB, HKV, B_MAX)
    mass = host(drv.mass) if mode == "mass" else None
    attend_ref.check(ref, host(out), ref["lse"].float(), mass, zero, T0)
    assert drv.t == prefix + T0 and drv.L == T0
    evictions = 0
    for _ in range(STEPS):
        k, v, y = r(LB, HKV, D), r(LB, HKV, D), r(LB, HQ, D)
        K, V, n = host(drv.K).clone(), host(drv.V).clone(), drv.L
        K[:, :, n], V[:, :, n] = k, v
        evicted = drv.step(k.cuda(), v.cuda(), y.cuda(), y.cuda())
        ref = attend_ref.reference(y.unsqueeze(2), K, V, n + 1, **pre)
        if mode == "mass":
            before, mass = mass, host(drv.events[-1][1]["mass"] if evicted else drv.mass)
        attend_ref.check(ref, host(drv.out).unsqueeze(2), host(drv.lse).unsqueeze(2), mass, before if mode == "mass" else None, n + 1)
        if not evicted:
            continue
        evictions += 1
        assert drv.L == drv.B_min
        if mode == "mass":
            flat = lambda t: t.reshape(LB * HKV, B_MAX, *t.shape[3:])  # noqa: E731
            want = attend_ref.evict(flat(K), flat(V), flat(mass), B_MAX, drv.B_min, NR, 2, compaction == "fill")
            for a, b in zip((drv.K, drv.V, drv.mass, drv.kept), want):
                assert torch.equal(host(a).view(b.shape), b)
            mass = host(drv.mass)
    assert evictions == 2


def test_refusals():
    with pytest.raises(ValueError):
        PeriodicEviction(1, 1, 4, 2, D, B_MAX, rope, n_recent=NR, mode="other")
    plain = PeriodicEviction(1, 1, 4, 2, D, B_MAX, rope, n_beacon=4, n_recent=NR)
    z = torch.zeros(1, 2, 9, D, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        plain.share_prefix(z, z)  # nothing would read it
    drv = PeriodicEviction(1, 1, 4, 2, D, B_MAX, rope, n_recent=NR, mode="mass")
    with pytest.raises(ValueError):
        drv.share_prefix(z[:, :1], z[:, :1])
    with pytest.raises(ValueError):
        drv.prefill(z, z, torch.zeros(1, 4, 9, D, dtype=torch.bfloat16, device="cuda"))  # no post-RoPE queries
    q = torch.zeros(1, 4, 9, D, dtype=torch.bfloat16, device="cuda")
    drv.prefill(z, z, q, q_rope=q)
    with pytest.raises(ValueError):
        drv.share_prefix(z, z)


def test_diagnostics_of_mode_mass():
    tr = synth.revisit_trace(2, 8, 2, 64, 192, n_plant=8, n_groups=2, p_global=0.1, local_dim=8, seed=7)
    dev = {k: (v.cuda() if torch.is_tensor(v) else v) for k, v in tr.items()}
    res = diagnostics.run(dev, "mass", 128, n_recent=4, prompt=64, record=True, compaction="fill")
    assert len(res["steps"]) == len(res["retention"]) == 5 and not res["coverage"]
    pos = host(res["pos"]).long()
    drv = res["driver"]
    want = torch.gather(tr["K"], 2, pos.unsqueeze(-1).expand(-1, -1, -1, 64))
    assert torch.equal(host(drv.K)[:, :, :drv.L], want)  # the tracked positions name the cached rows
    s = diagnostics.summary(res)
    assert s["coverage_mean"] is None and 0.0 <= s["retention_last"] <= 1.0

"""The periodic driver by mass, on a 4-bit cache and on a plain one that holds the same values:
the same outputs within both bounds and, where both go by the same masses, the same evictions."""
import pytest
import torch

import attend_ref
import paper_2609_04971_amd as bkv
from attend_more import reference
from gpu_util import host, say
from paper_2609_04971_amd.driver import PeriodicEviction
from test_gpu_driver_mx import B, B_MAX, D, HKV, HQ, LAYERS, LB, NR, STEPS, T0, rope, rounded, values

pytestmark = pytest.mark.gpu


class Follower(PeriodicEviction):
    """Evicts by the masses that `leader` has just evicted by: their last bits may differ between the caches."""
    leader = None

    def _evict(self):
        self.mass.copy_(self.leader.events[-1][1]["mass"])
        super()._evict()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("compaction", ["order", "fill"])
def test_mass(compaction, dtype):
    say(f"driver mx mass {compaction} {dtype}")
    g = torch.Generator().manual_seed(22)
    r = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    kw = dict(n_recent=NR, n_prefix=2, mode="mass", compaction=compaction, record=True, dtype=dtype)
    drv = PeriodicEviction(LAYERS, B, HQ, HKV, D, B_MAX, rope, cache="mx", **kw)
    plain = Follower(LAYERS, B, HQ, HKV, D, B_MAX, rope, **kw)
    plain.leader = drv
    K, V, q = rounded(r(LB, HKV, T0, D)), rounded(r(LB, HKV, T0, D)), r(LB, HQ, T0, D)
    zero, ref = torch.zeros(LB, HKV, B_MAX), reference(q, K, V, T0, True)
    for x in (drv, plain):
        out = x.prefill(K.cuda(), V.cuda(), q.cuda(), q_rope=q.cuda())
        attend_ref.check(ref, host(out), ref["lse"].float(), host(x.mass), zero, T0)
    evictions = 0
    for _ in range(STEPS):
        k, v, y = rounded(r(LB, HKV, D)), rounded(r(LB, HKV, D)), r(LB, HQ, D)
        n, before = drv.L, [host(x.mass) for x in (drv, plain)]
        K, V = values(drv.cache)
        K[:, :, n], V[:, :, n] = k.double(), v.double()
        ref = reference(y.unsqueeze(2), K, V, n + 1, True)
        evicted = [x.step(k.cuda(), v.cuda(), y.cuda(), y.cuda()) for x in (drv, plain)]
        assert evicted[0] == evicted[1] and drv.L == plain.L
        for x, was in zip((drv, plain), before):
            attend_ref.check(ref, host(x.out).unsqueeze(2), host(x.lse).unsqueeze(2), None if evicted[0] else host(x.mass), was, n + 1)
        if not evicted[0]:
            continue
        evictions += 1
        assert torch.equal(drv.kept, plain.kept) and torch.equal(drv.mass, plain.mass)
        for a, b in zip(values(drv.cache), (plain.K, plain.V)):
            assert torch.equal(a[:, :, :drv.L], host(b)[:, :, :drv.L].double())
    assert evictions == 2 and bkv.device_status(drv.ws) == bkv.OK and bkv.device_status(plain.ws) == bkv.OK

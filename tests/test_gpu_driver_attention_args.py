"""Arguments of the driver's attention that do not fit are refused before
anything of its state changes."""
import pytest
import torch

from gpu_util import host
from paper_2609_04971_amd import synth
from paper_2609_04971_amd.driver import PeriodicEviction

pytestmark = pytest.mark.gpu
LB, HQ, HKV, D, T = 2, 8, 2, 64, 20


def rope(t):
    c, s = synth.rope_table(D, t)
    return c.cuda(), s.cuda()


@pytest.mark.parametrize("mode", ["mass", "rpc"])
def test_queries_of_another_length_or_type(mode):
    drv = PeriodicEviction(1, LB, HQ, HKV, D, 64, rope, n_recent=4, mode=mode, attention=True)
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()  # noqa: E731
    K, V, q = r(LB, HKV, T, D), r(LB, HKV, T, D), r(LB, HQ, T, D)
    for bad in (q[:, :, :T - 1], r(LB, HQ, T + 1, D), q[:1], q.float(), q.cpu()):
        with pytest.raises(ValueError):
            drv.prefill(K, V, q, q_rope=bad)
        assert drv.L == 0 and drv.t == 0 and not host(drv.K).any()
    assert drv.prefill(K, V, q, q_rope=q).shape == q.shape and drv.L == T


def test_prefix_of_another_type():
    drv = PeriodicEviction(1, LB, HQ, HKV, D, 64, rope, n_recent=4, mode="mass")
    z = torch.zeros(1, HKV, 9, D, dtype=torch.bfloat16, device="cuda")
    for K, V in ((z.float(), z.float()), (z, z.float()), (z.cpu(), z.cpu())):
        with pytest.raises(ValueError):
            drv.share_prefix(K, V)
        assert drv.t == 0 and drv.prefix is None
    drv.share_prefix(z, z)
    assert drv.t == 9

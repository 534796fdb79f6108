"""The periodic driver on a 4-bit cache and with a window: every step's output
against the 64-bit reference on what the step saw, evictions against those of a
plain cache that holds the same values, bit for bit."""
import pytest
import torch

import attend_ref
import mx_ref
import paper_2609_04971_amd as bkv
from attend_more import reference
from gpu_util import host, say
from paper_2609_04971_amd import synth
from paper_2609_04971_amd.driver import PeriodicEviction

pytestmark = pytest.mark.gpu

LAYERS, B, HQ, HKV, D, B_MAX, NR, T0, STEPS = 2, 2, 8, 2, 64, 64, 4, 50, 24  # evictions after 14 and 22 steps
LB = LAYERS * B


def rope(t):
    c, s = synth.rope_table(D, t)
    return c.cuda(), s.cuda()


def values(cache):
    return mx_ref.values(host(cache.K), host(cache.KS)), mx_ref.values(host(cache.V), host(cache.VS))


def rounded(t):
    """What a 4-bit cache makes of t."""
    return mx_ref.values(*mx_ref.quantise(t)).to(t.dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("mode,compaction,window,sinks", [("mass", "order", 0, 0), ("mass", "fill", 0, 0), ("beacon", "order", 0, 0), ("rpc", "order", 20, 3),
                                                          ("ns", "order", 0, 0), ("initial", "order", 40, 0)])
def test_as_a_plain_cache_of_the_same_values(mode, compaction, window, sinks, dtype):
    """Keys and values that 4 bits hold exactly, in a plain cache and in a 4-bit one: the same rows are kept."""
    say(f"driver mx {mode} {compaction} window {window}+{sinks} {dtype}")
    g = torch.Generator().manual_seed(21)
    r = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    kw = dict(n_beacon=4, n_recent=NR, n_prefix=2, mode=mode, compaction=compaction, attention=True, record=True, dtype=dtype)
    drv = PeriodicEviction(LAYERS, B, HQ, HKV, D, B_MAX, rope, cache="mx", window=window, sinks=sinks, **kw)
    plain = PeriodicEviction(LAYERS, B, HQ, HKV, D, B_MAX, rope, window=window, sinks=sinks, **kw)
    K, V, q = rounded(r(LB, HKV, T0, D)), rounded(r(LB, HKV, T0, D)), r(LB, HQ, T0, D)
    outs = [d.prefill(K.cuda(), V.cuda(), q.cuda(), q_rope=q.cuda()) for d in (drv, plain)]
    ref = reference(q, K, V, T0, True, None, None, window, sinks)
    zero = torch.zeros(LB, HKV, B_MAX)
    mass = host(drv.mass) if mode == "mass" else None
    for o in outs:
        attend_ref.check(ref, host(o), ref["lse"].float(), None, None, T0)
    if mode == "mass":
        attend_ref.check(ref, host(outs[0]), ref["lse"].float(), mass, zero, T0)
    evictions = 0
    for _ in range(STEPS):
        k, v, y = rounded(r(LB, HKV, D)), rounded(r(LB, HKV, D)), r(LB, HQ, D)
        n = drv.L
        K, V = values(drv.cache)
        K[:, :, n], V[:, :, n] = k.double(), v.double()
        if mode == "mass":  # the weights' last bits may differ between the two: the plain one goes by the other's
            plain.mass.copy_(drv.mass)
        evicted = drv.step(k.cuda(), v.cuda(), y.cuda(), y.cuda())
        ref = reference(y.unsqueeze(2), K, V, n + 1, True, None, None, window, sinks)
        if mode == "mass":
            before, mass = mass, host(drv.events[-1][1]["mass"] if evicted else drv.mass)
        attend_ref.check(ref, host(drv.out).unsqueeze(2), host(drv.lse).unsqueeze(2), mass, before if mode == "mass" else None, n + 1)
        if mode != "mass":
            assert plain.step(k.cuda(), v.cuda(), y.cuda(), y.cuda()) == evicted
            attend_ref.check(ref, host(plain.out).unsqueeze(2), host(plain.lse).unsqueeze(2), None, None, n + 1)
        if not evicted:
            continue
        evictions += 1
        assert drv.L == drv.B_min
        if mode == "mass":
            was = drv.events[-1][1]["before"]
            join = lambda c: [torch.cat([host(a), host(b)], -1).flatten(0, 1) for a, b in ((c.K, c.KS), (c.V, c.VS))]  # noqa: E731
            want = attend_ref.evict(*join(was), mass.flatten(0, 1), B_MAX, drv.B_min, NR, 2, compaction == "fill")
            got = [*join(drv.cache), host(drv.mass).flatten(0, 1), host(drv.kept).flatten(0, 1)]
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            mass = host(drv.mass)
        else:
            assert torch.equal(drv.kept, plain.kept) and torch.equal(drv.scores, plain.scores)
            for a, b in zip(values(drv.cache), (plain.K, plain.V)):
                assert torch.equal(a[:, :, :drv.L], host(b)[:, :, :drv.L].double())
    assert evictions == 2 and bkv.device_status(drv.ws) == bkv.OK


@pytest.mark.parametrize("window,sinks", [(1, 0), (17, 4), (1000, 0)])
def test_windows_on_a_plain_cache(window, sinks):
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g).bfloat16()  # noqa: E731
    drv = PeriodicEviction(LAYERS, B, HQ, HKV, D, B_MAX, rope, n_beacon=4, n_recent=NR, attention=True, window=window, sinks=sinks)
    K, V, q = r(LB, HKV, T0, D), r(LB, HKV, T0, D), r(LB, HQ, T0, D)
    out = drv.prefill(K.cuda(), V.cuda(), q.cuda(), q_rope=q.cuda())
    ref = reference(q, K, V, T0, True, None, None, window, sinks)
    attend_ref.check(ref, host(out), ref["lse"].float(), None, None, T0)
    for _ in range(STEPS):
        k, v, y = r(LB, HKV, D), r(LB, HKV, D), r(LB, HQ, D)
        K, V, n = host(drv.K).clone(), host(drv.V).clone(), drv.L
        K[:, :, n], V[:, :, n] = k, v
        drv.step(k.cuda(), v.cuda(), y.cuda(), y.cuda())
        ref = reference(y.unsqueeze(2), K, V, n + 1, True, None, None, window, sinks)
        attend_ref.check(ref, host(drv.out).unsqueeze(2), host(drv.lse).unsqueeze(2), None, None, n + 1)


def test_refusals():
    make = lambda **kw: PeriodicEviction(1, 1, 4, 2, D, B_MAX, rope, n_beacon=4, n_recent=NR, **kw)  # noqa: E731
    for kw in (dict(cache="fp4"), dict(cache="mx", compaction="fill"), dict(window=5), dict(window=5, mode="mass"), dict(window=-1, attention=True),
               dict(sinks=-1), dict(window=5, attention=True, compaction="fill")):
        with pytest.raises(ValueError):
            make(**kw)
    z = torch.zeros(1, 2, 9, D, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(cache="mx", mode="mass"), dict(window=5, attention=True)):
        with pytest.raises(ValueError):
            make(**kw).share_prefix(z, z)
    drv = make(cache="mx")
    with pytest.raises(ValueError):
        drv.prefill(z.float(), z.float(), z)

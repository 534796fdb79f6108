"""Refusals of the 4-bit cache's eviction without a GPU: every call here is refused
or empty, and the addresses stand in for device memory that nothing reads."""
import ctypes

import pytest

import paper_2609_04971_amd as bkv

A = 1 << 40
LIB = bkv.lib()
NAMES = ("K", "KS", "V", "VS", "mass", "kept", "ws")


def good(**kw):
    return bkv.dims(B=4, Hq=8, Hkv=2, D=128, N=1000, N_cap=1100, W=8, C=0, budget=256, n_prefix=2).replace(**kw)


def evict(d=None, flags=0, n=1 << 40, cache=True, **at):
    a = {k: at.get(k, (i + 1) * A) for i, k in enumerate(NAMES)}
    c = bkv._MxPtrs(K=a["K"], KS=a["KS"], V=a["V"], VS=a["VS"])
    return LIB.bkv_evict_mass_mx(ctypes.byref(d or good()), flags, ctypes.byref(c) if cache else None, a["mass"], a["kept"], a["ws"], n, None)


def compact(d=None, n=1 << 40, cache=True, flags=0, **at):
    a = {k: at.get(k, (i + 1) * A) for i, k in enumerate(NAMES)}
    c = bkv._MxPtrs(K=a["K"], KS=a["KS"], V=a["V"], VS=a["VS"])
    return LIB.bkv_compact_mx(ctypes.byref(d or good()), ctypes.byref(c) if cache else None, a["kept"], a["ws"], n, None)


@pytest.mark.parametrize("call", [evict, compact])
def test_refusals(call):
    for kw, code in ((dict(D=96), bkv.ERR_SHAPE), (dict(dtype=4), bkv.ERR_DTYPE), (dict(N=1101), bkv.ERR_SHAPE), (dict(budget=5), bkv.ERR_SHAPE)):
        assert call(good(**kw)) == code
    assert call(cache=False) == bkv.ERR_INVALID
    for k in ("K", "KS", "V", "VS"):
        assert call(**{k: None}) == bkv.ERR_INVALID and call(**{k: 30 * A + 4}) == bkv.ERR_INVALID
    assert call(ws=None) == bkv.ERR_WORKSPACE and call(n=100) == bkv.ERR_WORKSPACE and call(ws=30 * A + 8) == bkv.ERR_WORKSPACE
    assert call(good(B=0), cache=False) == bkv.OK and call(good(N=0), cache=False) == bkv.OK


def test_refusals_of_one():
    assert evict(mass=None) == bkv.ERR_INVALID and evict(flags=2) == bkv.ERR_INVALID
    assert compact(kept=None) == bkv.ERR_INVALID
    assert evict(good(N=200), kept=None) == bkv.OK  # nothing to do, nothing to write
    assert LIB.bkv_evict_mass_mx(None, 0, None, None, None, None, 0, None) == bkv.ERR_INVALID
    assert LIB.bkv_compact_mx(None, None, None, None, 0, None) == bkv.ERR_INVALID


@pytest.mark.parametrize("N", [1000, 200])
@pytest.mark.parametrize("one", NAMES)
@pytest.mark.parametrize("other", NAMES)
def test_over_itself(one, other, N):
    if one == other:
        return
    d = good(N=N)
    need = LIB.bkv_mass_workspace_bytes(ctypes.byref(d))
    tokens = 7 * 1100 + N
    size = {"K": tokens * 64, "V": tokens * 64, "KS": tokens * 4, "VS": tokens * 4, "mass": tokens * 4, "kept": 8 * min(N, 256) * 4, "ws": need}
    for to in (((NAMES.index(other) + 1) * A), ((NAMES.index(other) + 1) * A) + (size[other] - 16 & ~15), ((NAMES.index(other) + 1) * A) - 16):
        assert evict(d, n=need, **{one: to}) == bkv.ERR_INVALID
        if "mass" not in (one, other) and not ("ws" in (one, other) and to % A):  # (its workspace is smaller)
            assert compact(d, n=need, **{one: to}) == bkv.ERR_INVALID

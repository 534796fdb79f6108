"""Refusals of attention with a window and over a 4-bit cache, and their workspace,
without a GPU: every call here is refused or empty, and the addresses stand in for
device memory that nothing reads."""
import ctypes

import pytest

import paper_2609_04971_amd as bkv
from test_attend_host_limits import SHAPES

A = 1 << 40
LIB = bkv.lib()


def good(**kw):
    return bkv.dims(B=4, Hq=8, Hkv=2, D=128, N=1000, N_cap=1100, W=8, C=0, budget=256, n_prefix=2).replace(**kw)


def window(d=None, w=100, sinks=4, T=1, n=1 << 40, scale=0.0, **at):
    a = {k: ctypes.c_void_p(at.get(k, (i + 1) * A)) for i, k in enumerate(("q", "K", "V", "lens", "out", "lse", "ws"))}
    return LIB.bkv_attend_window(ctypes.byref(d or good()), a["q"], T, a["K"], a["V"], w, sinks, a["lens"], scale, a["out"], a["lse"],
                                 a["ws"], n, None)


def mx(d=None, flags=bkv.ATTEND_CAUSAL, w=0, sinks=0, T=1, n=1 << 40, scale=0.0, cache=True, **at):
    a = {k: at.get(k, (i + 1) * A) for i, k in enumerate(("q", "K", "KS", "V", "VS", "lens", "out", "lse", "mass", "ws"))}
    c = bkv._MxPtrs(K=a["K"], KS=a["KS"], V=a["V"], VS=a["VS"]) if cache else None
    return LIB.bkv_attend_mx(ctypes.byref(d or good()), flags, a["q"], T, ctypes.byref(c) if c else None, w, sinks, a["lens"], scale,
                             a["out"], a["lse"], a["mass"], a["ws"], n, None)


def test_window_refusals():
    for w, sinks in ((0, 4), (-1, 0), (-2 ** 31, 0), (5, -1), (5, -2 ** 31)):
        assert window(w=w, sinks=sinks) == bkv.ERR_SHAPE
    assert LIB.bkv_attend_window(None, None, 1, None, None, 0, 0, None, 0.0, None, None, None, 0, None) == bkv.ERR_INVALID
    assert LIB.bkv_attend_window(None, None, 1, None, None, 1, 0, None, 0.0, None, None, None, 0, None) == bkv.ERR_INVALID
    assert window(good(D=96)) == bkv.ERR_SHAPE
    assert window(good(dtype=5)) == bkv.ERR_DTYPE
    assert window(T=-1) == bkv.ERR_SHAPE
    for k in ("q", "K", "V", "out"):
        assert window(**{k: None}) == bkv.ERR_INVALID
        assert window(**{k: 9 * A + 8}) == bkv.ERR_INVALID
    assert window(scale=-1.0) == bkv.ERR_INVALID and window(scale=float("nan")) == bkv.ERR_INVALID
    assert window(scale=3e38) == bkv.ERR_INVALID
    assert window(good(N=1100), w=1100, n=15) == bkv.ERR_WORKSPACE
    assert window(out=A) == bkv.ERR_INVALID and window(lse=2 * A + 16) == bkv.ERR_INVALID and window(out=7 * A, T=9, n=1 << 30) == bkv.ERR_INVALID
    assert window(T=0) == bkv.OK and window(good(B=0)) == bkv.OK


def test_mx_refusals():
    assert mx(flags=2) == bkv.ERR_INVALID and mx(flags=-1) == bkv.ERR_INVALID
    assert LIB.bkv_attend_mx(None, 0, None, 1, None, 0, 0, None, 0.0, None, None, None, None, 0, None) == bkv.ERR_INVALID
    assert mx(w=-1) == bkv.ERR_SHAPE and mx(w=5, sinks=-1, mass=None) == bkv.ERR_SHAPE
    assert mx(w=5) == bkv.ERR_INVALID                                   # weights of a window
    assert mx(w=5, T=2, flags=0, mass=None) == bkv.ERR_INVALID          # a window counts back from the query's own token
    assert mx(cache=False) == bkv.ERR_INVALID
    for k in ("q", "K", "KS", "V", "VS", "out"):
        assert mx(**{k: None}) == bkv.ERR_INVALID
        assert mx(**{k: 30 * A + 8}) == bkv.ERR_INVALID
    assert mx(good(D=32)) == bkv.ERR_SHAPE and mx(good(dtype=2)) == bkv.ERR_DTYPE
    assert mx(n=15) == bkv.ERR_WORKSPACE and mx(ws=None) == bkv.ERR_WORKSPACE
    assert mx(T=0, cache=False) == bkv.OK and mx(good(B=0), cache=False) == bkv.OK
    assert mx(scale=3e38) == bkv.ERR_INVALID


SIZES = {"out": 4 * 8 * 256, "lse": 4 * 8 * 4, "mass": (7 * 1100 + 1000) * 4, "ws": 1024, "q": 4 * 8 * 256,
         "K": (7 * 1100 + 1000) * 64, "KS": (7 * 1100 + 1000) * 4, "V": (7 * 1100 + 1000) * 64, "VS": (7 * 1100 + 1000) * 4, "lens": 16}


@pytest.mark.parametrize("written", ["out", "lse", "mass", "ws"])
@pytest.mark.parametrize("other", list(SIZES))
def test_mx_outputs_over_anything_else(written, other):
    if written == other:
        return
    at = {k: (i + 1) * A for i, k in enumerate(("q", "K", "KS", "V", "VS", "lens", "out", "lse", "mass", "ws"))}
    for to in (at[other], at[other] + (SIZES[other] - 16 & ~15), at[other] - 16 if SIZES[written] > 16 else at[other]):
        assert mx(n=1 << 20, **{written: to}) == bkv.ERR_INVALID


@pytest.mark.parametrize("dtype", [bkv.BF16, bkv.F32])
@pytest.mark.parametrize("B,Hkv,G,T,N_cap", sorted({s[:5] for s in SHAPES}))
def test_one_workspace_size_covers_every_length_and_window(B, Hkv, G, T, N_cap, dtype):
    """As of plain attention: with the size asked for at N 0 the next check refuses (outputs that overlap), with a byte less the
    workspace's."""
    for D in (64, 128):
        d = good(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=0, N_cap=N_cap, dtype=dtype)
        for mass in (0, 1):
            need = LIB.bkv_attend_workspace_bytes(ctypes.byref(d), T, mass, 0, 0)
            for N in sorted({0, 1, 129, 1000, N_cap // 2, N_cap} & set(range(N_cap + 1))):
                dn = d.replace(N=N)
                for w, sinks in ((0, 0), (1, 0), (100, 4), (N_cap // 3 + 1, N_cap // 3), (2 ** 31 - 1, 2 ** 31 - 1)):
                    for n, code in ((need, bkv.ERR_INVALID), (need - 1, bkv.ERR_WORKSPACE)):
                        if n < 0 or (w and mass):
                            continue
                        at = {"out": 100 * A, "lse": 100 * A, "ws": 200 * A}
                        assert mx(dn, w=w, sinks=sinks, T=T, n=n, mass=300 * A if mass else None, **at) == code
                        if w:
                            assert window(dn, w=w, sinks=sinks, T=T, n=n, **at) == code

"""Host-side rules of the attention and mass-eviction entry points: bad
arguments are refused before anything is enqueued, and workspace sizes cover
every length.  Only calls that fail validation or are no-ops are made."""
import ctypes

import pytest
import torch

import paper_2609_04971_amd as bkv

P = ctypes.c_void_p(1 << 20)    # 16-byte aligned stand-ins, never dereferenced
OUT = ctypes.c_void_p(1 << 28)
ODD = ctypes.c_void_p((1 << 20) + 8)
BIG = 1 << 40


def dims(**kw):
    return bkv.dims(B=4, Hq=8, Hkv=2, D=128, N=1000, N_cap=1100, W=8, C=0, budget=256, n_prefix=2).replace(**kw)


def attend(d=None, flags=0, q=P, T=1, K=P, V=P, lens=None, scale=0.0, out=OUT, lse=None, mass=None, ws=P, n=BIG):
    d = dims() if d is None else d
    return bkv.lib().bkv_attend(ctypes.byref(d), flags, q, T, K, V, lens, scale, out, lse, mass, ws, n, None)


def shared(d=None, flags=0, q=P, T=1, groups=2, PK=P, PV=P, n_pre=50, P_cap=60, p_lens=None, K=P, V=P, scale=0.0, out=OUT,
           mass=None, ws=P, n=BIG):
    d = dims() if d is None else d
    return bkv.lib().bkv_attend_shared(ctypes.byref(d), flags, q, T, groups, PK, PV, n_pre, P_cap, p_lens, K, V, None,
                                       scale, out, None, mass, ws, n, None)


def evict(d=None, flags=0, K=P, V=P, mass=P, kept=P, ws=P, n=BIG):
    d = dims() if d is None else d
    return bkv.lib().bkv_evict_mass(ctypes.byref(d), flags, K, V, mass, kept, ws, n, None)


@pytest.mark.parametrize("call", [attend, shared])
@pytest.mark.parametrize("kw,code", [
    (dict(flags=2), bkv.ERR_INVALID),
    (dict(T=-1), bkv.ERR_SHAPE),
    (dict(T=1 << 27), bkv.ERR_SHAPE),                # rows past 31 bits
    (dict(d=dims(D=96)), bkv.ERR_SHAPE),
    (dict(d=dims(Hq=7)), bkv.ERR_SHAPE),
    (dict(d=dims(N=1200)), bkv.ERR_SHAPE),
    (dict(d=dims(dtype=9)), bkv.ERR_DTYPE),
    (dict(q=None), bkv.ERR_INVALID), (dict(q=ODD), bkv.ERR_INVALID),
    (dict(K=None), bkv.ERR_INVALID), (dict(K=ODD), bkv.ERR_INVALID),
    (dict(V=None), bkv.ERR_INVALID), (dict(V=ODD), bkv.ERR_INVALID),
    (dict(out=None), bkv.ERR_INVALID), (dict(out=ODD), bkv.ERR_INVALID),
    (dict(out=P), bkv.ERR_INVALID),                  # over the queries
    (dict(out=ctypes.c_void_p((1 << 20) + 4096)), bkv.ERR_INVALID),
    (dict(scale=-1.0), bkv.ERR_INVALID), (dict(scale=float("inf")), bkv.ERR_INVALID),
    (dict(scale=float("nan")), bkv.ERR_INVALID),
    (dict(ws=None), bkv.ERR_WORKSPACE), (dict(ws=ODD), bkv.ERR_WORKSPACE), (dict(n=16), bkv.ERR_WORKSPACE),
])
def test_attend_rejects(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(groups=0), bkv.ERR_SHAPE),
    (dict(groups=3), bkv.ERR_SHAPE),                 # does not divide the batch
    (dict(n_pre=61), bkv.ERR_SHAPE), (dict(n_pre=-1), bkv.ERR_SHAPE),
    (dict(n_pre=0, P_cap=0), bkv.ERR_SHAPE),
    (dict(P_cap=1 << 30), bkv.ERR_SHAPE),            # keys past 31 bits
    (dict(PK=None), bkv.ERR_INVALID), (dict(PK=ODD), bkv.ERR_INVALID),
    (dict(PV=None), bkv.ERR_INVALID), (dict(PV=ODD), bkv.ERR_INVALID),
])
def test_shared_rejects(kw, code):
    assert shared(**kw) == code


def test_attend_no_ops_and_null_dims():
    for call in (attend, shared):
        assert call(T=0, q=None, out=None, ws=None) == bkv.OK
        assert call(d=dims(B=0), q=None, K=None, out=None, ws=None) == bkv.OK
    lib = bkv.lib()
    assert lib.bkv_attend(None, 0, P, 1, P, P, None, 0.0, P, None, None, P, BIG, None) == bkv.ERR_INVALID
    assert lib.bkv_attend_workspace_bytes(None, 1, 0, 0, 0) == 0
    assert lib.bkv_mass_workspace_bytes(None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(flags=2), bkv.ERR_INVALID),
    (dict(d=dims(budget=9)), bkv.ERR_SHAPE),
    (dict(d=dims(D=32)), bkv.ERR_SHAPE),
    (dict(K=None), bkv.ERR_INVALID), (dict(K=ODD), bkv.ERR_INVALID),
    (dict(V=None), bkv.ERR_INVALID), (dict(V=ODD), bkv.ERR_INVALID),
    (dict(mass=None), bkv.ERR_INVALID),
    (dict(ws=None), bkv.ERR_WORKSPACE), (dict(ws=ODD), bkv.ERR_WORKSPACE), (dict(n=256), bkv.ERR_WORKSPACE),
])
def test_evict_mass_rejects(kw, code):
    assert evict(**kw) == code


def test_evict_mass_no_ops():
    assert evict(d=dims(B=0), K=None, mass=None, ws=None) == bkv.OK
    assert evict(d=dims(N=0), K=None, mass=None, ws=None) == bkv.OK
    assert evict(d=dims(N=200), kept=None) == bkv.OK  # fits the budget and asks for no indices


def _bytes(d, T=1, mass=0, groups=0, P_cap=0):
    return bkv.lib().bkv_attend_workspace_bytes(ctypes.byref(d), T, mass, groups, P_cap)


@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("mass", [0, 1])
def test_workspace_does_not_depend_on_the_length(T, mass):
    want = _bytes(dims(N=1100), T, mass)
    assert {_bytes(dims(N=n), T, mass) for n in (0, 1, 17, 500, 1000, 1100)} == {want}
    assert bkv.lib().bkv_mass_workspace_bytes(ctypes.byref(dims(N=3))) == \
        bkv.lib().bkv_mass_workspace_bytes(ctypes.byref(dims(N=1100)))


def test_binding_refuses_what_the_library_cannot_see():
    d = dims()
    q, K = torch.zeros(4, 8, 1, 128, dtype=torch.bfloat16), torch.zeros(4, 2, 1100, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        bkv.attend(d, q, K, K, q, q)                 # host tensors
    with pytest.raises(ValueError):
        bkv.attend(d, q[0], K, K, q, q)              # no batch
    with pytest.raises(ValueError):
        bkv.attend_shared(d, q, K[0], K[0], K, K, q, q)
    with pytest.raises(ValueError):
        bkv.evict_mass(d, K, K, torch.zeros(4, 2, 1100), q)

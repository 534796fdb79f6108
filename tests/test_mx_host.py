"""The 4-bit cache's entry points without a GPU: what is refused before anything
is enqueued, and the reference's own properties."""
import ctypes

import pytest
import torch

import mx_ref

bkv = pytest.importorskip("paper_2609_04971_amd")
A = 1 << 20  # an address; nothing reads it, every call here is refused or empty


def good(**kw):
    return bkv.dims(B=2, Hq=8, Hkv=2, D=128, N=1000, N_cap=1024, W=0, C=0, budget=256).replace(**kw)


def cache(**kw):
    p = dict(K=A, KS=2 * A, V=3 * A, VS=4 * A)
    p.update(kw)
    return bkv._MxPtrs(**p)


def store(d, k=8 * A, v=16 * A, T=1, first=0, at=None, c=None):
    c = cache() if c is None else c
    return bkv.lib().bkv_store_mx(ctypes.byref(d), k, v, T, first, at, ctypes.byref(c) if c else None, None)


def load(d, k=8 * A, v=16 * A, T=1, first=0, at=None, c=None):
    c = cache() if c is None else c
    return bkv.lib().bkv_load_mx(ctypes.byref(d), ctypes.byref(c) if c else None, T, first, at, k, v, None)


@pytest.mark.parametrize("call", [store, load])
def test_refusals(call):
    d = good()
    assert call(good(D=96)) == bkv.ERR_SHAPE
    assert call(good(dtype=3)) == bkv.ERR_DTYPE
    assert call(d, T=-1) == bkv.ERR_SHAPE
    assert call(d, first=-1) == bkv.ERR_SHAPE
    assert call(d, T=25, first=1000) == bkv.ERR_SHAPE   # past the capacity
    assert call(d, T=2 ** 31 - 1, first=0) == bkv.ERR_SHAPE
    assert call(d, T=2 ** 29, at=A) == bkv.ERR_SHAPE    # 2^31 rows
    assert call(d, c=False) == bkv.ERR_INVALID
    assert call(d, k=None, v=None) == bkv.ERR_INVALID
    for name in ("K", "KS", "V", "VS"):
        assert call(d, c=cache(**{name: None})) == bkv.ERR_INVALID
        assert call(d, c=cache(**{name: A // 2 + 8})) == bkv.ERR_INVALID
    assert call(d, k=8 * A + 4) == bkv.ERR_INVALID
    assert call(d, v=16 * A + 8) == bkv.ERR_INVALID


@pytest.mark.parametrize("call", [store, load])
def test_nothing_to_do(call):
    assert call(good(B=0)) == bkv.OK
    assert call(good(), T=0) == bkv.OK
    assert call(good(), T=0, first=1024, k=None, v=None, c=False) == bkv.OK


def test_arrays_that_overlap_are_refused():
    d = good()
    codes, scales, row = 2 * 2 * 1024 * 64, 2 * 2 * 1024 * 4, 2 * 2 * 128 * 2
    for call in (store, load):
        assert call(d, k=A + codes - 16) == bkv.ERR_INVALID
        assert call(d, k=A - row + 16) == bkv.ERR_INVALID
        assert call(d, v=4 * A + scales - 16) == bkv.ERR_INVALID
    assert store(d, at=3 * A) == bkv.ERR_INVALID
    assert load(d, k=8 * A, v=8 * A) == bkv.ERR_INVALID           # two outputs in one place
    assert store(d, c=cache(V=A)) == bkv.ERR_INVALID
    assert store(d, c=cache(KS=A + codes - 16)) == bkv.ERR_INVALID
    assert load(d, at=8 * A) == bkv.ERR_INVALID


def test_binding_refuses():
    c = bkv.mx_cache(good(), device="cpu")
    assert [tuple(t.shape) for t in c] == [(2, 2, 1024, 64), (2, 2, 1024, 4)] * 2
    k = torch.zeros(2, 2, 1, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        bkv.store_mx(good(), k, k, c)      # not on a GPU
    with pytest.raises(ValueError):
        bkv.load_mx(good(), c, None, None)


def test_reference_on_its_own_values():
    # every code at every power of two is its own nearest, and ties go to the even code
    for e in (-124, -3, 0, 17, 125):
        x = torch.zeros(32, dtype=torch.float64)
        x[:16] = torch.cat([mx_ref.LEVELS, -mx_ref.LEVELS]) * 2.0 ** e
        codes, scales = mx_ref.quantise(x)
        assert scales.tolist() == [e + 127]
        assert torch.equal(mx_ref.values(codes, scales), x)
    x = torch.zeros(32, dtype=torch.float64)
    x[:9] = torch.tensor([4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6.99])
    codes, scales = mx_ref.quantise(x)
    assert scales.tolist() == [127]
    assert mx_ref.values(codes, scales)[:9].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6]


def test_reference_rounds_as_promised():
    x = torch.randn(4000, 64, generator=torch.Generator().manual_seed(1), dtype=torch.float64) * 3
    codes, scales = mx_ref.quantise(x)
    unit = torch.exp2(scales.double() - 127).repeat_interleave(32, -1)
    off = (mx_ref.values(codes, scales) - x).abs()
    assert bool((off <= torch.where(x.abs() >= unit, x.abs() / 5, unit / 4)).all())
    top = x.abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
    assert bool((top > 3.5 * unit).all() and (top <= 7 * unit).all())

"""Positions, windows and prefixes that are no 32-bit integers, without a GPU: ctypes would
cut them down to others (2**32 + 5 to 5), so the binding and the driver refuse them."""
import numpy as np
import pytest
import torch

import paper_2609_04971_amd as bkv
from paper_2609_04971_amd.driver import PeriodicEviction

BAD = [0.5, 2.9, 5.0, "5", None, float("nan"), 2 ** 31, -2 ** 31 - 1, 2 ** 32, 2 ** 32 + 5, np.int64(2 ** 32), np.float32(3)]
DIMS = bkv.dims(B=2, Hq=8, Hkv=2, D=128, N=1000, N_cap=1024, W=0, C=0, budget=256)


@pytest.mark.parametrize("bad", BAD)
def test_positions(bad):
    c, k = bkv.mx_cache(DIMS, device="cpu"), torch.zeros(2, 2, 1, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="^at must"):
        bkv.store_mx(DIMS, k, k, c, at=bad)
    with pytest.raises(ValueError, match="^at must"):
        bkv.load_mx(DIMS, c, k, k, at=bad)


@pytest.mark.parametrize("name", ["window", "sinks"])
@pytest.mark.parametrize("bad", BAD)
def test_windows(name, bad):
    q, c = torch.zeros(2, 8, 1, 128, dtype=torch.bfloat16), bkv.mx_cache(DIMS, device="cpu")
    kw = {"window": 5, "sinks": 1, name: bad}
    with pytest.raises(ValueError, match=f"^{name} must"):
        bkv.attend_window(DIMS, q, None, None, q, None, **kw)
    with pytest.raises(ValueError, match=f"^{name} must"):
        bkv.attend_mx(DIMS, q, c, q, None, **kw)
    for cache in ("plain", "mx"):
        with pytest.raises(ValueError, match=f"^{name} must"):
            PeriodicEviction(1, 1, 4, 2, 64, 64, None, n_beacon=4, n_recent=4, attention=True, device="cpu", cache=cache, **kw)


@pytest.mark.parametrize("good", [0, 7, -1, True, np.int32(7), np.int64(-3), 2 ** 31 - 1, -2 ** 31])
def test_integers_of_any_kind_pass(good):
    assert bkv._i32(good, "x") == int(good) and type(bkv._i32(good, "x")) in (int, bool)


@pytest.mark.parametrize("bad", [2 ** 31, -2 ** 31 - 1, 2 ** 32, 2 ** 32 + 5])
def test_prefixes(bad):
    q = torch.zeros(2, 8, 1, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="^P must"):
        bkv.attend_shared(DIMS, q, q, q, q, q, q, None, P=bad)

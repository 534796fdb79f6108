"""Host-side limits of the attention and mass-eviction entry points that the
basic refusals do not reach.  Only calls that fail validation are made: the
addresses stand in for device memory and are never dereferenced."""
import ctypes

import pytest

import paper_2609_04971_amd as bkv
from test_attend_host import attend, shared


@pytest.mark.parametrize("call", [attend, shared])
def test_a_scale_that_leaves_fp32_in_log2_units(call):
    # kernels work in log2 units: scale * log2(e) is finite up to 2.3587e38 (2^128 / log2(e))
    for scale in (2.36e38, 3.0e38, 3.4e38):
        assert ctypes.c_float(scale).value != float("inf")
        assert call(scale=scale, n=16) == bkv.ERR_INVALID
    assert call(scale=2.35e38, n=16) == bkv.ERR_WORKSPACE  # the next check


# what is written must not meet anything else: B 4, Hq 8, Hkv 2, D 128, 1000 of 1100 tokens, a prefix of 50 of 60
ROW = 256
SIZES = {"out": 4 * 8 * ROW, "lse": 4 * 8 * 4, "mass": (7 * 1100 + 1000) * 4, "ws": None, "q": 4 * 8 * ROW,
         "K": (7 * 1100 + 1000) * ROW, "V": (7 * 1100 + 1000) * ROW, "PK": (3 * 60 + 50) * ROW, "PV": (3 * 60 + 50) * ROW,
         "lens": 16, "p_lens": 8}
WRITTEN = ["out", "lse", "mass", "ws"]


def spread(groups, **moved):
    at = {k: (i + 1) << 36 for i, k in enumerate(SIZES)}
    at.update(moved)
    a = {k: ctypes.c_void_p(v) for k, v in at.items()}
    d = bkv.dims(B=4, Hq=8, Hkv=2, D=128, N=1000, N_cap=1100, W=8, C=0, budget=256, n_prefix=2)
    need = bkv.lib().bkv_attend_workspace_bytes(ctypes.byref(d), 1, 1, groups, 60 if groups else 0)
    if groups:
        return at, need, lambda: bkv.lib().bkv_attend_shared(
            ctypes.byref(d), 0, a["q"], 1, groups, a["PK"], a["PV"], 50, 60, a["p_lens"], a["K"], a["V"], a["lens"], 0.0, a["out"],
            a["lse"], a["mass"], a["ws"], need, None)
    return at, need, lambda: bkv.lib().bkv_attend(ctypes.byref(d), 0, a["q"], 1, a["K"], a["V"], a["lens"], 0.0, a["out"], a["lse"],
                                                  a["mass"], a["ws"], need, None)


@pytest.mark.parametrize("groups", [0, 2])
@pytest.mark.parametrize("written", WRITTEN)
@pytest.mark.parametrize("other", list(SIZES))
def test_outputs_over_anything_else(written, other, groups):
    if written == other or (not groups and other in ("PK", "PV", "p_lens")):
        return
    at, need, _ = spread(groups)
    size = {**SIZES, "ws": 1024}
    # at its start, across its end (16 bytes of it), and around all of it
    for to in (at[other], at[other] + (size[other] - 16 & ~15), at[other] - 16 if size[written] > 16 else at[other]):
        assert spread(groups, **{written: to})[2]() == bkv.ERR_INVALID


def _evict_spread(N, **moved):
    """evict_mass of 4 x 2 heads of N of 1100 tokens, budget 256, its arrays far apart but for those moved."""
    at = {k: (i + 1) << 36 for i, k in enumerate(("K", "V", "mass", "kept", "ws"))}
    at.update(moved)
    a = {k: ctypes.c_void_p(v) for k, v in at.items()}
    d = bkv.dims(B=4, Hq=8, Hkv=2, D=128, N=N, N_cap=1100, W=8, C=0, budget=256, n_prefix=2)
    need = bkv.lib().bkv_mass_workspace_bytes(ctypes.byref(d))
    size = {"K": (7 * 1100 + N) * ROW, "V": (7 * 1100 + N) * ROW, "mass": (7 * 1100 + N) * 4, "kept": 8 * min(N, 256) * 4, "ws": need}
    return at, size, lambda: bkv.lib().bkv_evict_mass(ctypes.byref(d), 0, a["K"], a["V"], a["mass"], a["kept"], a["ws"], need, None)


@pytest.mark.parametrize("N", [1000, 200])
@pytest.mark.parametrize("one", ["K", "V", "mass", "kept", "ws"])
@pytest.mark.parametrize("other", ["K", "V", "mass", "kept", "ws"])
def test_eviction_over_itself(one, other, N):
    if one == other:
        return
    at, size, _ = _evict_spread(N)
    for to in (at[other], at[other] + (size[other] - 16 & ~15), at[other] - 16):
        if {one, other} != {"K", "V"} or to != at[other]:  # K and V may be one array
            assert _evict_spread(N, **{one: to})[2]() == bkv.ERR_INVALID


# B, Hkv, G, T, N_cap, groups, P_cap: both sides of the items up to which a prefix is streamed (1024 of 32 rows and
# 128 keys), of 16, 32, 96 and 128 rows, of one split and many
SHAPES = [(4, 2, 4, 1, 1100, 2, 600), (64, 4, 4, 1, 500, 2, 6000), (48, 2, 7, 1, 900, 1, 40000), (6, 2, 8, 3, 20000, 3, 3000),
          (8, 8, 2, 8, 300, 8, 9000), (300, 1, 5, 2, 64, 30, 1000), (2, 1, 33, 1, 70000, 1, 70000), (1, 8, 4, 40, 5000, 1, 100),
          (16, 2, 16, 1, 2000, 4, 33000), (9, 3, 1, 97, 4000, 3, 129), (200, 8, 4, 1, 4096, 0, 0), (1, 2, 4, 1, 66000, 0, 0),
          (3, 2, 6, 11, 8000, 0, 0), (1, 4, 1, 700, 7000, 0, 0)]


@pytest.mark.parametrize("dtype", [bkv.BF16, bkv.F32])
@pytest.mark.parametrize("mass", [0, 1])
@pytest.mark.parametrize("B,Hkv,G,T,N_cap,groups,P_cap", SHAPES)
def test_one_workspace_size_covers_every_length_and_prefix(B, Hkv, G, T, N_cap, groups, P_cap, mass, dtype):
    """The size asked for with N 0 lets every N and P past the workspace's check: the next one, outputs that overlap,
    refuses the call then.  One byte less does not."""
    lib, out = bkv.lib(), ctypes.c_void_p(1 << 50)
    p = [ctypes.c_void_p((i + 1) << 44) for i in range(7)]
    for D in (64, 128):
        d = bkv.dims(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, N=0, N_cap=N_cap, W=0, C=0, budget=1).replace(dtype=dtype)
        need = lib.bkv_attend_workspace_bytes(ctypes.byref(d), T, mass, groups, P_cap)
        for N in sorted({0, 1, 127, 129, 1000, N_cap // 3, N_cap // 2, N_cap - 1, N_cap} & set(range(N_cap + 1))):
            dn = d.replace(N=N)
            for P in sorted({0, 1, 129, 1000, P_cap // 5, P_cap // 2, P_cap - 1, P_cap} & set(range(P_cap + 1))):
                for flags in (0, bkv.ATTEND_CAUSAL):
                    for n, code in ((need, bkv.ERR_INVALID), (need - 1, bkv.ERR_WORKSPACE)):
                        if not need and n < 0:
                            continue
                        m = p[5] if mass else None
                        if groups:
                            st = lib.bkv_attend_shared(ctypes.byref(dn), flags, p[0], T, groups, p[1], p[2], P, P_cap, None, p[3], p[4],
                                                       None, 0.0, out, out, m, p[6], n, None)
                        else:
                            st = lib.bkv_attend(ctypes.byref(dn), flags, p[0], T, p[3], p[4], None, 0.0, out, out, m, p[6], n, None)
                        assert st == code, (D, N, P, flags, n)


def test_no_room_for_logits_that_stay_on_the_chip():
    # 36 layers of 16 sequences, 8 kv-heads of 4 query heads, up to 4096 tokens: more heads than are ever split, and a head's
    # logits fit LDS, so that only the normalisers are left
    d = bkv.dims(B=576, Hq=32, Hkv=8, D=128, N=0, N_cap=4096, W=0, C=0, budget=1)
    rows, asked = 576 * 32, lambda **kw: bkv.lib().bkv_attend_workspace_bytes(ctypes.byref(d.replace(**kw)), 1, 1, 0, 0)  # noqa: E731
    assert asked() < 1 << 20
    assert asked(N_cap=5000) >= rows * 5000 * 4   # more than LDS holds
    assert asked(B=64) >= 64 * 32 * 4096 * 4      # split over two workgroups

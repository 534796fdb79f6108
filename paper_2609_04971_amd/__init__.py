"""Python binding of libbkv.so, the MI355X (gfx950) BeaconKV eviction step.

Argument marshalling only: every step of the path runs in the HIP kernels
behind include/bkv.h.  torch supplies device memory and the stream (work is
enqueued on torch's current stream).  Tensor shapes, dtypes, devices and
contiguity are checked here because the C ABI takes bare pointers and
cannot see them.  There is no fallback: the library is loaded on first use,
and if it is not built that first use raises ImportError.
"""
from __future__ import annotations

import ctypes
import operator
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libbkv.so")
_lib = None

OK, ERR_INVALID, ERR_SHAPE, ERR_DTYPE, ERR_WORKSPACE, ERR_HIP, ERR_DEVICE = range(7)
F32, BF16 = 0, 1
OP_BEACON_UPDATE, OP_SCORE, OP_TOPK, OP_COMPACT, OP_EVICT = range(5)

EXPORTS = ("bkv_validate", "bkv_workspace_bytes", "bkv_workspace_init", "bkv_device_status",
           "bkv_beacon_update", "bkv_score", "bkv_topk", "bkv_compact", "bkv_evict",
           "bkv_score_ex", "bkv_evict_ex", "bkv_fps", "bkv_fps_gather", "bkv_status_string",
           "bkv_abi_version", "bkv_compact_fill", "bkv_evict_noalloc", "bkv_append_rows",
           "bkv_attend", "bkv_attend_shared", "bkv_attend_workspace_bytes", "bkv_evict_mass",
           "bkv_mass_workspace_bytes", "bkv_store_mx", "bkv_load_mx", "bkv_attend_mx",
           "bkv_attend_window", "bkv_compact_mx", "bkv_evict_mass_mx")
APPEND_MAX = 4
SCORE_MEAN, SCORE_CAUSAL = 1, 2
ATTEND_CAUSAL = 1
EVICT_FILL = 1


class Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "Hq", "Hkv", "D", "N", "N_cap", "W", "C", "budget", "n_prefix", "dtype")]

    @property
    def G(self):
        return self.Hq // self.Hkv

    @property
    def P(self):
        return self.B * self.Hkv

    @property
    def n_keep(self):
        return min(self.budget, self.N)

    def replace(self, **kw):
        d = Dims()
        for n, _ in self._fields_:
            setattr(d, n, kw.get(n, getattr(self, n)))
        return d

    def __repr__(self):
        return "Dims(" + ", ".join(f"{n}={getattr(self, n)}" for n, _ in self._fields_) + ")"


class Rows(ctypes.Structure):
    """One array of append_rows: see bkv_rows."""
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("src_stride", ctypes.c_int64),
                ("dst_stride", ctypes.c_int64), ("heads", ctypes.c_int64)]


class _MxPtrs(ctypes.Structure):
    """See bkv_mx_cache."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("K", "KS", "V", "VS")]


class MxCache(NamedTuple):
    """A cache held in 4 bits: codes [B,Hkv,N_cap,D/2] and the blocks' bytes
    [B,Hkv,N_cap,D/32] of K and of V, all uint8."""
    K: torch.Tensor
    KS: torch.Tensor
    V: torch.Tensor
    VS: torch.Tensor


_APPEND = [Rows * n for n in range(APPEND_MAX + 1)]


def dims(B, Hq, Hkv, D, N, W, C, budget, n_prefix=0, dtype="bf16", N_cap=None) -> Dims:
    d = Dims()
    d.B, d.Hq, d.Hkv, d.D, d.N = B, Hq, Hkv, D, N
    d.N_cap = N if N_cap is None else N_cap
    d.W, d.C, d.budget, d.n_prefix = W, C, budget, n_prefix
    d.dtype = {"bf16": BF16, "fp32": F32, BF16: BF16, F32: F32}[dtype]
    return d


_P = ctypes.c_void_p
_D = ctypes.POINTER(Dims)
_S = ctypes.c_size_t
_I = ctypes.c_int32
_SIGS = {
    "bkv_validate": ([_D, ctypes.c_int32], ctypes.c_int),
    "bkv_workspace_bytes": ([_D, ctypes.c_int32], _S),
    "bkv_workspace_init": ([_D, _P, _S, _P], ctypes.c_int),
    "bkv_device_status": ([_P, _S, _P], ctypes.c_int),
    "bkv_beacon_update": ([_D, _P, ctypes.c_int32, _P, _P, _P, _P], ctypes.c_int),
    "bkv_score": ([_D, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_topk": ([_D, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_compact": ([_D, _P, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_compact_fill": ([_D, _P, _P, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_evict": ([_D, _P, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_score_ex": ([_D, _I, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_evict_ex": ([_D, _I, _P, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_evict_noalloc": ([_D, _I, _P, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, _P, _P], ctypes.c_int),
    "bkv_fps": ([_I] * 5 + [_P, _I, _P, _P], ctypes.c_int),
    "bkv_fps_gather": ([_I] * 5 + [_P, _I, _P, _I, _I, _P, _P, _P], ctypes.c_int),
    "bkv_append_rows": ([ctypes.POINTER(Rows), _I, _I, _P], ctypes.c_int),
    "bkv_attend_workspace_bytes": ([_D] + [_I] * 4, _S),
    "bkv_attend": ([_D, _I, _P, _I, _P, _P, _P, ctypes.c_float, _P, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_attend_shared": ([_D, _I, _P, _I, _I, _P, _P, _I, _I, _P, _P, _P, _P, ctypes.c_float, _P, _P, _P, _P, _S, _P],
                          ctypes.c_int),
    "bkv_mass_workspace_bytes": ([_D], _S),
    "bkv_evict_mass": ([_D, _I, _P, _P, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_store_mx": ([_D, _P, _P, _I, _I, _P, ctypes.POINTER(_MxPtrs), _P], ctypes.c_int),
    "bkv_load_mx": ([_D, ctypes.POINTER(_MxPtrs), _I, _I, _P, _P, _P, _P], ctypes.c_int),
    "bkv_attend_mx": ([_D, _I, _P, _I, ctypes.POINTER(_MxPtrs), _I, _I, _P, ctypes.c_float, _P, _P, _P, _P, _S, _P],
                      ctypes.c_int),
    "bkv_attend_window": ([_D, _P, _I, _P, _P, _I, _I, _P, ctypes.c_float, _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_compact_mx": ([_D, ctypes.POINTER(_MxPtrs), _P, _P, _S, _P], ctypes.c_int),
    "bkv_evict_mass_mx": ([_D, _I, ctypes.POINTER(_MxPtrs), _P, _P, _P, _S, _P], ctypes.c_int),
    "bkv_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "bkv_abi_version": ([], ctypes.c_int32),
}


def lib():
    """The loaded libbkv.so (loaded on first use; ImportError if not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2609_04971_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGS.items():
            fn = getattr(L, name)
            fn.argtypes = args
            fn.restype = res
        _lib = L
    return _lib


class BkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def status_string(st: int) -> str:
    return lib().bkv_status_string(st).decode()


def abi_version() -> int:
    return int(lib().bkv_abi_version())


def _check(st: int, where: str):
    if st != OK:
        raise BkvError(st, where)


def validate(d: Dims, op: int) -> int:
    """Host-only validation (no GPU needed); returns the bkv_status code."""
    return int(lib().bkv_validate(ctypes.byref(d), op))


def workspace_bytes(d: Dims, op: int = OP_EVICT) -> int:
    return int(lib().bkv_workspace_bytes(ctypes.byref(d), op))


# ---- marshalling helpers ---------------------------------------------------
def _stream():
    """The current stream of the current device, as a plain handle (what
    torch.cuda.current_stream().cuda_stream is, without a Stream object)."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _tdtype(d: Dims):
    return torch.bfloat16 if d.dtype == BF16 else torch.float32


def _ptr(t, shape=None, dtype=None, name="tensor", optional=False):
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _ws(ws):
    if ws is None:
        return None, 0
    if not isinstance(ws, torch.Tensor) or ws.device.type != "cuda" or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous CUDA tensor")
    return ctypes.c_void_p(ws.data_ptr()), ws.numel() * ws.element_size()


# ---- workspace -----------------------------------------------------------------
def workspace(d: Dims, op: int = OP_EVICT, device="cuda") -> torch.Tensor:
    """Allocate (through torch) and initialise a workspace for `op` on `d`."""
    n = workspace_bytes(d, op)
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=device)
    workspace_init(d, ws)
    return ws


def workspace_init(d: Dims, ws: torch.Tensor):
    p, n = _ws(ws)
    _check(lib().bkv_workspace_init(ctypes.byref(d), p, n, _stream()), "bkv_workspace_init")


def device_status(ws: torch.Tensor) -> int:
    """Synchronise the current stream and return the workspace's device status."""
    p, n = _ws(ws)
    return int(lib().bkv_device_status(p, n, _stream()))


# ---- operations ------------------------------------------------------------------
def beacon_update(d: Dims, q_new, beacons, counts, assign=None):
    """(a1) in place on beacons [B,Hkv,C,D] fp32 and counts [B,Hkv,C] int32."""
    T = q_new.shape[2]
    st = lib().bkv_beacon_update(
        ctypes.byref(d), _ptr(q_new, (d.B, d.Hq, T, d.D), _tdtype(d), "q_new"), T,
        _ptr(beacons, (d.B, d.Hkv, d.C, d.D), torch.float32, "beacons"),
        _ptr(counts, (d.B, d.Hkv, d.C), torch.int32, "counts"),
        _ptr(assign, (d.B, d.Hkv, T * d.G), torch.int32, "assign", optional=True), _stream())
    _check(st, "bkv_beacon_update")


def _rope(rope_cos, rope_sin, d):
    return (_ptr(rope_cos, (d.D // 2,), torch.float32, "rope_cos", optional=True),
            _ptr(rope_sin, (d.D // 2,), torch.float32, "rope_sin", optional=True))


def _flags(mean, causal):
    return (SCORE_MEAN if mean else 0) | (SCORE_CAUSAL if causal else 0)


def score(d: Dims, K, q_win, beacons, counts, scores, ws, row_lse=None, rope_cos=None, rope_sin=None,
          scale: float = 0.0, mean: bool = False, causal: bool = False):
    """(a2)+(a3): scores [B,Hkv,N] fp32 (and row_lse [B,Hkv,C+G*W]) written.
    mean / causal select the scoring options of bkv_score_ex."""
    rc, rs = _rope(rope_cos, rope_sin, d)
    wp, wn = _ws(ws)
    st = lib().bkv_score_ex(
        ctypes.byref(d), _flags(mean, causal), _ptr(K, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "K"),
        _ptr(q_win, (d.B, d.Hq, d.W, d.D), _tdtype(d), "q_win"),
        _ptr(beacons, (d.B, d.Hkv, d.C, d.D), torch.float32, "beacons"),
        _ptr(counts, (d.B, d.Hkv, d.C), torch.int32, "counts"), rc, rs, float(scale),
        _ptr(scores, (d.B, d.Hkv, d.N), torch.float32, "scores"),
        _ptr(row_lse, (d.B, d.Hkv, d.C + d.G * d.W), torch.float32, "row_lse", optional=True), wp, wn,
        _stream())
    _check(st, "bkv_score_ex")


def topk(d: Dims, scores, kept, ws=None):
    """(a4): kept [B,Hkv,min(budget,N)] int32 written, ascending."""
    wp, wn = _ws(ws)
    st = lib().bkv_topk(ctypes.byref(d), _ptr(scores, (d.B, d.Hkv, d.N), torch.float32, "scores"),
                       _ptr(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept"), wp, wn, _stream())
    _check(st, "bkv_topk")


def compact(d: Dims, K, V, kept, ws):
    """(a5): rows i < n of K and V become rows kept[i], in place."""
    wp, wn = _ws(ws)
    st = lib().bkv_compact(ctypes.byref(d), _ptr(K, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "K"),
                          _ptr(V, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "V"),
                          _ptr(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept"), wp, wn, _stream())
    _check(st, "bkv_compact")


def compact_fill(d: Dims, K, V, kept, src_of, ws):
    """Hole-filling compaction in place: kept rows below n stay, the holes
    below n take the kept rows past n; src_of [B,Hkv,n] int32 receives the
    old row now at each row."""
    wp, wn = _ws(ws)
    st = lib().bkv_compact_fill(ctypes.byref(d), _ptr(K, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "K"),
                                _ptr(V, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "V"),
                                _ptr(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept"),
                                _ptr(src_of, (d.B, d.Hkv, d.n_keep), torch.int32, "src_of"), wp, wn, _stream())
    _check(st, "bkv_compact_fill")


def evict(d: Dims, K, V, q_win, beacons, counts, ws, kept=None, scores=None, row_lse=None, rope_cos=None,
          rope_sin=None, scale: float = 0.0, mean: bool = False, causal: bool = False):
    """(a6): score -> select -> compact one layer in place (scoring options
    as in score)."""
    rc, rs = _rope(rope_cos, rope_sin, d)
    wp, wn = _ws(ws)
    st = lib().bkv_evict_ex(
        ctypes.byref(d), _flags(mean, causal), _ptr(K, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "K"),
        _ptr(V, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "V"),
        _ptr(q_win, (d.B, d.Hq, d.W, d.D), _tdtype(d), "q_win"),
        _ptr(beacons, (d.B, d.Hkv, d.C, d.D), torch.float32, "beacons"),
        _ptr(counts, (d.B, d.Hkv, d.C), torch.int32, "counts"), rc, rs, float(scale),
        _ptr(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept", optional=True),
        _ptr(scores, (d.B, d.Hkv, d.N), torch.float32, "scores", optional=True),
        _ptr(row_lse, (d.B, d.Hkv, d.C + d.G * d.W), torch.float32, "row_lse", optional=True), wp, wn,
        _stream())
    _check(st, "bkv_evict_ex")


def evict_noalloc(d: Dims, K, V, q_win, beacons, counts, kept=None, scores=None, row_lse=None, rope_cos=None,
                  rope_sin=None, scale: float = 0.0, mean: bool = False, causal: bool = False, status=None):
    """evict() with the library's fixed device array as its workspace: no
    workspace argument, nothing allocated.  status, an optional int32 tensor
    of one element, receives the call's device status (OK or ERR_DEVICE)."""
    rc, rs = _rope(rope_cos, rope_sin, d)
    st = lib().bkv_evict_noalloc(
        ctypes.byref(d), _flags(mean, causal), _ptr(K, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "K"),
        _ptr(V, (d.B, d.Hkv, d.N_cap, d.D), _tdtype(d), "V"),
        _ptr(q_win, (d.B, d.Hq, d.W, d.D), _tdtype(d), "q_win"),
        _ptr(beacons, (d.B, d.Hkv, d.C, d.D), torch.float32, "beacons"),
        _ptr(counts, (d.B, d.Hkv, d.C), torch.int32, "counts"), rc, rs, float(scale),
        _ptr(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept", optional=True),
        _ptr(scores, (d.B, d.Hkv, d.N), torch.float32, "scores", optional=True),
        _ptr(row_lse, (d.B, d.Hkv, d.C + d.G * d.W), torch.float32, "row_lse", optional=True),
        _ptr(status, (1,), torch.int32, "status", optional=True), _stream())
    _check(st, "bkv_evict_noalloc")


# ---- attention over the cache, eviction by accumulated weight ----------------------
def _arg(t, shape, dtype, name, dev):
    """Address of a contiguous tensor of this shape and type on GPU `dev`, the
    current device: its stream is where the work goes.  One test decides the
    usual case; what is wrong is found out only where it fails."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == dev
            and t.is_contiguous()):
        return t.data_ptr()
    _ptr(t, shape, dtype, name)
    raise ValueError(f"{name} is on GPU {t.get_device()}, the current device is {dev}")


def _i32(x, name):
    """x as a C int32, which ctypes would cut any other integer down to."""
    if type(x) is not int:
        try:
            x = operator.index(x)
        except TypeError:
            raise ValueError(f"{name} must be an integer, got {x!r}") from None
    if not -2**31 <= x < 2**31:
        raise ValueError(f"{name} must fit 32 bits, got {x}")
    return x


def _device_of(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    return torch._C._cuda_getDevice()


def _arg_ws(ws, dev):
    if ws is not None and (not isinstance(ws, torch.Tensor) or ws.get_device() != dev or not ws.is_contiguous()):
        raise ValueError("workspace must be a contiguous CUDA tensor on the current device")
    return (None, 0) if ws is None else (ws.data_ptr(), ws.nbytes)


def attend_workspace(d: Dims, T: int = 1, mass: bool = False, groups: int = 0, P_cap: int = 0, device="cuda"):
    """Workspace of attend (or, with groups and P_cap, attend_shared) for T
    queries on `d`, for every N <= N_cap and P <= P_cap; mass: whether calls
    pass a mass.  Nothing in it has to be initialised or outlives a call."""
    n = int(lib().bkv_attend_workspace_bytes(ctypes.byref(d), int(T), int(bool(mass)), int(groups), int(P_cap)))
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def _attend_rows(d, q, out, lens, lse, mass, dev):
    """What every attention takes beside its cache: T, the rows' type, and the addresses."""
    if q.dim() != 4:
        raise ValueError("q must be a tensor [B, Hq, T, D]")
    B, Hq, T, D = rows = q.shape
    dt = _tdtype(d)
    if (B, Hq, D) != (d.B, d.Hq, d.D):
        raise ValueError(f"q must have shape {(d.B, d.Hq, T, d.D)}, got {tuple(q.shape)}")
    return T, dt, (_arg(q, rows, dt, "q", dev), None if lens is None else _arg(lens, (B,), torch.int32, "lens", dev),
                   _arg(out, rows, dt, "out", dev),
                   None if lse is None else _arg(lse, (B, Hq, T), torch.float32, "lse", dev),
                   None if mass is None else _arg(mass, (B, d.Hkv, d.N_cap), torch.float32, "mass", dev))


def _attend_args(d, q, K, V, out, lens, lse, mass, dev):
    T, dt, (qp, lp, op, ep, mp) = _attend_rows(d, q, out, lens, lse, mass, dev)
    cache = (d.B, d.Hkv, d.N_cap, d.D)
    return T, dt, (qp, _arg(K, cache, dt, "K", dev), _arg(V, cache, dt, "V", dev), lp, op, ep, mp)


def attend(d: Dims, q, K, V, out, ws, lens=None, lse=None, mass=None, scale: float = 0.0, causal: bool = False):
    """Attention of the newest T queries q [B,Hq,T,D] (post-RoPE) over the
    cache: out [B,Hq,T,D] and, where given, lse [B,Hq,T] written, and every
    cached token's weights added to mass [B,Hkv,N_cap].  lens [B] int32:
    ragged lengths.  causal: query t sees the tokens up to its own."""
    dev = _device_of(q, "q")
    T, _, (qp, kp, vp, lp, op, ep, mp) = _attend_args(d, q, K, V, out, lens, lse, mass, dev)
    wp, wn = _arg_ws(ws, dev)
    st = lib().bkv_attend(ctypes.byref(d), ATTEND_CAUSAL if causal else 0, qp, T, kp, vp, lp, scale, op, ep, mp, wp, wn,
                          torch._C._cuda_getCurrentRawStream(dev))
    _check(st, "bkv_attend")


def attend_shared(d: Dims, q, PK, PV, K, V, out, ws, P: int | None = None, p_lens=None, lens=None, lse=None, mass=None,
                  scale: float = 0.0, causal: bool = False):
    """attend() for groups of consecutive sequences that share a prefix PK, PV
    [groups,Hkv,P_cap,D], of which the first P tokens are valid (default: all;
    p_lens [groups] int32: ragged).  mass collects the own tokens' weights."""
    P = None if P is None else _i32(int(P), "P")
    dev = _device_of(q, "q")
    if not isinstance(PK, torch.Tensor) or PK.dim() != 4:
        raise ValueError("PK must be a tensor [groups, Hkv, P_cap, D]")
    groups, P_cap = PK.shape[0], PK.shape[2]
    T, dt, (qp, kp, vp, lp, op, ep, mp) = _attend_args(d, q, K, V, out, lens, lse, mass, dev)
    shape = (groups, d.Hkv, P_cap, d.D)
    pk, pv = _arg(PK, shape, dt, "PK", dev), _arg(PV, shape, dt, "PV", dev)
    pl = None if p_lens is None else _arg(p_lens, (groups,), torch.int32, "p_lens", dev)
    wp, wn = _arg_ws(ws, dev)
    st = lib().bkv_attend_shared(ctypes.byref(d), ATTEND_CAUSAL if causal else 0, qp, T, groups, pk, pv,
                                 P_cap if P is None else P, P_cap, pl, kp, vp, lp, scale, op, ep, mp, wp, wn,
                                 torch._C._cuda_getCurrentRawStream(dev))
    _check(st, "bkv_attend_shared")


def attend_window(d: Dims, q, K, V, out, ws, window: int, sinks: int = 0, lens=None, lse=None, scale: float = 0.0):
    """attend() where query t, the cache's token p = len - T + t, sees the tokens
    j <= p with j > p - window or j < sinks.  The workspace is that of
    attend_workspace(d, T)."""
    window, sinks = _i32(window, "window"), _i32(sinks, "sinks")
    dev = _device_of(q, "q")
    T, _, (qp, kp, vp, lp, op, ep, _) = _attend_args(d, q, K, V, out, lens, lse, None, dev)
    wp, wn = _arg_ws(ws, dev)
    st = lib().bkv_attend_window(ctypes.byref(d), qp, T, kp, vp, window, sinks, lp, scale, op, ep, wp, wn,
                                 torch._C._cuda_getCurrentRawStream(dev))
    _check(st, "bkv_attend_window")


def mass_workspace(d: Dims, device="cuda") -> torch.Tensor:
    """Allocate and initialise a workspace of evict_mass, for every N <= N_cap."""
    n = int(lib().bkv_mass_workspace_bytes(ctypes.byref(d)))
    ws = torch.empty(max(n, 256), dtype=torch.uint8, device=device)
    workspace_init(d, ws)
    return ws


def evict_mass(d: Dims, K, V, mass, ws, kept=None, fill: bool = False):
    """Keep the prefix, the last W tokens and the largest masses of each head:
    K, V and mass [B,Hkv,N_cap] compacted in place (fill: the layout of
    compact_fill), mass 0 from the budget to N.  kept [B,Hkv,min(budget,N)]
    int32, optional, receives the old row now at each row."""
    dev = _device_of(K, "K")
    dt, cache = _tdtype(d), (d.B, d.Hkv, d.N_cap, d.D)
    kp, vp = _arg(K, cache, dt, "K", dev), _arg(V, cache, dt, "V", dev)
    mp = _arg(mass, cache[:3], torch.float32, "mass", dev)
    op = None if kept is None else _arg(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept", dev)
    wp, wn = _arg_ws(ws, dev)
    st = lib().bkv_evict_mass(ctypes.byref(d), EVICT_FILL if fill else 0, kp, vp, mp, op, wp, wn,
                              torch._C._cuda_getCurrentRawStream(dev))
    _check(st, "bkv_evict_mass")


# ---- the cache in 4 bits ----------------------------------------------------------
def mx_cache(d: Dims, device="cuda") -> MxCache:
    """Allocate (through torch) a 4-bit cache of `d`; rows hold nothing until they
    are stored."""
    return MxCache(*(torch.empty(d.B, d.Hkv, d.N_cap, n, dtype=torch.uint8, device=device)
                     for n in (d.D // 2, d.D // 32) * 2))


def _arg_mx(d, cache, dev):
    if not isinstance(cache, MxCache):
        raise ValueError("cache must be an MxCache")
    K, KS, V, VS = cache
    rows, D, u8 = (d.B, d.Hkv, d.N_cap), d.D, torch.uint8
    codes, scales = (*rows, D // 2), (*rows, D // 32)
    return _MxPtrs(_arg(K, codes, u8, "cache.K", dev), _arg(KS, scales, u8, "cache.KS", dev), _arg(V, codes, u8, "cache.V", dev),
                   _arg(VS, scales, u8, "cache.VS", dev))


def _mx_args(d, k, v, cache, at):
    each = isinstance(at, torch.Tensor)
    first = 0 if each else _i32(at, "at")
    t, name = (k, "k") if k is not None else (v, "v")
    if t is None:
        raise ValueError("k or v is required")
    dev = _device_of(t, name)
    if t.dim() != 4:
        raise ValueError(f"{name} must be a tensor [B, Hkv, T, D]")
    B, T, dt = d.B, t.shape[2], _tdtype(d)
    shape = (B, d.Hkv, T, d.D)
    kp = None if k is None else _arg(k, shape, dt, "k", dev)
    vp = None if v is None else _arg(v, shape, dt, "v", dev)
    ap = _arg(at, (B,), torch.int32, "at", dev) if each else None
    return kp, vp, T, first, ap, _arg_mx(d, cache, dev), torch._C._cuda_getCurrentRawStream(dev)


def store_mx(d: Dims, k, v, cache: MxCache, at=0):
    """Rows k, v [B,Hkv,T,D] into rows at.. of the 4-bit cache; at: a position, or
    [B] int32 with one for each sequence (rows outside of the cache are not
    stored).  k or v may be None: that side is left as it was."""
    kp, vp, T, first, ap, cp, s = _mx_args(d, k, v, cache, at)
    _check(lib().bkv_store_mx(ctypes.byref(d), kp, vp, T, first, ap, ctypes.byref(cp), s), "bkv_store_mx")


def load_mx(d: Dims, cache: MxCache, k, v, at=0):
    """The values of rows at.. of the 4-bit cache into k, v [B,Hkv,T,D], exact;
    k or v may be None."""
    kp, vp, T, first, ap, cp, s = _mx_args(d, k, v, cache, at)
    _check(lib().bkv_load_mx(ctypes.byref(d), ctypes.byref(cp), T, first, ap, kp, vp, s), "bkv_load_mx")


def attend_mx(d: Dims, q, cache: MxCache, out, ws, lens=None, lse=None, mass=None, scale: float = 0.0,
              causal: bool = False, window: int = 0, sinks: int = 0):
    """attend() over a 4-bit cache; q and out have the dims' type.  window > 0: as
    attend_window() (then causal, and without mass)."""
    window, sinks = _i32(window, "window"), _i32(sinks, "sinks")
    dev = _device_of(q, "q")
    T, _, (qp, lp, op, ep, mp) = _attend_rows(d, q, out, lens, lse, mass, dev)
    cp = _arg_mx(d, cache, dev)
    wp, wn = _arg_ws(ws, dev)
    st = lib().bkv_attend_mx(ctypes.byref(d), ATTEND_CAUSAL if causal else 0, qp, T, ctypes.byref(cp), window, sinks, lp, scale,
                             op, ep, mp, wp, wn, torch._C._cuda_getCurrentRawStream(dev))
    _check(st, "bkv_attend_mx")


def compact_mx(d: Dims, cache: MxCache, kept, ws):
    """compact() of a 4-bit cache."""
    dev = _device_of(kept, "kept")
    cp = _arg_mx(d, cache, dev)
    wp, wn = _arg_ws(ws, dev)
    kp = _arg(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept", dev)
    _check(lib().bkv_compact_mx(ctypes.byref(d), ctypes.byref(cp), kp, wp, wn, torch._C._cuda_getCurrentRawStream(dev)),
           "bkv_compact_mx")


def evict_mass_mx(d: Dims, cache: MxCache, mass, ws, kept=None, fill: bool = False):
    """evict_mass() of a 4-bit cache."""
    dev = _device_of(mass, "mass")
    cp = _arg_mx(d, cache, dev)
    mp = _arg(mass, (d.B, d.Hkv, d.N_cap), torch.float32, "mass", dev)
    op = None if kept is None else _arg(kept, (d.B, d.Hkv, d.n_keep), torch.int32, "kept", dev)
    wp, wn = _arg_ws(ws, dev)
    st = lib().bkv_evict_mass_mx(ctypes.byref(d), EVICT_FILL if fill else 0, ctypes.byref(cp), mp, op, wp, wn,
                                 torch._C._cuda_getCurrentRawStream(dev))
    _check(st, "bkv_evict_mass_mx")


# ---- appending a step's rows -------------------------------------------------------
def append_rows(writes):
    """dst[:, :, row] = src for every (dst [B, H, rows, D], row, src [B, H, D])
    of `writes`, as one launch where bkv_append_rows can read and write them
    (plain tensors of one dtype on one GPU, whole rows of 16-byte chunks, one
    stride from head to head), else array by array."""
    n = len(writes)
    if 0 < n <= APPEND_MAX:
        arrays = _APPEND[n]()
        d0 = writes[0][0]
        dtype, dev, D = d0.dtype, d0.get_device(), d0.shape[-1]
        row_bytes = D * d0.element_size()
        if dev >= 0 and dev == torch.cuda.current_device() and row_bytes % 16 == 0:
            for a, (dst, row, src) in zip(arrays, writes):
                B, H, rows, Dd = dst.shape
                if (type(src) is not torch.Tensor or type(dst) is not torch.Tensor or Dd != D or src.shape != (B, H, D)
                        or src.dtype is not dtype or dst.dtype is not dtype or src.get_device() != dev
                        or dst.get_device() != dev or src.requires_grad or dst.requires_grad or src.is_neg()
                        or dst.is_neg() or not 0 <= row < rows or not dst.is_contiguous()):
                    break
                s0, s1, s2 = src.stride()
                if s2 != 1 or (B > 1 and s0 != H * s1):
                    break
                sp, stride = src.data_ptr(), s1 * d0.element_size()
                dp = dst.data_ptr() + row * row_bytes
                if (sp | stride | dp) & 15:
                    break
                a.src, a.dst, a.src_stride, a.dst_stride, a.heads = sp, dp, stride, rows * row_bytes, B * H
            else:
                _check(lib().bkv_append_rows(arrays, n, row_bytes, _stream()), "bkv_append_rows")
                return
    for dst, row, src in writes:
        dst[:, :, row] = src


# ---- Continual FPS -------------------------------------------------------------
_FPS_DT = {torch.bfloat16: BF16, torch.float32: F32}


def _fps_src(q, n, name):
    if not isinstance(q, torch.Tensor) or q.dim() < 2:
        raise ValueError(f"{name} must be a tensor [..., rows, D]")
    if q.dtype not in _FPS_DT:
        raise ValueError(f"{name} must be bfloat16 or float32, got {q.dtype}")
    rows, D = q.shape[-2], q.shape[-1]
    H = q.numel() // max(1, rows * D) if rows * D else 0
    n = rows if n is None else int(n)
    return _ptr(q, name=name), H, rows, D, n


def fps(q, m: int, n: int | None = None, picks=None):
    """Farthest point sampling (Appendix D.1, Algorithm 1) of the first n rows
    (default: all) of every head of q [..., rows, D]: returns picks
    [..., min(m, n)] int32 in selection order."""
    qp, H, rows, D, n = _fps_src(q, n, "q")
    k = max(0, min(int(m), n))
    shape = tuple(q.shape[:-2]) + (k,)
    if picks is None:
        picks = torch.empty(shape, dtype=torch.int32, device=q.device)
    pp = _ptr(picks, shape, torch.int32, "picks")
    _check(lib().bkv_fps(H, n, int(m), D, _FPS_DT[q.dtype], qp, rows, pp, _stream()), "bkv_fps")
    return picks


def fps_gather(src, m: int, dst=None, n: int | None = None, picks=None, counts=None):
    """FPS of the first n rows of every head of src [..., rows, D], then rows
    0..k-1 of dst [..., dst_rows, D] (default: src itself, in place) become
    the picked rows in selection order, k = min(m, n) (Section 4.2, Eq.
    fps_q).  dst may be float32 for a bfloat16 src.  picks [..., k] and
    counts [..., dst_rows] are optional outputs.  Returns dst."""
    sp, H, rows, D, n = _fps_src(src, n, "src")
    k = max(0, min(int(m), n))
    if dst is None:
        dst = src
    if dst.dtype not in _FPS_DT or dst.dim() != src.dim() or dst.shape[:-2] != src.shape[:-2] \
            or dst.shape[-1] != D:
        raise ValueError("dst must be [..., dst_rows, D] with the leading shape and D of src")
    dst_rows = dst.shape[-2]
    lead = tuple(src.shape[:-2])
    pp = _ptr(picks, lead + (k,), torch.int32, "picks", optional=True)
    cp = _ptr(counts, lead + (dst_rows,), torch.int32, "counts", optional=True)
    st = lib().bkv_fps_gather(H, n, int(m), D, _FPS_DT[src.dtype], sp, rows, _ptr(dst, name="dst"),
                              _FPS_DT[dst.dtype], dst_rows, pp, cp, _stream())
    _check(st, "bkv_fps_gather")
    return dst

"""Python binding of libmita (the gfx950 MiTA forward library).

Argument marshalling only: every step of the forward runs in the HIP kernels
behind the C ABI declared in include/mita.h. Tensors are torch device tensors
(torch provides device memory and the current HIP stream); the functions
allocate outputs and workspaces with torch when they are not given.

There is no CPU fallback: if libmita.so is missing or no GPU is visible the
calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import operator
import os
from dataclasses import dataclass
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmita.so")

MITA_OK, MITA_ERR_INVALID_ARG, MITA_ERR_UNSUPPORTED, MITA_ERR_WORKSPACE, MITA_ERR_HIP = range(5)
MITA_F32, MITA_BF16 = 0, 1
MITA_FLAG_STAGED_GATHER = 0x1
MITA_FLAG_FULL_SCORES = 0x2
WS_FORWARD, WS_SCORES, WS_TOPK, WS_ROUTE, WS_ATTEND, WS_BACKWARD, WS_TOME = range(7)
NUM_STAGES = 6
MAX_LAUNCHES = 32
STAGES = ("landmarks", "scores", "topk", "gather", "route", "attend")
MAX_N = 65536
MAX_S = 4

EXPORTED = ("mita_check", "mita_workspace_size", "mita_status_string", "mita_last_error", "mita_forward",
            "mita_landmarks", "mita_scores", "mita_topk", "mita_gather", "mita_route", "mita_attend",
            "mita_timer_create", "mita_timer_destroy", "mita_timer_reset", "mita_timer_read",
            "mita_forward_timed", "mita_forward_fallbacks", "mita_select_plan", "mita_timer_launches",
            "mita_forward_noalloc", "mita_landmarks_select", "mita_forward_lm", "mita_forward_lm_timed",
            "mita_backward", "mita_backward_timed", "mita_landmarks_tome",
            "mita_dense_check", "mita_dense_workspace_size", "mita_dense_forward", "mita_dense_backward",
            "mita_norm_check", "mita_norm_workspace_size", "mita_norm_forward", "mita_norm_backward")


class CfgStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "H", "N", "d", "grid_h", "grid_w", "M", "lm_h", "lm_w", "k", "s", "use_shared",
                 "use_routed", "dtype")] + [("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class StridesStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("b", "h", "n")]


class DenseCfgStruct(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("B", "H", "H_kv", "N", "N_k", "d", "dtype", "left", "right")]
                + [("scale", ctypes.c_float)]
                + [(n, StridesStruct) for n in ("q", "k", "v", "o", "dO", "dq", "dk", "dv")])


class NormCfgStruct(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32 * 3), ("C", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("wdtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("x", ctypes.c_int64 * 3), ("y", ctypes.c_int64 * 3), ("dy", ctypes.c_int64 * 3),
                ("dx", ctypes.c_int64 * 3)]


class MitaError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"mita status {status}: {msg}")
        self.status = status


_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libmita.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found: build it with `python -m paper_2602_01219_amd.build`")
    lib = ctypes.CDLL(path)
    P, I, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    cfgp = ctypes.POINTER(CfgStruct)
    densep, normp = ctypes.POINTER(DenseCfgStruct), ctypes.POINTER(NormCfgStruct)
    sig = {
        "mita_check": (I, [cfgp]),
        "mita_workspace_size": (Z, [cfgp, I]),
        "mita_status_string": (ctypes.c_char_p, [I]),
        "mita_last_error": (ctypes.c_char_p, []),
        "mita_forward": (I, [cfgp, P, P, P, P, P, Z, P]),
        "mita_forward_timed": (I, [cfgp, P, P, P, P, P, Z, P, P]),
        "mita_forward_noalloc": (I, [cfgp, P, P, P, P, P]),
        "mita_forward_fallbacks": (I, [cfgp, P, Z, ctypes.POINTER(ctypes.c_int64), P]),
        "mita_select_plan": (I, [cfgp] + [ctypes.POINTER(ctypes.c_int32)] * 4),
        "mita_landmarks": (I, [cfgp, P, P, P]),
        "mita_landmarks_select": (I, [cfgp, P, P, P, P]),
        "mita_forward_lm": (I, [cfgp, P, P, P, P, P, P, Z, P]),
        "mita_forward_lm_timed": (I, [cfgp, P, P, P, P, P, P, Z, P, P]),
        "mita_backward": (I, [cfgp, P, P, P, P, P, P, P, P, P, Z, P]),
        "mita_landmarks_tome": (I, [cfgp, P, P, P, P, Z, P]),
        "mita_backward_timed": (I, [cfgp, P, P, P, P, P, P, P, P, P, Z, P, P]),
        "mita_scores": (I, [cfgp, P, P, P, P, P, P, Z, P]),
        "mita_dense_check": (I, [densep]),
        "mita_dense_workspace_size": (Z, [densep, I]),
        "mita_dense_forward": (I, [densep, P, P, P, P, P, P, P, P, Z, P]),
        "mita_dense_backward": (I, [densep, P, P, P, P, P, P, P, P, P, P, P, P, Z, P]),
        "mita_norm_check": (I, [normp]),
        "mita_norm_workspace_size": (Z, [normp]),
        "mita_norm_forward": (I, [normp, P, P, P, P, P, P, P]),
        "mita_norm_backward": (I, [normp, P, P, P, P, P, P, P, P, P, Z, P]),
        "mita_topk": (I, [cfgp, P, P, P, Z, P]),
        "mita_gather": (I, [cfgp, P, P, P, P, P, P]),
        "mita_route": (I, [cfgp, P, P, P, P, P, P, Z, P]),
        "mita_attend": (I, [cfgp, P, P, P, P, P, P, P, P, P, Z, P]),
        "mita_timer_create": (I, [ctypes.POINTER(P), I]),
        "mita_timer_destroy": (I, [P]),
        "mita_timer_reset": (I, [P]),
        "mita_timer_read": (I, [P, ctypes.POINTER(ctypes.c_float), I, ctypes.POINTER(I)]),
        "mita_timer_launches": (I, [P, I, I, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_int32),
                                    ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32)]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


def _check(status: int):
    if status != MITA_OK:
        lib = load_library()
        raise MitaError(status, lib.mita_last_error().decode() or lib.mita_status_string(status).decode())


@dataclass(frozen=True)
class Config:
    """Problem description (mirrors mita_cfg_t)."""
    B: int
    H: int
    N: int
    d: int
    grid_h: int
    grid_w: int
    M: int
    lm_h: int
    lm_w: int
    k: int
    dtype: str = "bf16"          # "f32" | "bf16"
    use_shared: int = 1
    use_routed: int = 1
    s: int = 1
    scale: float = 0.0           # 0 -> 1/sqrt(d)
    staged_gather: bool = False
    full_scores: bool = False    # store S and select from it instead of the fused selection

    @staticmethod
    def from_workload(wl, **kw) -> "Config":
        c = dict(B=wl.B, H=wl.H, N=wl.N, d=wl.d, grid_h=wl.grid_h, grid_w=wl.grid_w, M=wl.M, lm_h=wl.lm_h,
                 lm_w=wl.lm_w, k=wl.k, dtype=wl.dtype, use_shared=wl.use_shared, use_routed=wl.use_routed)
        c.update(kw)
        return Config(**c)

    def struct(self) -> CfgStruct:
        return CfgStruct(self.B, self.H, self.N, self.d, self.grid_h, self.grid_w, self.M, self.lm_h, self.lm_w,
                         self.k, self.s, self.use_shared, self.use_routed,
                         MITA_F32 if self.dtype == "f32" else MITA_BF16, float(self.scale),
                         (MITA_FLAG_STAGED_GATHER if self.staged_gather else 0)
                         | (MITA_FLAG_FULL_SCORES if self.full_scores else 0))

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == "f32" else torch.bfloat16

    @property
    def eff_scale(self) -> float:
        return self.scale if self.scale else 1.0 / math.sqrt(self.d)


def _p(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def check(cfg: Config) -> int:
    return load_library().mita_check(ctypes.byref(cfg.struct()))


def workspace_size(cfg: Config, which: int = WS_FORWARD) -> int:
    return int(load_library().mita_workspace_size(ctypes.byref(cfg.struct()), which))


def _ws(cfg, which, ws, device):
    n = workspace_size(cfg, which)
    if ws is None and n:
        ws = torch.empty(n, dtype=torch.uint8, device=device)
    return ws, (ws.numel() if ws is not None else 0)


def _dev(t):
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU")
    return t.device


def forward(cfg: Config, q, k, v, o=None, ws=None, stream=None, timer: "Timer" = None, q_lm=None):
    """MiTA forward: o [B, H, N, d]. With q_lm [B, H, M, d] given (e.g. from
    landmarks_select), the forward uses those landmark queries instead of
    pooling them (mita_forward_lm)."""
    lib = load_library()
    dev = _dev(q)
    if o is None:
        o = torch.empty_like(q)
    ws, nws = _ws(cfg, WS_FORWARD, ws, dev)
    c = cfg.struct()
    if q_lm is not None:
        if timer is None:
            st = lib.mita_forward_lm(ctypes.byref(c), _p(q), _p(k), _p(v), _p(q_lm), _p(o), _p(ws), nws,
                                     _stream(stream))
        else:
            st = lib.mita_forward_lm_timed(ctypes.byref(c), _p(q), _p(k), _p(v), _p(q_lm), _p(o), _p(ws), nws,
                                           _stream(stream), timer.handle)
        _check(st)
        return o
    if timer is None:
        st = lib.mita_forward(ctypes.byref(c), _p(q), _p(k), _p(v), _p(o), _p(ws), nws, _stream(stream))
    else:
        st = lib.mita_forward_timed(ctypes.byref(c), _p(q), _p(k), _p(v), _p(o), _p(ws), nws, _stream(stream),
                                    timer.handle)
    _check(st)
    return o


def backward(cfg: Config, q, k, v, o, dO, dq=None, dk=None, dv=None, ws=None, stream=None,
             timer: "Timer" = None):
    """Gradients (dq, dk, dv) [B, H, N, d] of the forward's output o for the
    upstream gradient dO, the top-k sets and routing held fixed
    (mita_backward)."""
    lib = load_library()
    dev = _dev(q)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    ws, nws = _ws(cfg, WS_BACKWARD, ws, dev)
    c = cfg.struct()
    args = [ctypes.byref(c), _p(q), _p(k), _p(v), _p(o), _p(dO), _p(dq), _p(dk), _p(dv), _p(ws), nws, _stream(stream)]
    if timer is None:
        _check(lib.mita_backward(*args))
    else:
        _check(lib.mita_backward_timed(*args, timer.handle))
    return dq, dk, dv


NOALLOC_SCRATCH_BYTES = 64 << 20


def forward_noalloc(cfg: Config, q, k, v, o=None, stream=None):
    """MiTA forward with the library's static scratch as workspace (no
    allocation by the library; only the output is allocated here if not
    given). Raises MitaError(MITA_ERR_WORKSPACE) if the forward needs more
    than NOALLOC_SCRATCH_BYTES of workspace."""
    lib = load_library()
    _dev(q)
    if o is None:
        o = torch.empty_like(q)
    _check(lib.mita_forward_noalloc(ctypes.byref(cfg.struct()), _p(q), _p(k), _p(v), _p(o), _stream(stream)))
    return o


def forward_fallbacks(cfg: Config, ws, stream=None) -> int:
    """Landmark rows whose fused top-k selection fell back to the full score
    row in the last forward on workspace ws (synchronises the stream)."""
    n = ctypes.c_int64()
    _check(load_library().mita_forward_fallbacks(ctypes.byref(cfg.struct()), _p(ws), ws.numel(), ctypes.byref(n),
                                                 _stream(stream)))
    return n.value


def select_plan(cfg: Config) -> dict:
    """How the forward selects the top-k sets (host only): fused in the score
    pass (with its sample size, pivot rank and list cap) or from the stored
    score matrix."""
    v = [ctypes.c_int32() for _ in range(4)]
    _check(load_library().mita_select_plan(ctypes.byref(cfg.struct()), *[ctypes.byref(x) for x in v]))
    return dict(zip(("fused", "ns", "rank", "cap"), (x.value for x in v)))


def landmarks(cfg: Config, q, q_lm=None, stream=None):
    lib = load_library()
    if q_lm is None:
        q_lm = torch.empty((cfg.B, cfg.H, cfg.M, cfg.d), dtype=q.dtype, device=_dev(q))
    _check(lib.mita_landmarks(ctypes.byref(cfg.struct()), _p(q), _p(q_lm), _stream(stream)))
    return q_lm


def landmarks_select(cfg: Config, q, sel, q_lm=None, stream=None):
    """Random-selection landmarks: q_lm[b, h, i] = q[b, h, sel[b, h, i]];
    sel: [B, H, M] int32 device tensor of drawn token indices."""
    lib = load_library()
    if sel.dtype != torch.int32 or tuple(sel.shape) != (cfg.B, cfg.H, cfg.M) or not sel.is_contiguous():
        raise ValueError("sel must be a contiguous [B, H, M] int32 tensor")
    if q_lm is None:
        q_lm = torch.empty((cfg.B, cfg.H, cfg.M, cfg.d), dtype=q.dtype, device=_dev(q))
    _check(lib.mita_landmarks_select(ctypes.byref(cfg.struct()), _p(q), _p(sel), _p(q_lm), _stream(stream)))
    return q_lm


def landmarks_tome(cfg: Config, q, q_lm=None, want_assign=True, ws=None, stream=None):
    """Token-merging landmarks: (q_lm [B, H, M, d], assign [B, H, N] int32 or
    None), mita_landmarks_tome."""
    lib = load_library()
    dev = _dev(q)
    if q_lm is None:
        q_lm = torch.empty((cfg.B, cfg.H, cfg.M, cfg.d), dtype=q.dtype, device=dev)
    assign = torch.empty((cfg.B, cfg.H, cfg.N), dtype=torch.int32, device=dev) if want_assign else None
    ws, nws = _ws(cfg, WS_TOME, ws, dev)
    _check(lib.mita_landmarks_tome(ctypes.byref(cfg.struct()), _p(q), _p(q_lm), _p(assign), _p(ws), nws,
                                   _stream(stream)))
    return q_lm, assign


def scores(cfg: Config, q_lm, k, v=None, want_scores=True, want_v_lm=True, ws=None, stream=None):
    """Returns (scores [B,H,M,N] fp32 or None, v_lm [B,H,M,d] or None)."""
    lib = load_library()
    dev = _dev(q_lm)
    S = torch.empty((cfg.B, cfg.H, cfg.M, cfg.N), dtype=torch.float32, device=dev) if want_scores else None
    v_lm = torch.empty((cfg.B, cfg.H, cfg.M, cfg.d), dtype=q_lm.dtype, device=dev) if want_v_lm else None
    ws, nws = _ws(cfg, WS_SCORES, ws, dev) if want_v_lm else (None, 0)
    _check(lib.mita_scores(ctypes.byref(cfg.struct()), _p(q_lm), _p(k), _p(v), _p(S), _p(v_lm), _p(ws), nws,
                           _stream(stream)))
    return S, v_lm


def topk(cfg: Config, S, idx=None, stream=None):
    lib = load_library()
    if idx is None:
        idx = torch.empty((cfg.B, cfg.H, cfg.M, cfg.k), dtype=torch.int32, device=_dev(S))
    _check(lib.mita_topk(ctypes.byref(cfg.struct()), _p(S), _p(idx), None, 0, _stream(stream)))
    return idx


def gather(cfg: Config, k, v, idx, stream=None):
    lib = load_library()
    shape = (cfg.B, cfg.H, cfg.M, cfg.k, cfg.d)
    kx = torch.empty(shape, dtype=k.dtype, device=_dev(k))
    vx = torch.empty(shape, dtype=v.dtype, device=_dev(v))
    _check(lib.mita_gather(ctypes.byref(cfg.struct()), _p(k), _p(v), _p(idx), _p(kx), _p(vx), _stream(stream)))
    return kx, vx


def route(cfg: Config, q, q_lm, ws=None, stream=None):
    """Returns (expert, perm, offsets) int32: with s = 1 expert [B,H,N],
    perm [B,H,N], offsets [B,H,M+1]; with s > 1 expert [B,H,N,s] (rank
    order), perm [B,H,N*s] (pair ids n*s+j grouped into 2M groups),
    offsets [B,H,2M+1]."""
    lib = load_library()
    dev = _dev(q)
    s = cfg.s if cfg.use_routed else 1
    G = 2 * cfg.M if s > 1 else cfg.M
    expert = torch.empty((cfg.B, cfg.H, cfg.N) + ((s,) if s > 1 else ()), dtype=torch.int32, device=dev)
    perm = torch.empty((cfg.B, cfg.H, cfg.N * s), dtype=torch.int32, device=dev)
    offsets = torch.empty((cfg.B, cfg.H, G + 1), dtype=torch.int32, device=dev)
    ws, nws = _ws(cfg, WS_ROUTE, ws, dev)
    _check(lib.mita_route(ctypes.byref(cfg.struct()), _p(q), _p(q_lm), _p(expert), _p(perm), _p(offsets), _p(ws),
                          nws, _stream(stream)))
    return expert, perm, offsets


def attend(cfg: Config, q, q_lm, v_lm, k_x, v_x, perm, offsets, o=None, ws=None, stream=None):
    lib = load_library()
    dev = _dev(q)
    if o is None:
        o = torch.empty_like(q)
    ws, nws = _ws(cfg, WS_ATTEND, ws, dev)
    _check(lib.mita_attend(ctypes.byref(cfg.struct()), _p(q), _p(q_lm), _p(v_lm), _p(k_x), _p(v_x), _p(perm),
                           _p(offsets), _p(o), _p(ws), nws, _stream(stream)))
    return o


# ---------------------------------------------------------------------------
# Dense attention and layer norm
# ---------------------------------------------------------------------------
class _Planned:
    """Keeps the plans of its calls (see _Plan) out of copies and pickles."""

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_plans"}


@dataclass(frozen=True)
class DenseConfig(_Planned):
    """Dense attention problem (mita_dense_cfg_t without the strides, which are
    the tensors' own). H_kv = 0 means H, N_k = 0 means N; a query at position p
    sees the keys p - left .. p + right (-1: no bound; right = 0: causal)."""
    B: int
    H: int
    N: int
    d: int
    H_kv: int = 0
    N_k: int = 0
    dtype: str = "bf16"          # "f32" | "bf16"
    left: int = -1
    right: int = -1
    scale: float = 0.0           # 0 -> 1/sqrt(d)

    @property
    def q_shape(self):
        return (self.B, self.H, self.N, self.d)

    @property
    def k_shape(self):
        return (self.B, self.H_kv or self.H, self.N_k or self.N, self.d)

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == "f32" else torch.bfloat16

    def struct(self, **tensors) -> DenseCfgStruct:
        B, H, N, d, left, right = (_int32(n, getattr(self, n)) for n in ("B", "H", "N", "d", "left", "right"))
        c = DenseCfgStruct(B, H, _int32("H_kv", self.H_kv) or H, N, _int32("N_k", self.N_k) or N, d,
                           _dtype_code(self.dtype), left, right, _fp32("scale", self.scale))
        for name, t in tensors.items():
            setattr(c, name, StridesStruct(*_strides(t)))
        return c


@dataclass(frozen=True)
class NormConfig(_Planned):
    """Layer norm of rows of C elements (mita_norm_cfg_t without the strides):
    rows is the shape in front of the last dimension, up to three dimensions."""
    rows: tuple
    C: int
    dtype: str = "bf16"          # x, y and their gradients
    wdtype: str = "f32"          # weight, bias and their gradients
    eps: float = 1e-5

    @property
    def shape(self):
        return tuple(self.rows) + (self.C,)

    @property
    def torch_dtype(self):
        return torch.float32 if self.dtype == "f32" else torch.bfloat16

    @property
    def torch_wdtype(self):
        return torch.float32 if self.wdtype == "f32" else torch.bfloat16

    def struct(self, **tensors) -> NormCfgStruct:
        if not 1 <= len(self.rows) <= 3:
            raise ValueError("rows must have one to three dimensions")
        pad = 3 - len(self.rows)
        c = NormCfgStruct()
        c.n = (ctypes.c_int32 * 3)(*([1] * pad + [_int32("rows", n) for n in self.rows]))
        c.C, c.eps = _int32("C", self.C), _fp32("eps", self.eps)
        c.dtype, c.wdtype = _dtype_code(self.dtype), _dtype_code(self.wdtype)
        for name, t in tensors.items():
            s = [0] * pad + _row_strides(t)
            if any(s):
                # dimensions in front of the rows have one entry: any distance will do
                setattr(c, name, (ctypes.c_int64 * 3)(*[x or self.C for x in s[:pad]], *s[pad:]))
        return c


def _int32(name: str, value) -> int:
    """The value, if the C struct's field holds it (ctypes would cut it off)."""
    v = operator.index(value)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name} = {v} does not fit in 32 bits")
    return v


def _fp32(name: str, value) -> float:
    v = float(value)
    if v != 0.0 and ctypes.c_float(v).value == 0.0:
        raise ValueError(f"{name} = {v} is 0 in fp32")
    return v


def _dtype_code(name: str) -> int:
    if name not in ("f32", "bf16"):
        raise ValueError(f"dtype must be 'f32' or 'bf16', got {name!r}")
    return MITA_F32 if name == "f32" else MITA_BF16


def _row_strides(t):
    """Distances of a tensor's leading dimensions (a dimension of one entry: that
    of a contiguous tensor)."""
    out, inner = [], t.shape[-1]
    for n, s in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        out.append(inner if n == 1 else s)
        inner *= n
    out.reverse()
    if not any(out):
        raise ValueError("a tensor that repeats one row everywhere has to be made contiguous")
    return out


def _strides(t):
    s = _row_strides(t)
    if t.shape[2] > 1 and s[2] == 0:
        raise ValueError("tokens must not be repeated (stride 0 between tokens)")
    return s


def _tensor(t, name, shape, dtype, device):
    """A device tensor of this shape and type whose last dimension is dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on the GPU")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the other tensors on {device}")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return t


def _packed(t, name, shape, dtype, device):
    """The same, contiguous."""
    if not _tensor(t, name, shape, dtype, device).is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _lengths(t, name, B, device):
    return None if t is None else _packed(t, name, (B,), torch.int32, device)


class _Plan:
    """What a call needs besides addresses, for one configuration and the shapes,
    strides, types and devices of its tensors (never their addresses)."""
    __slots__ = ("cfg", "ref", "need", "device", "index", "outs")

    def __init__(self, struct, need, device, outs):
        self.cfg, self.ref, self.need, self.device, self.index = struct, ctypes.byref(struct), need, device, device.index
        self.outs = outs  # per output: (shape, strides, dtype)

    def out(self, t, i):
        return self.new(i) if t is None else t

    def new(self, i):
        shape, strides, dtype = self.outs[i]
        return torch.empty_strided(shape, strides, dtype=dtype, device=self.device)


def _like(t):
    """(shape, strides, dtype) of an output beside t: tokens before heads in
    memory where t has them so (a projection's layout), else contiguous."""
    shape = tuple(t.shape)
    if t.dim() == 4 and shape[1] > 1 and shape[2] > 1 and t.stride(1) < t.stride(2):
        B, H, N, d = shape
        return shape, (N * H * d, d, H * d, 1), t.dtype
    return _dense(shape, t.dtype)


def _dense(shape, dtype):
    strides, n = [], 1
    for x in reversed(shape):
        strides.append(n)
        n *= x
    return tuple(shape), tuple(reversed(strides)), dtype


def _place(given, like):
    """A stand-in with the strides of an output: the given tensor or the one to come."""
    return given if given is not None else torch.empty_strided(*like[:2], dtype=like[2], device="meta")


def _signature(ts):
    return tuple([None if t is None else (t.shape, t.stride(), t.dtype, t.device) for t in ts])


def _plan_for(cfg, kind, ts, make):
    """The call's plan: looked up by the tensors' signature, checked and made the
    first time."""
    plans = cfg.__dict__.get("_plans")
    if plans is None:
        plans = cfg.__dict__["_plans"] = {}
    try:
        key = (kind, _signature(ts))
        plan = plans.get(key)
    except AttributeError:
        plan = key = None  # not a tensor: make() says so
    if plan is None:
        plan = make(cfg, *ts)
        if len(plans) >= 1024:
            plans.clear()
        plans[key] = plan
    return plan


_NOW = contextlib.nullcontext()


def _on(plan, stream):
    """A call's own allocations belong to the stream it is given."""
    if stream.device != plan.device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {plan.device}")
    return torch.cuda.stream(stream)


def _ws_for(plan, ws):
    if ws is None:
        if not plan.need:
            return None, None, 0
        ws = torch.empty(plan.need, dtype=torch.uint8, device=plan.device)
    elif ws.device != plan.device or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous tensor on the tensors' device")
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def _call(plan, fn, args, stream):
    """fn(cfg, *args, stream) with the tensors' device current."""
    raw = torch._C._cuda_getCurrentRawStream(plan.index) if stream is None else stream.cuda_stream
    if torch.cuda.current_device() == plan.index:
        st = fn(plan.ref, *args, raw)
    else:
        with torch.cuda.device(plan.index):
            st = fn(plan.ref, *args, raw)
    if st != MITA_OK:
        _check(st)


def _ptr(t):
    return None if t is None else t.data_ptr()


def dense_check(cfg: DenseConfig) -> int:
    return load_library().mita_dense_check(ctypes.byref(cfg.struct()))


def dense_workspace_size(cfg: DenseConfig, which: int = WS_FORWARD) -> int:
    return int(load_library().mita_dense_workspace_size(ctypes.byref(cfg.struct()), which))


def _dense_forward_plan(cfg, q, k, v, q_len, k_len, o, lse):
    _tensor(q, "q", cfg.q_shape, cfg.torch_dtype, None)
    dev = q.device
    _tensor(k, "k", cfg.k_shape, cfg.torch_dtype, dev)
    _tensor(v, "v", cfg.k_shape, cfg.torch_dtype, dev)
    _lengths(q_len, "q_len", cfg.B, dev)
    _lengths(k_len, "k_len", cfg.B, dev)
    if o is not None:
        _tensor(o, "o", cfg.q_shape, cfg.torch_dtype, dev)
    if lse is not None:
        _packed(lse, "lse", cfg.q_shape[:3], torch.float32, dev)
    outs = (_like(q), _dense(cfg.q_shape[:3], torch.float32))
    c = cfg.struct(q=q, k=k, v=v, o=_place(o, outs[0]))
    return _Plan(c, int(load_library().mita_dense_workspace_size(ctypes.byref(c), WS_FORWARD)), dev, outs)


def dense_forward(cfg: DenseConfig, q, k, v, q_len=None, k_len=None, o=None, lse=None, want_lse=True, ws=None,
                  stream=None):
    """Dense attention (mita_dense_forward): (o [B, H, N, d], lse [B, H, N] fp32
    or None). q, k, v may be strided (their last dimension dense); q_len, k_len
    are [B] int32 device tensors."""
    lib = load_library()
    plan = _plan_for(cfg, "forward", (q, k, v, q_len, k_len, o, lse), _dense_forward_plan)
    with _NOW if stream is None else _on(plan, stream):
        o = plan.out(o, 0)
        if lse is None and want_lse:
            lse = plan.new(1)
        ws, wp, wn = _ws_for(plan, ws)
    _call(plan, lib.mita_dense_forward, (q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(q_len), _ptr(k_len),
                                         o.data_ptr(), _ptr(lse), wp, wn), stream)
    return o, lse


def _dense_backward_plan(cfg, q, k, v, o, lse, dO, q_len, k_len, dq, dk, dv):
    _tensor(q, "q", cfg.q_shape, cfg.torch_dtype, None)
    dev, dt = q.device, cfg.torch_dtype
    for t, name, shape in ((k, "k", cfg.k_shape), (v, "v", cfg.k_shape), (o, "o", cfg.q_shape),
                           (dO, "dO", cfg.q_shape)):
        _tensor(t, name, shape, dt, dev)
    _packed(lse, "lse", cfg.q_shape[:3], torch.float32, dev)
    _lengths(q_len, "q_len", cfg.B, dev)
    _lengths(k_len, "k_len", cfg.B, dev)
    for t, name, shape in ((dq, "dq", cfg.q_shape), (dk, "dk", cfg.k_shape), (dv, "dv", cfg.k_shape)):
        if t is not None:
            _tensor(t, name, shape, dt, dev)
    outs = (_like(q), _like(k), _like(v))
    c = cfg.struct(q=q, k=k, v=v, o=o, dO=dO, dq=_place(dq, outs[0]), dk=_place(dk, outs[1]), dv=_place(dv, outs[2]))
    return _Plan(c, int(load_library().mita_dense_workspace_size(ctypes.byref(c), WS_BACKWARD)), dev, outs)


def dense_backward(cfg: DenseConfig, q, k, v, o, lse, dO, q_len=None, k_len=None, dq=None, dk=None, dv=None, ws=None,
                   stream=None):
    """Gradients (dq, dk, dv) of dense_forward's o for the upstream gradient dO
    (mita_dense_backward)."""
    lib = load_library()
    plan = _plan_for(cfg, "backward", (q, k, v, o, lse, dO, q_len, k_len, dq, dk, dv), _dense_backward_plan)
    with _NOW if stream is None else _on(plan, stream):
        dq, dk, dv = plan.out(dq, 0), plan.out(dk, 1), plan.out(dv, 2)
        ws, wp, wn = _ws_for(plan, ws)
    _call(plan, lib.mita_dense_backward, (q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                          dO.data_ptr(), _ptr(q_len), _ptr(k_len), dq.data_ptr(), dk.data_ptr(),
                                          dv.data_ptr(), wp, wn), stream)
    return dq, dk, dv


def norm_check(cfg: NormConfig) -> int:
    return load_library().mita_norm_check(ctypes.byref(cfg.struct()))


def norm_workspace_size(cfg: NormConfig) -> int:
    """Bytes of workspace norm_backward needs for the weight's gradients."""
    return int(load_library().mita_norm_workspace_size(ctypes.byref(cfg.struct())))


def _norm_forward_plan(cfg, x, w, b, y, mean, rstd):
    dt, wt = cfg.torch_dtype, cfg.torch_wdtype
    _tensor(x, "x", cfg.shape, dt, None)
    dev = x.device
    for t, name in ((w, "w"), (b, "b")):
        if t is not None:
            _packed(t, name, (cfg.C,), wt, dev)
    if y is not None:
        _tensor(y, "y", cfg.shape, dt, dev)
    for t, name in ((mean, "mean"), (rstd, "rstd")):
        if t is not None:
            _packed(t, name, cfg.rows, torch.float32, dev)
    outs = (_like(x), _dense(cfg.rows, torch.float32))
    return _Plan(cfg.struct(x=x, y=_place(y, outs[0])), 0, dev, outs)


def norm_forward(cfg: NormConfig, x, w=None, b=None, y=None, mean=None, rstd=None, want_stats=True, stream=None):
    """Layer norm (mita_norm_forward): (y like x, mean and rstd [rows] fp32 or
    None). x may be strided (its last dimension dense)."""
    lib = load_library()
    plan = _plan_for(cfg, "forward", (x, w, b, y, mean, rstd), _norm_forward_plan)
    with _NOW if stream is None else _on(plan, stream):
        y = plan.out(y, 0)
        if want_stats:
            mean, rstd = plan.out(mean, 1), plan.out(rstd, 1)
    _call(plan, lib.mita_norm_forward, (x.data_ptr(), _ptr(w), _ptr(b), y.data_ptr(), _ptr(mean), _ptr(rstd)), stream)
    return y, mean, rstd


def _norm_backward_plan(cfg, x, mean, rstd, dy, w, dx, dw, db):
    dt, wt = cfg.torch_dtype, cfg.torch_wdtype
    _tensor(x, "x", cfg.shape, dt, None)
    dev = x.device
    _tensor(dy, "dy", cfg.shape, dt, dev)
    _packed(mean, "mean", cfg.rows, torch.float32, dev)
    _packed(rstd, "rstd", cfg.rows, torch.float32, dev)
    if dx is not None:
        _tensor(dx, "dx", cfg.shape, dt, dev)
    for t, name in ((w, "w"), (dw, "dw"), (db, "db")):
        if t is not None:
            _packed(t, name, (cfg.C,), wt, dev)
    outs = (_like(x), _dense((cfg.C,), wt))
    c = cfg.struct(x=x, dy=dy, dx=_place(dx, outs[0]))
    return _Plan(c, int(load_library().mita_norm_workspace_size(ctypes.byref(c))), dev, outs)


def norm_backward(cfg: NormConfig, x, mean, rstd, dy, w=None, dx=None, dw=None, db=None, want_dx=True,
                  want_weights=True, ws=None, stream=None):
    """Gradients (dx, dw, db) of norm_forward (mita_norm_backward); dx, or dw and
    db, are None unless wanted."""
    lib = load_library()
    plan = _plan_for(cfg, "backward", (x, mean, rstd, dy, w, dx, dw, db), _norm_backward_plan)
    with _NOW if stream is None else _on(plan, stream):
        if want_dx:
            dx = plan.out(dx, 0)
        if want_weights:
            dw, db = plan.out(dw, 1), plan.out(db, 1)
        ws, wp, wn = _ws_for(plan, ws) if dw is not None or db is not None else (None, None, 0)
    _call(plan, lib.mita_norm_backward, (x.data_ptr(), _ptr(w), mean.data_ptr(), rstd.data_ptr(), dy.data_ptr(),
                                         _ptr(dx), _ptr(dw), _ptr(db), wp, wn), stream)
    return dx, dw, db


class Timer:
    """HIP-event stage timer for mita_forward_timed."""

    def __init__(self, max_calls: int):
        self.lib = load_library()
        h = ctypes.c_void_p()
        _check(self.lib.mita_timer_create(ctypes.byref(h), int(max_calls)))
        self.handle = h
        self.max_calls = max_calls

    def reset(self):
        _check(self.lib.mita_timer_reset(self.handle))

    def launches(self):
        """Waits for the events; returns a list (one per call) of
        (kernel name, stage index, ms) tuples, one per kernel launched."""
        out = []
        n_calls = len(self.read())
        for c in range(n_calls):
            names = (ctypes.c_char_p * MAX_LAUNCHES)()
            stages = (ctypes.c_int32 * MAX_LAUNCHES)()
            ms = (ctypes.c_float * MAX_LAUNCHES)()
            n = ctypes.c_int32()
            _check(self.lib.mita_timer_launches(self.handle, c, MAX_LAUNCHES, names, stages, ms, ctypes.byref(n)))
            out.append([(names[i].decode(), stages[i], ms[i]) for i in range(n.value)])
        return out

    def read(self):
        """Waits for the events; returns a list (one per call) of per-stage ms
        lists (each stage the sum of its launches' times)."""
        n = ctypes.c_int()
        buf = (ctypes.c_float * (self.max_calls * NUM_STAGES))()
        _check(self.lib.mita_timer_read(self.handle, buf, len(buf), ctypes.byref(n)))
        return [[buf[c * NUM_STAGES + s] for s in range(NUM_STAGES)] for c in range(n.value)]

    def close(self):
        if self.handle:
            self.lib.mita_timer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

"""Thin Python binding of libecokv.so (argument marshalling only).

Every step of the eviction pass runs in the HIP kernels behind the C ABI
declared in ``include/ecokv.h``; this module turns torch tensors into device
pointers, the current HIP stream into a handle, and error codes into
exceptions.  PyTorch provides device memory and streams only.  If the built
library is missing, importing this module raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Sequence

import torch

# ECOKV_LIBRARY names another build of the library to load instead of the
# in-tree one (for instance one whose host code is built with sanitizers).
_LIB_PATH = os.environ.get("ECOKV_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libecokv.so")

OK, EINVAL, EWORKSPACE, EUNSUPPORTED, EHIP, ETIMEOUT = 0, -1, -2, -3, -4, -5
BF16, F32 = 0, 1
PER_HEAD, LAYER_FLAT, HEAD_BUDGETS = 0, 1, 2
IMP_ATTN, IMP_ATTN_VNORM = 0, 1
NORM_MINMAX, NORM_WINSOR, NORM_MAD = 0, 1, 2
RED_EUCLID, RED_STD = 0, 1
CENTROID_ALL, CENTROID_PREFIX = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = 0, 1, 2, 3
MAX_SEQS, MAX_ROWS = 64, 64
NSTATS = 12
STAT = dict(lambda_=0, rC=1, rE=2, DE=3, dmin=4, dmax=5, sdmin=6, sdmax=7, imp_mean=8, sbar_mean=9,
            mu_norm2=10, scale=11)

EXPORTS = ["ecokv_default_params", "ecokv_workspace_size", "ecokv_workspace_status", "ecokv_score", "ecokv_score_v",
           "ecokv_score_pre", "ecokv_score_noalloc", "ecokv_prefill_workspace_size", "ecokv_prefill_write",
           "ecokv_index_count",
           "ecokv_index_count_mode", "ecokv_select_workspace_size", "ecokv_select", "ecokv_compact",
           "ecokv_pyramid_budgets",
           "ecokv_decode_workspace_size", "ecokv_decode",
           "ecokv_rope_freqs", "ecokv_prefill_rope", "ecokv_append", "ecokv_decode_shared_workspace_size",
           "ecokv_decode_shared",
           "ecokv_last_error", "ecokv_stage_times"]


class _StageTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("ms", ctypes.c_double), ("launches", ctypes.c_int64)]


class EcoKVError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libecokv error {code}: {msg}")
        self.code = code


class _Shape(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("window", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
                ("cu_seqlens", ctypes.POINTER(ctypes.c_int32))]


class Params(ctypes.Structure):
    """ecokv_params; defaults are the paper's (Table 6)."""
    _fields_ = [("alpha", ctypes.c_float), ("beta", ctypes.c_float), ("eps", ctypes.c_float),
                ("tau", ctypes.c_float), ("pool_kernel", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("lambda_override", ctypes.c_float), ("imp_mode", ctypes.c_int32),
                ("norm_mode", ctypes.c_int32), ("winsor_q", ctypes.c_float), ("mad_tau", ctypes.c_float),
                ("redundancy", ctypes.c_int32), ("centroid_scope", ctypes.c_int32)]

    def __init__(self, alpha=0.8, beta=0.6, eps=1e-6, tau=0.0, pool_kernel=5, causal=True,
                 lambda_override=math.nan, imp_mode=IMP_ATTN, norm_mode=NORM_MINMAX, winsor_q=0.01,
                 mad_tau=1.0, redundancy=RED_EUCLID, centroid_scope=CENTROID_ALL):
        super().__init__(alpha, beta, eps, tau, int(pool_kernel), int(bool(causal)), lambda_override,
                         int(imp_mode), int(norm_mode), winsor_q, mad_tau, int(redundancy), int(centroid_scope))


class Shape:
    """ecokv_shape plus the host array of sequence offsets it points to."""

    def __init__(self, num_layers: int, num_q_heads: int, num_kv_heads: int, head_dim: int, window: int,
                 cu_seqlens: Sequence[int]):
        self.cu = (ctypes.c_int32 * len(cu_seqlens))(*[int(x) for x in cu_seqlens])
        self.c = _Shape(num_layers, num_q_heads, num_kv_heads, head_dim, window, len(cu_seqlens) - 1,
                        ctypes.cast(self.cu, ctypes.POINTER(ctypes.c_int32)))

    @property
    def cu_seqlens(self):
        return list(self.cu)

    # element counts of the tensors of a call, for the binding's checks
    @property
    def units(self) -> int:
        c = self.c
        return c.num_layers * c.num_kv_heads * c.num_seqs

    @property
    def ttot(self) -> int:
        return int(self.cu[self.c.num_seqs])

    @property
    def ptot(self) -> int:
        return self.ttot - self.c.num_seqs * self.c.window

    def kv_numel(self) -> int:
        c = self.c
        return c.num_layers * c.num_kv_heads * self.ttot * c.head_dim

    def q_numel(self) -> int:
        c = self.c
        return c.num_layers * c.num_q_heads * c.num_seqs * c.window * c.head_dim

    def score_numel(self) -> int:
        return self.c.num_layers * self.c.num_kv_heads * self.ptot


class _Rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("freq", ctypes.c_void_p),
                ("factor", ctypes.c_float), ("norm_eps", ctypes.c_float), ("q_norm", ctypes.c_void_p),
                ("k_norm", ctypes.c_void_p)]


def _int32(v, name: str) -> int:
    """v, which ctypes would cut to 32 bits without a word."""
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name} {v} does not fit 32 bits")
    return v


def _held(name: str):
    """A handle's tensor.  The structure keeps its pointer from call to call, so
    putting another in its place has the next call check that one and take its
    pointer and sizes."""
    def put(self, t):
        self.__dict__[name] = t
        self._for = None
    return property(lambda self: self.__dict__[name], put)


class Rope:
    """ecokv_rope: rotary positions (`freq` float32 [rot_dim / 2], see
    ecokv_rope_freqs) and, where `q_norm` / `k_norm` [D] weights are given, the
    per-head norms before them.  Holds the tensors that it points to: other
    tensors may be assigned, and a tensor's values may change, but not its
    storage."""

    freq, q_norm, k_norm = _held("freq"), _held("q_norm"), _held("k_norm")

    def __init__(self, rot_dim: int, freq: Optional[torch.Tensor] = None, interleaved: bool = False, factor: float = 1.0,
                 q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None, norm_eps: float = 1e-6):
        self.freq, self.q_norm, self.k_norm = freq, q_norm, k_norm
        self.c = _Rope(_int32(rot_dim, "rot_dim"), int(bool(interleaved)), None, factor, norm_eps, None, None)

    def _arg(self, head_dim: int, dtype, device):
        """Pointer to the structure, checked for rows of this size, element type and
        device when these differ from the last call's or a tensor was replaced."""
        if self._for != (head_dim, dtype, device):
            self._for = None
            self.c.freq = _arg(self.freq, "freq", _F32, max(self.c.rot_dim, 0) // 2, device, optional=self.c.rot_dim <= 0)
            self.c.q_norm = _arg(self.q_norm, "q_norm", (dtype,), head_dim, device, optional=True)
            self.c.k_norm = _arg(self.k_norm, "k_norm", (dtype,), head_dim, device, optional=True)
            self._for = head_dim, dtype, device
        return ctypes.byref(self.c)


class _Tails(ctypes.Structure):
    _fields_ = [("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("num_conts", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("max_pages", ctypes.c_int32)]


class Tails:
    """ecokv_tails: K, V [L][num_pages][H_kv][page_size][D] and table (int32)
    [num_conts][max_pages].  Holds the tensors that it points to: others may be
    assigned (a larger table or pool), and a tensor's values may change, but not
    its storage."""

    K, V, table = _held("K"), _held("V"), _held("table")

    def __init__(self, K: torch.Tensor, V: torch.Tensor, table: torch.Tensor):
        self.K, self.V, self.table = K, V, table
        self.c = _Tails()
        self._sizes()

    def _sizes(self):
        """The structure's sizes, those of the tensors."""
        K, V, table = self.K, self.V, self.table
        if K.dim() != 5 or V.shape != K.shape or V.dtype != K.dtype:
            raise ValueError("the tails' K and V are two tensors [L][num_pages][H_kv][page_size][D] of one element type")
        if table.dim() != 2:
            raise ValueError("the tails' table is [num_conts][max_pages]")
        c = self.c
        c.num_conts, c.num_pages, c.page_size, c.max_pages = table.shape[0], K.shape[1], K.shape[3], table.shape[1]

    def _arg(self, shape: "Shape", dtype, device):
        """Pointer to the structure, checked for calls of this shape, element type
        and device when these differ from the last call's or a tensor was replaced."""
        c = shape.c
        now = c.num_layers, c.num_kv_heads, c.head_dim, dtype, device
        if self._for != now:
            self._for = None
            self._sizes()
            L, _, H, _, D = self.K.shape
            if (L, H, D) != now[:3]:
                raise ValueError(f"the tails have {L} layers of {H} KV heads of {D} dimensions, the shape "
                                 f"{c.num_layers} of {c.num_kv_heads} of {c.head_dim}")
            self.c.K = _arg(self.K, "the tails' K", (dtype,), self.K.numel(), device)
            self.c.V = _arg(self.V, "the tails' V", (dtype,), self.K.numel(), device)
            self.c.table = _arg(self.table, "the tails' table", _I32, self.table.numel(), device)
            self._for = now
        return ctypes.byref(self.c)


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is not built; run `python paper_2609_06663_amd/build.py`")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, sp, pp = ctypes.c_void_p, ctypes.POINTER(_Shape), ctypes.POINTER(Params)
    i32p = ctypes.POINTER(ctypes.c_int32)
    lib.ecokv_default_params.argtypes = [pp]
    lib.ecokv_workspace_size.argtypes = [sp, pp, ctypes.POINTER(ctypes.c_size_t)]
    lib.ecokv_workspace_status.argtypes = [vp, vp]
    lib.ecokv_score.argtypes = [vp, vp, ctypes.c_int, sp, pp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ecokv_score_v.argtypes = [vp, vp, vp, ctypes.c_int, sp, pp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ecokv_score_pre.argtypes = [vp, vp, vp, ctypes.c_int, sp, pp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ecokv_score_noalloc.argtypes = [vp, vp, vp, ctypes.c_int, sp, pp, vp, vp, vp, vp, vp]
    lib.ecokv_prefill_workspace_size.argtypes = [sp, ctypes.POINTER(ctypes.c_size_t)]
    lib.ecokv_prefill_write.argtypes = [vp, vp, vp, ctypes.c_int, sp, pp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ecokv_index_count.argtypes = [sp, i32p, ctypes.POINTER(ctypes.c_int64)]
    lib.ecokv_index_count_mode.argtypes = [sp, ctypes.c_int, i32p, ctypes.POINTER(ctypes.c_int64)]
    lib.ecokv_decode_workspace_size.argtypes = [sp, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)]
    lib.ecokv_decode.argtypes = [vp, vp, vp, ctypes.c_int, sp, vp, vp, ctypes.c_int32, vp, vp, vp,
                                 ctypes.c_size_t, vp]
    rp, tp, i64 = ctypes.POINTER(_Rope), ctypes.POINTER(_Tails), ctypes.c_int64
    f32p = ctypes.POINTER(ctypes.c_float)
    lib.ecokv_rope_freqs.argtypes = [ctypes.c_int, ctypes.c_double, ctypes.c_int, ctypes.c_double, ctypes.c_double,
                                     f32p, f32p]
    lib.ecokv_prefill_rope.argtypes = [vp, i64, vp, i64, ctypes.c_int, sp, rp, vp, vp, vp, vp, vp]
    lib.ecokv_append.argtypes = [vp, i64, vp, i64, vp, i64, ctypes.c_int, sp, rp, vp, vp, vp, ctypes.c_int32, tp, vp, vp]
    lib.ecokv_decode_shared_workspace_size.argtypes = [sp, i32p, ctypes.c_int32, ctypes.c_int32,
                                                       ctypes.POINTER(ctypes.c_size_t)]
    lib.ecokv_decode_shared.argtypes = [vp, vp, vp, ctypes.c_int, sp, i32p, vp, vp, ctypes.c_int32, tp, vp,
                                        ctypes.c_int32, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ecokv_pyramid_budgets.argtypes = [ctypes.c_int, ctypes.c_double, ctypes.c_double, ctypes.c_int, i32p]
    lib.ecokv_select_workspace_size.argtypes = [sp, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)]
    lib.ecokv_select.argtypes = [vp, sp, ctypes.c_int, i32p, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.ecokv_compact.argtypes = [vp, vp, ctypes.c_int, sp, ctypes.c_int, i32p, vp, vp, vp, vp, vp, vp]
    lib.ecokv_last_error.restype = ctypes.c_char_p
    lib.ecokv_stage_times.argtypes = [ctypes.POINTER(_StageTime), ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    for name in EXPORTS:
        if name != "ecokv_last_error":
            getattr(lib, name).restype = ctypes.c_int
    return lib


lib = _load()


def _check(rc: int):
    if rc != OK:
        raise EcoKVError(rc, lib.ecokv_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libecokv must be contiguous")
    return t.data_ptr()


_ELEM = {torch.bfloat16: "bf16", torch.float32: "float32", torch.int32: "int32", torch.uint8: "uint8"}


def _arg(t: Optional[torch.Tensor], name: str, dtypes, numel: int, device, optional: bool = False):
    """Device pointer of `t` after checking that it is a contiguous tensor on
    `device` with an allowed element type and at least `numel` elements: the
    kernels trust these sizes, so a mismatch is refused here rather than read
    or written out of bounds on the GPU."""
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    # (one test for a call in order; what is wrong with another is told apart below)
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in dtypes and t.numel() >= numel and t.is_contiguous()
            and (device is None or t.device == device)):
        return t.data_ptr()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the call's tensors on {device}")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(_ELEM.get(d, str(d)) for d in dtypes)} (got {t.dtype})")
    if t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, the call needs {numel}")
    return _ptr(t)


_KV_TYPES = (torch.bfloat16, torch.float32)
_F32 = (torch.float32,)
_I32 = (torch.int32,)
_U8 = (torch.uint8,)


def _workspace(workspace: Optional[torch.Tensor], nbytes: int, device, stream):
    """The caller's workspace, or a zero-filled one allocated here, on `stream`
    where one is given: its memory's last use, the filling and torch's next use
    are then all in order with the call."""
    if workspace is not None:
        return workspace
    with torch.cuda.stream(stream):  # (None: the current stream stays)
        return torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=device)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported element type {t.dtype} (bf16 or fp32)")


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if torch.cuda.is_initialized():
        # the current stream's handle alone: the Stream object of
        # torch.cuda.current_stream() costs a quarter of a short call's host work
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _flat_ints(x) -> list:
    if hasattr(x, "reshape"):  # numpy array or tensor
        x = x.reshape(-1).tolist()
    if isinstance(x, (list, tuple)) and all(type(v) is int for v in x):
        return list(x)
    out = []
    for v in x:
        if isinstance(v, (list, tuple)):
            out.extend(_flat_ints(v))
        else:
            out.append(int(v))
    return out


def _budget(shape: Shape, budget, mode: int = PER_HEAD):
    """Host budget array: one per sequence, or [L][H_kv] for HEAD_BUDGETS."""
    vals = _flat_ints(budget)
    c = shape.c
    n = c.num_layers * c.num_kv_heads if mode == HEAD_BUDGETS else c.num_seqs
    if len(vals) != n:
        raise ValueError("HEAD_BUDGETS takes one budget per (layer, KV head)" if mode == HEAD_BUDGETS
                         else "one budget per sequence")
    return (ctypes.c_int32 * max(n, 1))(*vals)


def ecokv_default_params() -> Params:
    p = Params()
    _check(lib.ecokv_default_params(ctypes.byref(p)))
    return p


def ecokv_workspace_size(shape: Shape, params: Optional[Params] = None) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.ecokv_workspace_size(ctypes.byref(shape.c), ctypes.byref(params or Params()), ctypes.byref(n)))
    return n.value


def _score_args(K, V, Q_win, shape: Shape, p: Params, scores, lambda_, stats, workspace, stream, pre=None):
    """Checked pointers of a score call, in the order of ecokv_score_pre."""
    L = shape.c.num_layers
    if L == 0:  # nothing is read or written
        return [_ptr(K), _ptr(V), _ptr(Q_win), _dtype_code(K) if K is not None else BF16, ctypes.byref(shape.c),
                ctypes.byref(p), _ptr(pre), _ptr(scores), _ptr(lambda_), _ptr(stats), _ptr(workspace),
                0 if workspace is None else workspace.numel(), _stream(stream)]
    dev = K.device if isinstance(K, torch.Tensor) else None
    kp = _arg(K, "K", _KV_TYPES, shape.kv_numel(), dev)
    if Q_win.dtype != K.dtype or (V is not None and V.dtype != K.dtype):
        raise TypeError("K, V and Q_win must have the same element type")
    vp = _arg(V, "V", _KV_TYPES, shape.kv_numel(), dev, optional=p.imp_mode != IMP_ATTN_VNORM)
    qp = _arg(Q_win, "Q_win", _KV_TYPES, shape.q_numel(), dev)
    R = shape.c.num_q_heads // shape.c.num_kv_heads * shape.c.window
    pp = _arg(pre, "pre", _F32, shape.units * (2 * shape.c.head_dim + 2 * R), dev, optional=True)
    sp_ = _arg(scores, "scores", _F32, shape.score_numel(), dev)
    lp = _arg(lambda_, "lambda", _F32, shape.units, dev, optional=True)
    stp = _arg(stats, "stats", _F32, shape.units * NSTATS, dev, optional=True)
    need = ecokv_workspace_size(shape, p)
    workspace = _workspace(workspace, need, dev, stream)
    wp = _arg(workspace, "workspace", _U8, need, dev)
    return [kp, vp, qp, _dtype_code(K), ctypes.byref(shape.c), ctypes.byref(p), pp, sp_, lp, stp, wp,
            workspace.numel(), _stream(stream)]


def ecokv_score(K: torch.Tensor, Q_win: torch.Tensor, shape: Shape, params: Optional[Params],
                scores: torch.Tensor, lambda_: Optional[torch.Tensor] = None,
                stats: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream=None) -> None:
    """Enqueue ecokv_score.  `workspace` (uint8, >= ecokv_workspace_size bytes,
    zero-filled before its first use) is allocated here when not given."""
    p = params or Params()
    a = _score_args(K, None, Q_win, shape, p, scores, lambda_, stats, workspace, stream)
    del a[1], a[5]  # no V, no pre
    _check(lib.ecokv_score(*a))


def ecokv_score_v(K: torch.Tensor, V: Optional[torch.Tensor], Q_win: torch.Tensor, shape: Shape,
                  params: Optional[Params], scores: torch.Tensor, lambda_: Optional[torch.Tensor] = None,
                  stats: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream=None) -> None:
    """Enqueue ecokv_score_v (V is read with imp_mode IMP_ATTN_VNORM)."""
    p = params or Params()
    a = _score_args(K, V, Q_win, shape, p, scores, lambda_, stats, workspace, stream)
    del a[6]  # no pre
    _check(lib.ecokv_score_v(*a))


def ecokv_score_pre(K: torch.Tensor, V: Optional[torch.Tensor], Q_win: torch.Tensor, shape: Shape,
                    params: Optional[Params], pre: torch.Tensor, scores: torch.Tensor,
                    lambda_: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ecokv_score_pre: `pre` (float32 [L][Hkv][B][2D + 2R]) holds the
    key sums and window softmax statistics a prefill produced."""
    p = params or Params()
    if pre is not None and pre.dtype != torch.float32:
        raise TypeError("pre is float32")
    a = _score_args(K, V, Q_win, shape, p, scores, lambda_, stats, workspace, stream, pre=pre)
    _check(lib.ecokv_score_pre(*a))


def ecokv_prefill_workspace_size(shape: Shape) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.ecokv_prefill_workspace_size(ctypes.byref(shape.c), ctypes.byref(n)))
    return n.value


def ecokv_prefill_write(K_new: torch.Tensor, V_new: Optional[torch.Tensor], Q_win: torch.Tensor, shape: Shape,
                        params: Optional[Params], K_cache: torch.Tensor, V_cache: Optional[torch.Tensor],
                        pre: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ecokv_prefill_write: K_new / V_new token-major ([L][T_total][Hkv][D])
    into K_cache / V_cache (the pass's [L][Hkv][T_total][D]), and `pre` (float32
    [L][Hkv][B][2D + 2R]) for ecokv_score_pre.  V_new and V_cache: both or neither."""
    p = params or Params()
    if shape.c.num_layers == 0:
        return
    if (V_new is None) != (V_cache is None):
        raise ValueError("V_new and V_cache: both or neither")
    dev = K_new.device
    kn = _arg(K_new, "K_new", _KV_TYPES, shape.kv_numel(), dev)
    for t, n in ((Q_win, "Q_win"), (K_cache, "K_cache"), (V_new, "V_new"), (V_cache, "V_cache")):
        if t is not None and t.dtype != K_new.dtype:
            raise TypeError(f"{n} must have the element type of K_new")
    vn = _arg(V_new, "V_new", _KV_TYPES, shape.kv_numel(), dev, optional=True)
    qp = _arg(Q_win, "Q_win", _KV_TYPES, shape.q_numel(), dev)
    kc = _arg(K_cache, "K_cache", _KV_TYPES, shape.kv_numel(), dev)
    vc = _arg(V_cache, "V_cache", _KV_TYPES, shape.kv_numel(), dev, optional=True)
    R = shape.c.num_q_heads // shape.c.num_kv_heads * shape.c.window
    pp = _arg(pre, "pre", _F32, shape.units * (2 * shape.c.head_dim + 2 * R), dev)
    need = ecokv_prefill_workspace_size(shape)
    workspace = _workspace(workspace, need, dev, stream)
    wp = _arg(workspace, "workspace", _U8, need, dev)
    _check(lib.ecokv_prefill_write(kn, vn, qp, _dtype_code(K_new), ctypes.byref(shape.c), ctypes.byref(p), kc, vc, pp,
                                   wp, workspace.numel(), _stream(stream)))


def ecokv_score_noalloc(K: torch.Tensor, V: Optional[torch.Tensor], Q_win: torch.Tensor, shape: Shape,
                        params: Optional[Params], pre: Optional[torch.Tensor], scores: torch.Tensor,
                        lambda_: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """Enqueue ecokv_score_noalloc: ecokv_score_pre (pre may be None) with the
    library's own per-device scratch; nothing is allocated here either."""
    p = params or Params()
    if pre is not None and pre.dtype != torch.float32:
        raise TypeError("pre is float32")
    if shape.c.num_layers == 0:
        return
    dev = K.device
    kp = _arg(K, "K", _KV_TYPES, shape.kv_numel(), dev)
    if Q_win.dtype != K.dtype or (V is not None and V.dtype != K.dtype):
        raise TypeError("K, V and Q_win must have the same element type")
    vp = _arg(V, "V", _KV_TYPES, shape.kv_numel(), dev, optional=p.imp_mode != IMP_ATTN_VNORM)
    qp = _arg(Q_win, "Q_win", _KV_TYPES, shape.q_numel(), dev)
    R = shape.c.num_q_heads // shape.c.num_kv_heads * shape.c.window
    prp = _arg(pre, "pre", _F32, shape.units * (2 * shape.c.head_dim + 2 * R), dev, optional=True)
    _check(lib.ecokv_score_noalloc(kp, vp, qp, _dtype_code(K), ctypes.byref(shape.c), ctypes.byref(p), prp,
                                   _arg(scores, "scores", _F32, shape.score_numel(), dev),
                                   _arg(lambda_, "lambda", _F32, shape.units, dev, optional=True),
                                   _arg(stats, "stats", _F32, shape.units * NSTATS, dev, optional=True),
                                   _stream(stream)))


def ecokv_workspace_status(workspace: torch.Tensor, stream=None) -> None:
    """Synchronise `stream` and raise EcoKVError (code ETIMEOUT) if a score call
    on `workspace` since the last query had a wait between blocks give up (its
    lambda and scores of the affected units are then NaN); clears the record."""
    _check(lib.ecokv_workspace_status(_arg(workspace, "workspace", _U8, 4, None), _stream(stream)))


def ecokv_index_count(shape: Shape, budget: Sequence[int]) -> int:
    n = ctypes.c_int64(0)
    _check(lib.ecokv_index_count(ctypes.byref(shape.c), _budget(shape, budget), ctypes.byref(n)))
    return n.value


def ecokv_index_count_mode(shape: Shape, mode: int, budget) -> int:
    return _index_count(shape, mode, _budget(shape, budget, mode))


def _index_count(shape: Shape, mode: int, bud) -> int:
    n = ctypes.c_int64(0)
    _check(lib.ecokv_index_count_mode(ctypes.byref(shape.c), int(mode), bud, ctypes.byref(n)))
    return n.value


def ecokv_pyramid_budgets(num_layers: int, total: float, beta: float, window: int) -> list:
    out = (ctypes.c_int32 * max(int(num_layers), 1))()
    _check(lib.ecokv_pyramid_budgets(int(num_layers), float(total), float(beta), int(window), out))
    return [int(v) for v in out[:num_layers]]


def ecokv_select_workspace_size(shape: Shape, mode: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.ecokv_select_workspace_size(ctypes.byref(shape.c), int(mode), ctypes.byref(n)))
    return n.value


def ecokv_select(scores: torch.Tensor, shape: Shape, mode: int, budget, idx: torch.Tensor,
                 counts: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ecokv_select.  `workspace` (uint8, >= ecokv_select_workspace_size
    bytes, zero-filled before its first use) is allocated here when not given."""
    bud = _budget(shape, budget, mode)
    if shape.c.num_layers == 0:
        _check(lib.ecokv_select(_ptr(scores), ctypes.byref(shape.c), int(mode), bud, _ptr(idx), _ptr(counts),
                                _ptr(offsets), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                                _stream(stream)))
        return
    n = _index_count(shape, mode, bud)
    dev = scores.device if isinstance(scores, torch.Tensor) else None
    flat = int(mode) == LAYER_FLAT
    sp_ = _arg(scores, "scores", _F32, shape.score_numel(), dev)
    ip = _arg(idx, "idx", _I32, n, dev)
    cp = _arg(counts, "counts", _I32, shape.units, dev, optional=not flat)
    op = _arg(offsets, "offsets", _I32, shape.units, dev, optional=not flat)
    need = ecokv_select_workspace_size(shape, mode)
    workspace = _workspace(workspace, need, dev, stream)
    _check(lib.ecokv_select(sp_, ctypes.byref(shape.c), int(mode), bud, ip, cp, op,
                            _arg(workspace, "workspace", _U8, need, dev), workspace.numel(), _stream(stream)))


def ecokv_compact(K: torch.Tensor, V: torch.Tensor, shape: Shape, mode: int, budget,
                  idx: torch.Tensor, counts: Optional[torch.Tensor], offsets: Optional[torch.Tensor],
                  Kc: torch.Tensor, Vc: torch.Tensor, stream=None) -> None:
    if V.dtype != K.dtype or Kc.dtype != K.dtype or Vc.dtype != K.dtype:
        raise TypeError("K, V, Kc and Vc must share one element type")
    bud = _budget(shape, budget, mode)
    if shape.c.num_layers == 0:
        _check(lib.ecokv_compact(_ptr(K), _ptr(V), _dtype_code(K), ctypes.byref(shape.c), int(mode), bud,
                                 _ptr(idx), _ptr(counts), _ptr(offsets), _ptr(Kc), _ptr(Vc), _stream(stream)))
        return
    n = _index_count(shape, mode, bud)
    dev = K.device
    flat = int(mode) == LAYER_FLAT
    D = shape.c.head_dim
    _check(lib.ecokv_compact(_arg(K, "K", _KV_TYPES, shape.kv_numel(), dev),
                             _arg(V, "V", _KV_TYPES, shape.kv_numel(), dev), _dtype_code(K), ctypes.byref(shape.c),
                             int(mode), bud, _arg(idx, "idx", _I32, n, dev),
                             _arg(counts, "counts", _I32, shape.units, dev, optional=True),
                             _arg(offsets, "offsets", _I32, shape.units, dev, optional=not flat),
                             _arg(Kc, "Kc", _KV_TYPES, n * D, dev), _arg(Vc, "Vc", _KV_TYPES, n * D, dev),
                             _stream(stream)))


def ecokv_decode_workspace_size(shape: Shape, max_count: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.ecokv_decode_workspace_size(ctypes.byref(shape.c), int(max_count), ctypes.byref(n)))
    return n.value


def ecokv_decode(Q_dec: torch.Tensor, Kc: torch.Tensor, Vc: torch.Tensor, shape: Shape, counts: torch.Tensor,
                 offsets: torch.Tensor, max_count: int, O: torch.Tensor, lse: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ecokv_decode (attention of one query per head over the compressed cache).
    The rows each unit reads (offsets[u] .. + counts[u]) are device values the
    binding cannot see; the caller guarantees they lie inside Kc and Vc, as
    ecokv_select writes them for a cache that ecokv_compact filled.
    `workspace`: ecokv_decode_workspace_size bytes, or fewer down to one chunk
    of rows for every 768 of max_count."""
    if Kc.dtype != Q_dec.dtype or Vc.dtype != Q_dec.dtype:
        raise TypeError("Q_dec, Kc and Vc must share one element type")
    c = shape.c
    need = ecokv_decode_workspace_size(shape, max_count)
    if c.num_layers == 0:
        return
    dev = Q_dec.device
    D = c.head_dim
    nq = c.num_layers * c.num_q_heads * c.num_seqs
    if Kc.numel() % D or Vc.numel() != Kc.numel():
        raise ValueError("Kc and Vc must hold the same whole number of rows of head_dim elements")
    if workspace is not None:  # what the call can do with (a size held for another shape, say)
        need = 4 * nq * -(-int(max_count) // 768) * (D + 2)
    workspace = _workspace(workspace, need, dev, stream)
    _check(lib.ecokv_decode(_arg(Q_dec, "Q_dec", _KV_TYPES, nq * D, dev), _arg(Kc, "Kc", _KV_TYPES, D, dev),
                            _arg(Vc, "Vc", _KV_TYPES, D, dev), _dtype_code(Q_dec), ctypes.byref(shape.c),
                            _arg(counts, "counts", _I32, shape.units, dev),
                            _arg(offsets, "offsets", _I32, shape.units, dev), int(max_count),
                            _arg(O, "O", _F32, nq * D, dev), _arg(lse, "lse", _F32, nq, dev, optional=True),
                            _arg(workspace, "workspace", _U8, need, dev), workspace.numel(), _stream(stream)))


def _enqueue(fn, device, stream, *args):
    """fn(*args, stream) on `stream` or the current stream of the tensors' device."""
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the call's tensors on {device}")
        raw = stream.cuda_stream
    else:
        raw = torch._C._cuda_getCurrentRawStream(device.index)
    if device.index == torch._C._cuda_getDevice():
        _check(fn(*args, raw))
    else:
        with torch.cuda.device(device):
            _check(fn(*args, raw))


def _fit(t: Optional[torch.Tensor], name: str, dtype, numel: int, device, optional: bool = False):
    """_arg for one element type: a call in order costs fewer Python steps."""
    if t is None and optional:
        return None
    try:
        if t.get_device() == device.index and t.dtype is dtype and t.numel() >= numel and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    return _arg(t, name, (dtype,), numel, device, optional)


def _first(t, name: str):
    """Device and element type of the tensor that the call's others are held to."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
    return t.device, t.dtype, _dtype_code(t)


def _token_rows(t: Optional[torch.Tensor], name: str, dtype, want, device):
    """(pointer, stride) of rows `want` = (L, tokens, heads, dim) (or, for one
    layer, without L) that may lie further apart than they are long: a view of a
    fused projection's output, say."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.get_device() != device.index:
        raise ValueError(f"{name} is on {t.device}, the call's tensors on {device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {_ELEM.get(dtype, str(dtype))} (got {t.dtype})")
    layers, tokens, heads, dim = want
    if t.shape != want and not (layers == 1 and t.shape == want[1:]):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, the call needs {want}")
    packed = heads * dim
    s = t.stride()
    stride = s[-3] if tokens > 1 else s[0] if layers > 1 else packed
    if tokens and ((dim > 1 and s[-1] != 1) or (heads > 1 and s[-2] != dim)
                   or (layers > 1 and s[0] != tokens * stride)):
        raise ValueError(f"{name}: the heads of a token must lie together and the tokens of all layers evenly apart")
    return t.data_ptr(), stride if tokens else packed


def ecokv_rope_freqs(rot_dim: int, base: float = 10000.0, kind: int = ROPE_PLAIN, stretch: float = 1.0,
                     context: float = 0.0):
    """(frequencies as a list of rot_dim / 2 floats, factor) for Rope: radians per position of each pair."""
    rot_dim, kind = _int32(rot_dim, "rot_dim"), _int32(kind, "kind")
    out = (ctypes.c_float * max(rot_dim // 2, 1))()
    factor = ctypes.c_float(0.0)
    _check(lib.ecokv_rope_freqs(rot_dim, float(base), kind, float(stretch), float(context), out,
                                ctypes.byref(factor)))
    return [float(v) for v in out], float(factor.value)


def ecokv_prefill_rope(Q: Optional[torch.Tensor], K: Optional[torch.Tensor], shape: Shape, rope: Rope,
                       positions: Optional[torch.Tensor] = None, Q_out: Optional[torch.Tensor] = None,
                       K_out: Optional[torch.Tensor] = None, Q_win: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ecokv_prefill_rope: Q [L][T_total][H_q][D], K [L][T_total][H_kv][D]
    (views of a fused projection will do) normed and rotated into Q_out, K_out
    (contiguous; K_out is ecokv_prefill_write's K_new) and the window's queries
    into Q_win [L][H_q][B][w][D].  Q without Q_out: only the window's."""
    c = shape.c
    if c.num_layers == 0:
        return
    if Q is None and K is None:
        raise ValueError("Q or K is required")
    if (Q is None) != (Q_out is None and Q_win is None) or (K is None) != (K_out is None):
        raise ValueError("Q goes with Q_out, Q_win or both, K with K_out")
    dev, dt, code = _first(Q if Q is not None else K, "Q" if Q is not None else "K")
    L, Hq, Hkv, D, n = c.num_layers, c.num_q_heads, c.num_kv_heads, c.head_dim, shape.ttot
    qp, qs = _token_rows(Q, "Q", dt, (L, n, Hq, D), dev)
    kp, ks = _token_rows(K, "K", dt, (L, n, Hkv, D), dev)
    _enqueue(lib.ecokv_prefill_rope, dev, stream, qp, qs, kp, ks, code, ctypes.byref(c), rope._arg(D, dt, dev),
             _fit(positions, "positions", torch.int32, n, dev, True), _fit(Q_out, "Q_out", dt, L * n * Hq * D, dev, True),
             _fit(K_out, "K_out", dt, L * n * Hkv * D, dev, True),
             _fit(Q_win, "Q_win", dt, shape.q_numel() if Q_win is not None else 0, dev, True))


def ecokv_append(Q_new: Optional[torch.Tensor], K_new: torch.Tensor, V_new: torch.Tensor, shape: Shape, rope: Rope,
                 positions: torch.Tensor, conts: Optional[torch.Tensor], rows: torch.Tensor, tails: Tails,
                 Q_dec: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ecokv_append: new tokens' keys (normed, rotated) and values into
    the tails, their queries into Q_dec [L][H_q][tokens][D].  Q_new, K_new,
    V_new: [L][tokens][heads][D], views of a fused projection will do;
    positions, conts (None: token t continues t), rows: int32 [tokens], rows of
    -1 mark padding."""
    c = shape.c
    if c.num_layers == 0:
        return
    if V_new is None:
        raise ValueError("V_new is required")
    if (Q_new is None) != (Q_dec is None):
        raise ValueError("Q_new and Q_dec: both or neither")
    dev, dt, code = _first(K_new, "K_new")
    L, Hq, Hkv, D = c.num_layers, c.num_q_heads, c.num_kv_heads, c.head_dim
    n = K_new.shape[-3] if K_new.dim() >= 3 else 0
    kp, ks = _token_rows(K_new, "K_new", dt, (L, n, Hkv, D), dev)
    vp, vs = _token_rows(V_new, "V_new", dt, (L, n, Hkv, D), dev)
    qp, qs = _token_rows(Q_new, "Q_new", dt, (L, n, Hq, D), dev)
    _enqueue(lib.ecokv_append, dev, stream, qp, qs, kp, ks, vp, vs, code, ctypes.byref(c), rope._arg(D, dt, dev),
             _fit(positions, "positions", torch.int32, n, dev), _fit(conts, "conts", torch.int32, n, dev, True),
             _fit(rows, "rows", torch.int32, n, dev), n, tails._arg(shape, dt, dev),
             _fit(Q_dec, "Q_dec", dt, L * Hq * n * D, dev, True))


def _fan(shape: Shape, fan):
    n = shape.c.num_seqs + 1
    if not (type(fan) is list and len(fan) == n):
        fan = _flat_ints(fan)
        if len(fan) != n:
            raise ValueError("fan has one entry per prompt and one more")
    f = (ctypes.c_int32 * n)(*fan)
    if f[:] != fan:
        raise ValueError(f"fan {fan} does not fit 32 bits")
    return f


def ecokv_decode_shared_workspace_size(shape: Shape, fan: Sequence[int], max_count: int, max_tail: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib.ecokv_decode_shared_workspace_size(ctypes.byref(shape.c), _fan(shape, fan), _int32(max_count, "max_count"),
                                                  _int32(max_tail, "max_tail"), ctypes.byref(n)))
    return n.value


def ecokv_decode_shared(Q_dec: torch.Tensor, Kc: Optional[torch.Tensor], Vc: Optional[torch.Tensor], shape: Shape,
                        fan: Sequence[int], counts: Optional[torch.Tensor], offsets: Optional[torch.Tensor],
                        max_count: int, tails: Optional[Tails], tail_counts: Optional[torch.Tensor], max_tail: int,
                        O: torch.Tensor, lse: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue ecokv_decode_shared: one query of each continuation over its
    prompt's kept rows (`fan`: continuations fan[s] .. fan[s + 1] - 1 continue
    prompt s) and its own tail.  As for ecokv_decode, the caller guarantees that
    the rows offsets[u] .. + counts[u] lie inside Kc and Vc."""
    c = shape.c
    f = _fan(shape, fan)
    N = f[c.num_seqs]
    if c.num_layers == 0 or N == 0:
        return
    dev, dt, code = _first(Q_dec, "Q_dec")
    D = c.head_dim
    nq = c.num_layers * c.num_q_heads * N
    max_count, max_tail = _int32(max_count, "max_count"), _int32(max_tail, "max_tail")
    kept, tailed = max_count > 0, max_tail > 0
    qp = _fit(Q_dec, "Q_dec", dt, nq * D, dev)
    units = shape.units
    # (what a bound of 0 leaves unread may be anything)
    kp = vp = cp = op = tp = tc = None
    if kept:
        kp, vp = _fit(Kc, "Kc", dt, D, dev), _fit(Vc, "Vc", dt, D, dev)
        if Kc.numel() % D or Vc.numel() != Kc.numel():
            raise ValueError("Kc and Vc must hold the same whole number of rows of head_dim elements")
        cp, op = _fit(counts, "counts", torch.int32, units, dev), _fit(offsets, "offsets", torch.int32, units, dev)
    if tailed:
        if tails is None:
            raise ValueError("tails is required")
        tp, tc = tails._arg(shape, dt, dev), _fit(tail_counts, "tail_counts", torch.int32, N, dev)
    if workspace is None:
        workspace = _workspace(None, ecokv_decode_shared_workspace_size(shape, fan, max_count, max_tail), dev, stream)
    _enqueue(lib.ecokv_decode_shared, dev, stream, qp, kp, vp, code, ctypes.byref(c), f, cp, op, max_count, tp, tc, max_tail,
             _fit(O, "O", torch.float32, nq * D, dev), _fit(lse, "lse", torch.float32, nq, dev, True),
             _fit(workspace, "workspace", torch.uint8, 0, dev), workspace.numel())


def ecokv_last_error() -> str:
    return lib.ecokv_last_error().decode()


def ecokv_stage_times(max_entries: int = 32) -> dict:
    """Per-kernel times recorded while ECOKV_STAGE_TIMING=1: {name: (ms, launches)}; clears the record."""
    arr = (_StageTime * max_entries)()
    n = ctypes.c_int(0)
    _check(lib.ecokv_stage_times(arr, int(max_entries), ctypes.byref(n)))
    return {arr[i].name.decode(): (arr[i].ms, int(arr[i].launches)) for i in range(n.value)}

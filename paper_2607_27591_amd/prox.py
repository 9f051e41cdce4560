"""Thin ctypes binding of libprox.so (declared in include/prox.h).

Argument marshalling only: every step of the decode FFN runs in the HIP
kernels of libprox.  PyTorch provides device memory and streams.  There is no
fallback: if the library is missing or a call fails, this module raises.
"""
from __future__ import annotations

import ctypes
import dataclasses
import operator
import os
from typing import List, Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libprox.so")

F16, BF16 = 0, 1
INT8, INT4, NONE = 0, 1, 2   # NONE: unquantised 16-bit proxy (group = d_model)
MAX_BATCH = 64   # PROX_MAX_BATCH of include/prox.h
SPARSE_STAGES = 3

_TORCH_DT = {torch.float16: F16, torch.bfloat16: BF16}
_DT_TORCH = {F16: torch.float16, BF16: torch.bfloat16}


class ProxError(RuntimeError):
    """A libprox entry point returned a status other than PROX_OK."""

    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


class _Weights(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int), ("d_ff", ctypes.c_int), ("dtype", ctypes.c_int),
                ("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p),
                ("w_down", ctypes.c_void_p), ("act", ctypes.c_int)]


SILU, GELU = 0, 1   # gate activations: SwiGLU, GeGLU


class _Proxy(ctypes.Structure):
    _fields_ = [("fmt", ctypes.c_int), ("group", ctypes.c_int), ("blob", ctypes.c_void_p),
                ("bytes", ctypes.c_size_t)]


class _W4(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("d_model", ctypes.c_int), ("d_ff", ctypes.c_int),
                ("group", ctypes.c_int), ("act", ctypes.c_int), ("blob", ctypes.c_void_p),
                ("bytes", ctypes.c_size_t)]


class _W4Linear(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("n", ctypes.c_int), ("k", ctypes.c_int),
                ("group", ctypes.c_int), ("blob", ctypes.c_void_p), ("bytes", ctypes.c_size_t)]


class _KVCache(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("group", ctypes.c_int), ("page_size", ctypes.c_int), ("n_pages", ctypes.c_int),
                ("blob", ctypes.c_void_p), ("bytes", ctypes.c_size_t)]


class _KVSeqs(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int), ("max_new", ctypes.c_int), ("n_tokens", ctypes.c_int),
                ("max_kv", ctypes.c_int), ("max_pages", ctypes.c_int), ("cu_new", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("page_table", ctypes.c_void_p)]


class _Rope(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("n_pos", ctypes.c_int), ("dim", ctypes.c_int),
                ("interleaved", ctypes.c_int)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libprox.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_27591_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, I, S, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
        WP, PP = ctypes.POINTER(_Weights), ctypes.POINTER(_Proxy)
        L.prox_proxy_bytes.argtypes = [I, I, I, I]
        L.prox_proxy_bytes.restype = S
        L.prox_pack_proxy.argtypes = [WP, PP, P]
        L.prox_unpack_proxy.argtypes = [PP, I, I, P, P, P, P, P]
        L.prox_workspace_bytes.argtypes = [I, I, I]
        L.prox_workspace_bytes.restype = S
        L.prox_w4_workspace_bytes.argtypes = [I, I, I]
        L.prox_w4_workspace_bytes.restype = S
        L.prox_stage1_mfma_rows.argtypes = [I, I, I, I, I]
        L.prox_stage1_mfma_rows.restype = I
        L.prox_stage2_rows.argtypes = [I, I, I, I]
        L.prox_stage2_rows.restype = I
        L.prox_ffn_dense.argtypes = [WP, P, I, P, P, S, P]
        L.prox_ffn_sparse.argtypes = [WP, PP, P, I, I, I, P, P, P, P, P, S, P]
        L.prox_ffn_sparse_noalloc.argtypes = [WP, PP, P, I, I, I, P, P, P, P, P]
        L.prox_noalloc_max_bytes.argtypes = []
        L.prox_noalloc_max_bytes.restype = S
        L.prox_ffn_sparse_staged.argtypes = [WP, PP, P, I, I, I, P, P, P, P, P, S, P, P]
        L.prox_ffn_sparse_tau.argtypes = [WP, PP, P, I, Z, Z, P, P, P, P, P, P, S, P]
        L.prox_reservoir_add.argtypes = [P, S, P, P, S, P]
        L.prox_quantile_threshold.argtypes = [P, S, ctypes.c_double, P]
        Dd = ctypes.c_double
        L.prox_effective_sparsity.argtypes = [Dd, Dd, Dd]
        L.prox_effective_sparsity.restype = Dd
        L.prox_allocate_sparsity.argtypes = [Dd, Dd, Dd, Dd, Dd, P, P]
        L.prox_sparse_stage_name.argtypes = [I]
        L.prox_sparse_stage_name.restype = ctypes.c_char_p
        L.prox_add_rmsnorm.argtypes = [P, P, I, I, I, Z, P, P]
        QP = ctypes.POINTER(_W4)
        L.prox_w4_bytes.argtypes = [I, I, I]
        L.prox_w4_bytes.restype = S
        L.prox_pack_w4.argtypes = [WP, QP, P]
        L.prox_unpack_w4.argtypes = [QP, I, P, P, P]
        L.prox_ffn_dense_w4.argtypes = [QP, P, I, P, P, S, P]
        L.prox_ffn_sparse_w4.argtypes = [QP, PP, P, I, I, I, P, P, P, P, P, S, P, P]
        L.prox_ffn_sparse_tau_w4.argtypes = [QP, PP, P, I, Z, Z, P, P, P, P, P, P, S, P]
        LP, CP, KP, RP = (ctypes.POINTER(t) for t in (_W4Linear, _KVCache, _KVSeqs, _Rope))
        N = ctypes.c_int64
        L.prox_linear_w4_bytes.argtypes = [I, I, I]
        L.prox_linear_w4_bytes.restype = S
        L.prox_pack_linear_w4.argtypes = [P, LP, P]
        L.prox_unpack_linear_w4.argtypes = [LP, P, P, P]
        L.prox_linear_w4.argtypes = [LP, P, N, I, P, P, N, P]
        L.prox_kv_bytes.argtypes = [I, I, I, I, I]
        L.prox_kv_bytes.restype = S
        L.prox_kv_append.argtypes = [CP, KP, P, N, P, N, P, I, N, P, N, RP, P]
        L.prox_kv_read.argtypes = [CP, KP, P, P, P]
        L.prox_kv_attn_workspace_bytes.argtypes = [I]
        L.prox_kv_attn_workspace_bytes.restype = S
        L.prox_kv_attn.argtypes = [CP, KP, P, I, N, Z, I, P, N, P, S, P]
        L.prox_strerror.argtypes = [I]
        L.prox_strerror.restype = ctypes.c_char_p
        for name in ("prox_pack_proxy", "prox_unpack_proxy", "prox_ffn_dense", "prox_ffn_sparse",
                     "prox_ffn_sparse_staged", "prox_ffn_sparse_tau", "prox_add_rmsnorm",
                     "prox_reservoir_add", "prox_quantile_threshold", "prox_allocate_sparsity",
                     "prox_pack_w4", "prox_unpack_w4", "prox_ffn_dense_w4", "prox_ffn_sparse_w4",
                     "prox_ffn_sparse_tau_w4", "prox_pack_linear_w4", "prox_unpack_linear_w4",
                     "prox_linear_w4", "prox_kv_append", "prox_kv_read", "prox_kv_attn"):
            getattr(L, name).restype = I
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().prox_strerror(int(status)).decode()


def stage_names() -> List[str]:
    return [lib().prox_sparse_stage_name(i).decode() for i in range(SPARSE_STAGES)]


def _check(status: int, where: str) -> None:
    if status != 0:
        raise ProxError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device: torch.device):
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _dev_tensor(t: torch.Tensor, what: str, dtype=None) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise ValueError(f"{what} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what} must have dtype {dtype}, got {t.dtype}")
    return t


@dataclasses.dataclass
class Weights:
    """Channel-major gated-FFN weights, each [d_ff][d_model] in fp16 or bf16;
    act is the gate activation (SILU: SwiGLU, GELU: GeGLU)."""
    w_gate: torch.Tensor
    w_up: torch.Tensor
    w_down: torch.Tensor
    act: int = SILU

    @property
    def d_ff(self) -> int:
        return self.w_gate.shape[0]

    @property
    def d_model(self) -> int:
        return self.w_gate.shape[1]

    @property
    def dtype(self) -> torch.dtype:
        return self.w_gate.dtype

    def struct(self) -> _Weights:
        dt = _TORCH_DT.get(self.w_gate.dtype)
        if dt is None:
            raise ValueError("weights must be float16 or bfloat16")
        for name in ("w_gate", "w_up", "w_down"):
            t = _dev_tensor(getattr(self, name), name, self.w_gate.dtype)
            if tuple(t.shape) != (self.d_ff, self.d_model):
                raise ValueError(f"{name} must be [d_ff][d_model]")
        return _Weights(self.d_model, self.d_ff, dt, self.w_gate.data_ptr(),
                        self.w_up.data_ptr(), self.w_down.data_ptr(), int(self.act))


@dataclasses.dataclass
class Proxy:
    """A packed proxy blob (opaque device bytes) with its format."""
    blob: torch.Tensor
    fmt: int
    group: int

    def struct(self) -> _Proxy:
        _dev_tensor(self.blob, "proxy blob", torch.uint8)
        return _Proxy(self.fmt, self.group, self.blob.data_ptr(), self.blob.numel())


def proxy_bytes(d_model: int, d_ff: int, fmt: int, group: int) -> int:
    return int(lib().prox_proxy_bytes(d_model, d_ff, fmt, group))


def stage1_mfma_rows(d_model: int, fmt: int, group: int, batch: int, k_in: int) -> int:
    """Batch rows per launch of the 16-row matrix-core Stage-1 kernel, 0 when a
    call takes another one (threshold mode: pass k_in = d_model)."""
    return int(lib().prox_stage1_mfma_rows(d_model, fmt, group, batch, k_in))


def stage2_rows(d_model: int, d_ff: int, w4: bool, batch: int) -> int:
    """Batch rows per Stage-2 launch: 16 on the matrix-core kernel, else the
    VALU kernel's row count; 0 for an unsupported shape or batch."""
    return int(lib().prox_stage2_rows(d_model, d_ff, int(w4), batch))


def workspace_bytes(d_model: int, d_ff: int, batch: int, w4: bool = False) -> int:
    """prox_workspace_bytes, or prox_w4_workspace_bytes for INT4 base weights."""
    f = lib().prox_w4_workspace_bytes if w4 else lib().prox_workspace_bytes
    return int(f(d_model, d_ff, batch))


def new_workspace(d_model: int, d_ff: int, batch: int, device="cuda", w4: bool = False) -> torch.Tensor:
    n = workspace_bytes(d_model, d_ff, batch, w4)
    if n == 0:
        raise ProxError(2, "prox_w4_workspace_bytes" if w4 else "prox_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def pack_proxy(w: Weights, fmt: int = INT4, group: int = 128) -> Proxy:
    if fmt == NONE:
        group = w.d_model   # the unquantised proxy has one unit scale per channel
    n = proxy_bytes(w.d_model, w.d_ff, fmt, group)
    if n == 0:
        raise ProxError(2, "prox_proxy_bytes")
    p = Proxy(torch.empty(n, dtype=torch.uint8, device=w.w_gate.device), fmt, group)
    ws, ps = w.struct(), p.struct()
    _check(lib().prox_pack_proxy(ctypes.byref(ws), ctypes.byref(ps), _stream(w.w_gate.device)),
           "prox_pack_proxy")
    return p


def unpack_proxy(p: Proxy, d_model: int, d_ff: int):
    """(codes_gate int8 [f][d], scales_gate fp16-bits int16 [f][d/g], codes_up, scales_up)."""
    dev = p.blob.device
    ng = d_model // p.group
    cg = torch.empty((d_ff, d_model), dtype=torch.int8, device=dev)
    cu = torch.empty_like(cg)
    sg = torch.empty((d_ff, ng), dtype=torch.int16, device=dev)
    su = torch.empty_like(sg)
    ps = p.struct()
    _check(lib().prox_unpack_proxy(ctypes.byref(ps), d_model, d_ff, _ptr(cg), _ptr(sg), _ptr(cu),
                                   _ptr(su), _stream(dev)), "prox_unpack_proxy")
    return cg, sg, cu, su


def _as_batch(x: torch.Tensor, w: Weights) -> torch.Tensor:
    x = _dev_tensor(x, "x", w.dtype)
    if x.dim() == 1:
        x = x.view(1, -1)
    if x.dim() != 2 or x.shape[1] != w.d_model:
        raise ValueError("x must be [batch][d_model]")
    return x


def ffn_dense(w: Weights, x: torch.Tensor, y: Optional[torch.Tensor] = None,
              ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    x = _as_batch(x, w)
    B = x.shape[0]
    y = torch.empty_like(x) if y is None else _dev_tensor(y, "y", w.dtype)
    ws = new_workspace(w.d_model, w.d_ff, B, x.device) if ws is None else ws
    wst = w.struct()
    _check(lib().prox_ffn_dense(ctypes.byref(wst), _ptr(x), B, _ptr(y), _ptr(ws), ws.numel(),
                                _stream(x.device)), "prox_ffn_dense")
    return y


def ffn_sparse(w: Weights, p: Proxy, x: torch.Tensor, k_in: int, k_ff: int, *,
               y: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
               in_mask: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None,
               ws: Optional[torch.Tensor] = None,
               events: Optional[Sequence[torch.cuda.Event]] = None):
    """Prox sparse decode step.  Returns (y, mask).  ``in_mask`` / ``scores``
    are filled when given.  ``events`` (PROX_SPARSE_STAGES + 1 timing events,
    already recorded once so they exist) selects the staged entry point."""
    x = _as_batch(x, w)
    B = x.shape[0]
    dev = x.device
    y = torch.empty_like(x) if y is None else _dev_tensor(y, "y", w.dtype)
    mask = (torch.empty(w.d_ff, dtype=torch.uint8, device=dev) if mask is None
            else _dev_tensor(mask, "mask", torch.uint8))
    if in_mask is not None:
        _dev_tensor(in_mask, "in_mask", torch.uint8)
    if scores is not None:
        _dev_tensor(scores, "scores", torch.float32)
    ws = new_workspace(w.d_model, w.d_ff, B, dev) if ws is None else ws
    wst, pst = w.struct(), p.struct()
    args = [ctypes.byref(wst), ctypes.byref(pst), _ptr(x), B, int(k_in), int(k_ff), _ptr(y),
            _ptr(mask), _ptr(in_mask), _ptr(scores), _ptr(ws), ws.numel()]
    if events is None:
        _check(lib().prox_ffn_sparse(*args, _stream(dev)), "prox_ffn_sparse")
    else:
        if len(events) != SPARSE_STAGES + 1:
            raise ValueError(f"need {SPARSE_STAGES + 1} events")
        arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
        _check(lib().prox_ffn_sparse_staged(*args, arr, _stream(dev)), "prox_ffn_sparse_staged")
    return y, mask


def ffn_sparse_noalloc(w: Weights, p: Proxy, x: torch.Tensor, k_in: int, k_ff: int, *,
                       y: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                       in_mask: Optional[torch.Tensor] = None,
                       scores: Optional[torch.Tensor] = None):
    """prox_ffn_sparse_noalloc: the sparse decode step on the library's own
    device scratch (no workspace argument; the C call allocates nothing).
    Returns (y, mask); y and mask are allocated here when not given."""
    x = _as_batch(x, w)
    B = x.shape[0]
    dev = x.device
    y = torch.empty_like(x) if y is None else _dev_tensor(y, "y", w.dtype)
    mask = (torch.empty(w.d_ff, dtype=torch.uint8, device=dev) if mask is None
            else _dev_tensor(mask, "mask", torch.uint8))
    if in_mask is not None:
        _dev_tensor(in_mask, "in_mask", torch.uint8)
    if scores is not None:
        _dev_tensor(scores, "scores", torch.float32)
    wst, pst = w.struct(), p.struct()
    _check(lib().prox_ffn_sparse_noalloc(ctypes.byref(wst), ctypes.byref(pst), _ptr(x), B,
                                         int(k_in), int(k_ff), _ptr(y), _ptr(mask),
                                         _ptr(in_mask), _ptr(scores), _stream(dev)),
           "prox_ffn_sparse_noalloc")
    return y, mask


def noalloc_max_bytes() -> int:
    """Scratch bytes per GPU of prox_ffn_sparse_noalloc (the workspace of a call
    must fit)."""
    return int(lib().prox_noalloc_max_bytes())


def ffn_sparse_tau(w: Weights, p: Proxy, x: torch.Tensor, tau_x: float, tau_s: float, *,
                   y: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                   in_mask: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None,
                   counts: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Prox decode step with layer-wise thresholds (keep |x| >= tau_x and
    score >= tau_s).  Returns (y, mask, counts) with counts an int32 [2]
    device tensor (k_in, k_ff realised by this call)."""
    x = _as_batch(x, w)
    B = x.shape[0]
    dev = x.device
    y = torch.empty_like(x) if y is None else _dev_tensor(y, "y", w.dtype)
    mask = (torch.empty(w.d_ff, dtype=torch.uint8, device=dev) if mask is None
            else _dev_tensor(mask, "mask", torch.uint8))
    counts = (torch.empty(2, dtype=torch.int32, device=dev) if counts is None
              else _dev_tensor(counts, "counts", torch.int32))
    if in_mask is not None:
        _dev_tensor(in_mask, "in_mask", torch.uint8)
    if scores is not None:
        _dev_tensor(scores, "scores", torch.float32)
    ws = new_workspace(w.d_model, w.d_ff, B, dev) if ws is None else ws
    wst, pst = w.struct(), p.struct()
    _check(lib().prox_ffn_sparse_tau(ctypes.byref(wst), ctypes.byref(pst), _ptr(x), B,
                                     float(tau_x), float(tau_s), _ptr(y), _ptr(mask),
                                     _ptr(in_mask), _ptr(scores), _ptr(counts), _ptr(ws),
                                     ws.numel(), _stream(dev)), "prox_ffn_sparse_tau")
    return y, mask, counts


@dataclasses.dataclass
class W4Weights:
    """INT4 copy of the three FFN matrices for Stage 2 (W4A16): an opaque
    device blob in the layout include/prox.h describes."""
    blob: torch.Tensor
    dtype: torch.dtype
    d_model: int
    d_ff: int
    group: int
    act: int = SILU

    def struct(self) -> _W4:
        _dev_tensor(self.blob, "W4 blob", torch.uint8)
        return _W4(_TORCH_DT[self.dtype], self.d_model, self.d_ff, self.group, int(self.act),
                   self.blob.data_ptr(), self.blob.numel())


def w4_bytes(d_model: int, d_ff: int, group: int = 128) -> int:
    return int(lib().prox_w4_bytes(d_model, d_ff, group))


def pack_w4(w: Weights, group: int = 128) -> W4Weights:
    n = w4_bytes(w.d_model, w.d_ff, group)
    if n == 0:
        raise ProxError(2, "prox_w4_bytes")
    q = W4Weights(torch.empty(n, dtype=torch.uint8, device=w.w_gate.device), w.dtype, w.d_model,
                  w.d_ff, group, w.act)
    ws, qs = w.struct(), q.struct()
    _check(lib().prox_pack_w4(ctypes.byref(ws), ctypes.byref(qs), _stream(w.w_gate.device)),
           "prox_pack_w4")
    return q


def unpack_w4(q: W4Weights, matrix: int):
    """(codes int8 [d_ff][d_model], scales fp16 bits int16 [d_ff][d_model / group]) of
    matrix 0 (gate), 1 (up) or 2 (down)."""
    dev = q.blob.device
    codes = torch.empty((q.d_ff, q.d_model), dtype=torch.int8, device=dev)
    scales = torch.empty((q.d_ff, q.d_model // q.group), dtype=torch.int16, device=dev)
    qs = q.struct()
    _check(lib().prox_unpack_w4(ctypes.byref(qs), int(matrix), _ptr(codes), _ptr(scales),
                                _stream(dev)), "prox_unpack_w4")
    return codes, scales


def _as_batch_w4(x: torch.Tensor, q: W4Weights) -> torch.Tensor:
    x = _dev_tensor(x, "x", q.dtype)
    if x.dim() == 1:
        x = x.view(1, -1)
    if x.dim() != 2 or x.shape[1] != q.d_model:
        raise ValueError("x must be [batch][d_model]")
    return x


def ffn_dense_w4(q: W4Weights, x: torch.Tensor, y: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The dense FFN on the INT4 weights."""
    x = _as_batch_w4(x, q)
    B = x.shape[0]
    y = torch.empty_like(x) if y is None else _dev_tensor(y, "y", q.dtype)
    ws = new_workspace(q.d_model, q.d_ff, B, x.device, w4=True) if ws is None else ws
    qs = q.struct()
    _check(lib().prox_ffn_dense_w4(ctypes.byref(qs), _ptr(x), B, _ptr(y), _ptr(ws), ws.numel(),
                                   _stream(x.device)), "prox_ffn_dense_w4")
    return y


def ffn_sparse_w4(q: W4Weights, p: Proxy, x: torch.Tensor, k_in: int, k_ff: int, *,
                  y: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                  in_mask: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None,
                  events: Optional[Sequence[torch.cuda.Event]] = None):
    """The sparse decode step with Stage 2 on the INT4 weights.  Returns
    (y, mask); arguments as ffn_sparse."""
    x = _as_batch_w4(x, q)
    B = x.shape[0]
    dev = x.device
    y = torch.empty_like(x) if y is None else _dev_tensor(y, "y", q.dtype)
    mask = (torch.empty(q.d_ff, dtype=torch.uint8, device=dev) if mask is None
            else _dev_tensor(mask, "mask", torch.uint8))
    if in_mask is not None:
        _dev_tensor(in_mask, "in_mask", torch.uint8)
    if scores is not None:
        _dev_tensor(scores, "scores", torch.float32)
    ws = new_workspace(q.d_model, q.d_ff, B, dev, w4=True) if ws is None else ws
    arr = None
    if events is not None:
        if len(events) != SPARSE_STAGES + 1:
            raise ValueError(f"need {SPARSE_STAGES + 1} events")
        arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    qs, pst = q.struct(), p.struct()
    _check(lib().prox_ffn_sparse_w4(ctypes.byref(qs), ctypes.byref(pst), _ptr(x), B, int(k_in),
                                    int(k_ff), _ptr(y), _ptr(mask), _ptr(in_mask), _ptr(scores),
                                    _ptr(ws), ws.numel(), arr, _stream(dev)), "prox_ffn_sparse_w4")
    return y, mask


def ffn_sparse_tau_w4(q: W4Weights, p: Proxy, x: torch.Tensor, tau_x: float, tau_s: float, *,
                      y: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                      in_mask: Optional[torch.Tensor] = None,
                      scores: Optional[torch.Tensor] = None,
                      counts: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """Threshold-mode step with Stage 2 on the INT4 weights.  Returns
    (y, mask, counts) like ffn_sparse_tau."""
    x = _as_batch_w4(x, q)
    B = x.shape[0]
    dev = x.device
    y = torch.empty_like(x) if y is None else _dev_tensor(y, "y", q.dtype)
    mask = (torch.empty(q.d_ff, dtype=torch.uint8, device=dev) if mask is None
            else _dev_tensor(mask, "mask", torch.uint8))
    counts = (torch.empty(2, dtype=torch.int32, device=dev) if counts is None
              else _dev_tensor(counts, "counts", torch.int32))
    if in_mask is not None:
        _dev_tensor(in_mask, "in_mask", torch.uint8)
    if scores is not None:
        _dev_tensor(scores, "scores", torch.float32)
    ws = new_workspace(q.d_model, q.d_ff, B, dev, w4=True) if ws is None else ws
    qs, pst = q.struct(), p.struct()
    _check(lib().prox_ffn_sparse_tau_w4(ctypes.byref(qs), ctypes.byref(pst), _ptr(x), B,
                                        float(tau_x), float(tau_s), _ptr(y), _ptr(mask),
                                        _ptr(in_mask), _ptr(scores), _ptr(counts), _ptr(ws),
                                        ws.numel(), _stream(dev)), "prox_ffn_sparse_tau_w4")
    return y, mask, counts


def effective_sparsity(s1: float, s2: float, alpha: float = 1.0 / 3.0) -> float:
    """Sec. 4.2 effective sparsity of stage sparsities (s1, s2)."""
    return float(lib().prox_effective_sparsity(float(s1), float(s2), float(alpha)))


def allocate_sparsity(e: float, alpha: float = 1.0 / 3.0, s_ref: float = 0.7,
                      s1_min: float = 0.0, s1_max: float = 0.7):
    """Sec. 4.2 allocation of a target effective sparsity: (s1, s2)."""
    a, b = ctypes.c_double(), ctypes.c_double()
    _check(lib().prox_allocate_sparsity(float(e), float(alpha), float(s_ref), float(s1_min),
                                        float(s1_max), ctypes.byref(a), ctypes.byref(b)),
           "prox_allocate_sparsity")
    return a.value, b.value


def add_rmsnorm(x: torch.Tensor, y: torch.Tensor, eps: float = 1e-6,
                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    dt = _TORCH_DT.get(x.dtype)
    if dt is None:
        raise ValueError("x must be float16 or bfloat16")
    x = _dev_tensor(x, "x")
    y = _dev_tensor(y, "y", x.dtype)
    x2 = x.view(1, -1) if x.dim() == 1 else x
    out = torch.empty_like(x) if out is None else _dev_tensor(out, "out", x.dtype)
    _check(lib().prox_add_rmsnorm(_ptr(x), _ptr(y), x2.shape[0], x2.shape[1], dt,
                                  ctypes.c_float(eps), _ptr(out), _stream(x.device)),
           "prox_add_rmsnorm")
    return out


# ---------------------------------------------------------------------------
# The attention half of a decoder layer
# ---------------------------------------------------------------------------

# These calls sit between small kernels of a decode step, so they keep their own cost low:
# a handle's C struct is built once (and again if its tensor's memory has moved), pointers go
# as integers.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # without the Stream object
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _on(device: torch.device, f, *args) -> int:
    """f(*args, stream) on the current stream of `device`, which may not be the
    current device."""
    index = device.index
    if index != _current_device():
        with torch.cuda.device(device):
            return f(*args, torch.cuda.current_stream(device).cuda_stream)
    return f(*args, torch.cuda.current_stream(device).cuda_stream if _raw_stream is None else _raw_stream(index))


def _int32(v) -> int:
    """v, or the nearest end of a C int: an argument past 32 bits is refused (or, a window, as good as none)
    instead of losing its upper bits."""
    return max(-2 ** 31, min(operator.index(v), 2 ** 31 - 1))


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _same_device(device: torch.device, *tensors) -> None:
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"every tensor of a call must be on one device: {t.device} and {device}")


class _Handle:
    """Keeps the C struct of an immutable dataclass, as a pointer to pass (which copies of
    the object make anew)."""

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_kept"}

    _kept = None

    def _pointer(self, t: torch.Tensor):
        kept, at, shape = self._kept, t.data_ptr(), t.shape
        if kept is None or kept[0] != at or kept[1] != shape:
            kept = (at, shape, ctypes.byref(self.struct()))
            object.__setattr__(self, "_kept", kept)
        return kept[2]


@dataclasses.dataclass(frozen=True)
class LinearW4(_Handle):
    """A projection's weights in INT4 (W4A16): an opaque device blob."""
    blob: torch.Tensor
    dtype: torch.dtype
    n: int
    k: int
    group: int

    def struct(self) -> _W4Linear:
        _dev_tensor(self.blob, "linear blob", torch.uint8)
        return _W4Linear(_TORCH_DT[self.dtype], _int32(self.n), _int32(self.k), _int32(self.group),
                         self.blob.data_ptr(), self.blob.numel())

    def pointer(self):
        return self._pointer(self.blob)


def linear_w4_bytes(n: int, k: int, group: int = 128) -> int:
    return int(lib().prox_linear_w4_bytes(*map(_int32, (n, k, group))))


def pack_linear_w4(w: torch.Tensor, group: int = 128) -> LinearW4:
    """Quantise nn.Linear's weight w [n][k] (float16 or bfloat16)."""
    if w.dtype not in _TORCH_DT:
        raise ValueError("weights must be float16 or bfloat16")
    _dev_tensor(w, "w")
    if w.dim() != 2:
        raise ValueError("w must be [n][k]")
    n, k = w.shape
    size = linear_w4_bytes(n, k, group)
    if size == 0:
        raise ProxError(2, "prox_linear_w4_bytes")
    q = LinearW4(torch.empty(size, dtype=torch.uint8, device=w.device), w.dtype, n, k, group)
    _check(_on(w.device, lib().prox_pack_linear_w4, _at(w), q.pointer()), "prox_pack_linear_w4")
    return q


def unpack_linear_w4(q: LinearW4):
    """(codes int8 [n][k], scales fp16 bits int16 [n][k / group])."""
    dev = q.blob.device
    codes = torch.empty((q.n, q.k), dtype=torch.int8, device=dev)
    scales = torch.empty((q.n, q.k // q.group), dtype=torch.int16, device=dev)
    _check(_on(dev, lib().prox_unpack_linear_w4, q.pointer(), _at(codes), _at(scales)),
           "prox_unpack_linear_w4")
    return codes, scales


def _rows2(t: torch.Tensor, what: str, dtype: torch.dtype, cols: int):
    """(rows, row stride) of a device tensor [rows][cols], or [cols], whose rows may stand apart."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA (HIP) tensor")
    if t.dtype != dtype:
        raise ValueError(f"{what} must have dtype {dtype}, got {t.dtype}")
    shape, stride = t.shape, t.stride()
    if not 1 <= len(shape) <= 2 or shape[-1] != cols or (cols > 1 and stride[-1] != 1):
        raise ValueError(f"{what} must be [rows][{cols}] with contiguous rows")
    return (shape[0], stride[0]) if len(shape) == 2 and shape[0] != 1 else (1, cols)


def linear_w4(q: LinearW4, x: torch.Tensor, bias: Optional[torch.Tensor] = None,
              y: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [batch][k] (or [k]) times the INT4 weights, plus bias [n]; rows of x and y may
    stand apart (parts of wider tensors)."""
    batch, ldx = _rows2(x, "x", q.dtype, q.k)
    dev = x.device
    if y is None:
        y = torch.empty(x.shape[:-1] + (q.n,), dtype=q.dtype, device=dev)
    rows, ldy = _rows2(y, "y", q.dtype, q.n)
    if rows != batch:
        raise ValueError("y must have the rows of x")
    if bias is not None:
        _dev_tensor(bias, "bias", q.dtype)
        if bias.numel() != q.n:
            raise ValueError("bias must be [n]")
    _same_device(dev, q.blob, y, bias)
    _check(_on(dev, lib().prox_linear_w4, q.pointer(), x.data_ptr(), ldx, batch, _at(bias), y.data_ptr(), ldy),
           "prox_linear_w4")
    return y


@dataclasses.dataclass(frozen=True)
class KVCache(_Handle):
    """Paged key/value cache in 4 bits: an opaque device blob."""
    blob: torch.Tensor
    dtype: torch.dtype
    kv_heads: int
    head_dim: int
    group: int
    page_size: int
    n_pages: int

    def struct(self) -> _KVCache:
        _dev_tensor(self.blob, "cache blob", torch.uint8)
        shape = map(_int32, (self.kv_heads, self.head_dim, self.group, self.page_size, self.n_pages))
        return _KVCache(_TORCH_DT[self.dtype], *shape, self.blob.data_ptr(), self.blob.numel())

    def pointer(self):
        return self._pointer(self.blob)


def kv_bytes(kv_heads: int, head_dim: int, group: int, page_size: int, n_pages: int) -> int:
    return int(lib().prox_kv_bytes(*map(_int32, (kv_heads, head_dim, group, page_size, n_pages))))


def new_kv_cache(n_pages: int, page_size: int, kv_heads: int, head_dim: int, dtype: torch.dtype,
                 group: int = 64, device="cuda") -> KVCache:
    if dtype not in _TORCH_DT:
        raise ValueError("dtype must be float16 or bfloat16")
    n = kv_bytes(kv_heads, head_dim, group, page_size, n_pages)
    if n == 0:
        raise ProxError(2, "prox_kv_bytes")
    return KVCache(torch.empty(n, dtype=torch.uint8, device=device), dtype, kv_heads, head_dim, group,
                   page_size, n_pages)


@dataclasses.dataclass(frozen=True)
class KVSeqs(_Handle):
    """The sequences of a call (prox_kv_seqs): device int32 kv_len [n_seq] (the new
    tokens included), page_table [n_seq][max_pages] and, where sequences have unequal
    numbers of new tokens (at most max_new), cu_new [n_seq + 1].  max_kv bounds kv_len
    (0: what the page table holds)."""
    kv_len: torch.Tensor
    page_table: torch.Tensor
    max_new: int = 1
    cu_new: Optional[torch.Tensor] = None
    max_kv: int = 0

    def struct(self, n_tokens: int = 0) -> _KVSeqs:
        _dev_tensor(self.kv_len, "kv_len", torch.int32)
        _dev_tensor(self.page_table, "page_table", torch.int32)
        n = self.kv_len.numel()
        if self.page_table.dim() != 2 or self.page_table.shape[0] != n:
            raise ValueError("page_table must be [n_seq][max_pages]")
        if self.cu_new is not None:
            _dev_tensor(self.cu_new, "cu_new", torch.int32)
            if self.cu_new.numel() != n + 1:
                raise ValueError("cu_new must be [n_seq + 1]")
        counts = map(_int32, (n, self.max_new, n_tokens, self.max_kv, self.page_table.shape[1]))
        return _KVSeqs(*counts, _at(self.cu_new), self.kv_len.data_ptr(), self.page_table.data_ptr())

    def pointer(self, device: torch.device, n_tokens: int):
        """For a call of n_tokens rows on `device`."""
        key = (device, n_tokens, self.kv_len.data_ptr(), self.page_table.data_ptr(), _at(self.cu_new),
               self.kv_len.shape, self.page_table.shape)
        kept = self._kept
        if kept is None or kept[0] != key:
            _same_device(device, self.kv_len, self.page_table, self.cu_new)
            kept = (key, ctypes.byref(self.struct(n_tokens)))
            object.__setattr__(self, "_kept", kept)
        return kept[1]


@dataclasses.dataclass(frozen=True)
class Rope(_Handle):
    """Rotation table, device float32 [n_pos][dim]: dim / 2 cosines, then the sines, of
    every position; pairs (i, i + dim / 2), or (2 i, 2 i + 1) if interleaved."""
    table: torch.Tensor
    interleaved: bool = False

    def struct(self) -> _Rope:
        _dev_tensor(self.table, "rope table", torch.float32)
        if self.table.dim() != 2:
            raise ValueError("rope table must be [n_pos][dim]")
        return _Rope(self.table.data_ptr(), self.table.shape[0], self.table.shape[1], int(self.interleaved))

    def pointer(self):
        return self._pointer(self.table)


def _heads(t: torch.Tensor, what: str, c: KVCache, heads: int = 0):
    """(tokens, heads, token stride) of a device tensor [tokens][heads][head_dim]."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{what} must be a CUDA (HIP) tensor")
    if t.dtype != c.dtype:
        raise ValueError(f"{what} must have dtype {c.dtype}, got {t.dtype}")
    shape, stride, d = t.shape, t.stride(), c.head_dim
    if (len(shape) != 3 or shape[2] != d or (heads and shape[1] != heads) or stride[2] != 1 or
            (shape[1] > 1 and stride[1] != d)):
        raise ValueError(f"{what} must be [tokens][{heads or 'heads'}][{d}] with the heads of a token contiguous")
    return shape[0], shape[1], stride[0] if shape[0] > 1 else shape[1] * d


def kv_append(c: KVCache, s: KVSeqs, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, rope: Optional[Rope] = None) -> Optional[torch.Tensor]:
    """Append the new tokens' k and v [tokens][kv_heads][head_dim] to the cache, rotated by
    rope if given.  Returns the rotated queries (q_out, which may be q; made here when
    not given), None without q."""
    T, _, ldk = _heads(k, "k", c, c.kv_heads)
    tv, _, ldv = _heads(v, "v", c, c.kv_heads)
    tq = to = T
    ldq = ldo = heads = 0
    dev = k.device
    if q is not None:
        tq, heads, ldq = _heads(q, "q", c)
        if q_out is None:   # rows without a place are not written
            q_out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        to, _, ldo = _heads(q_out, "q_out", c, heads)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if not T == tv == tq == to:
        raise ValueError("k, v, q and q_out must have the same tokens")
    _same_device(dev, c.blob, v, q, q_out, None if rope is None else rope.table)
    _check(_on(dev, lib().prox_kv_append, c.pointer(), s.pointer(dev, T), k.data_ptr(), ldk, v.data_ptr(), ldv,
               _at(q), heads, ldq, _at(q_out), ldo, None if rope is None else rope.pointer()), "prox_kv_append")
    return q_out


def kv_read(c: KVCache, s: KVSeqs, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
            n_tokens: Optional[int] = None):
    """(k, v) float32 [n_tokens][kv_heads][head_dim]: what the cache holds of the call's
    tokens.  n_tokens: needed with cu_new when neither k nor v is given."""
    if n_tokens is None:
        given = k if k is not None else v
        if given is None and s.cu_new is not None:
            raise ValueError("n_tokens is needed")
        n_tokens = s.kv_len.numel() * s.max_new if given is None else given.shape[0]
    shape = (n_tokens, c.kv_heads, c.head_dim)
    dev = c.blob.device
    k = torch.zeros(shape, dtype=torch.float32, device=dev) if k is None else _dev_tensor(k, "k", torch.float32)
    v = torch.zeros(shape, dtype=torch.float32, device=dev) if v is None else _dev_tensor(v, "v", torch.float32)
    if tuple(k.shape) != shape or tuple(v.shape) != shape:
        raise ValueError("k and v must be [n_tokens][kv_heads][head_dim]")
    _same_device(dev, k, v)
    _check(_on(dev, lib().prox_kv_read, c.pointer(), s.pointer(dev, n_tokens), k.data_ptr(), v.data_ptr()),
           "prox_kv_read")
    return k, v


def kv_attn_workspace_bytes(head_dim: int) -> int:
    return int(lib().prox_kv_attn_workspace_bytes(_int32(head_dim)))


def new_kv_attn_workspace(head_dim: int, device="cuda") -> torch.Tensor:
    n = kv_attn_workspace_bytes(head_dim)
    if n == 0:
        raise ProxError(2, "prox_kv_attn_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def kv_attn(c: KVCache, s: KVSeqs, q: torch.Tensor, scale: Optional[float] = None, window: int = 0,
            out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the new tokens' queries [tokens][q_heads][head_dim] over the cache
    (which holds the tokens' own keys and values already).  scale: head_dim ** -0.5 when
    not given; window > 0: the last `window` positions only."""
    T, heads, ldq = _heads(q, "q", c)
    dev = q.device
    if out is None:   # rows of no sequence are not written
        out = (torch.empty if s.cu_new is None else torch.zeros)(q.shape, dtype=q.dtype, device=dev)
    rows, _, ldo = _heads(out, "out", c, heads)
    if rows != T:
        raise ValueError("out must have the tokens of q")
    ws = new_kv_attn_workspace(c.head_dim, dev) if ws is None else _dev_tensor(ws, "ws", torch.uint8)
    _same_device(dev, c.blob, out, ws)
    _check(_on(dev, lib().prox_kv_attn, c.pointer(), s.pointer(dev, T), q.data_ptr(), heads, ldq,
               c.head_dim ** -0.5 if scale is None else float(scale), _int32(int(window)), out.data_ptr(), ldo,
               ws.data_ptr(), ws.numel()), "prox_kv_attn")
    return out


def from_bits(bits, dtype_code: int, device="cuda") -> torch.Tensor:
    """numpy uint16 bit patterns -> device tensor of the matching 16-bit dtype."""
    import numpy as np
    t = torch.from_numpy(np.ascontiguousarray(bits, dtype=np.uint16).view(np.int16))
    return t.to(device).view(_DT_TORCH[dtype_code])


def to_bits(t: torch.Tensor):
    """Device 16-bit tensor -> numpy uint16 bit patterns."""
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view("uint16")

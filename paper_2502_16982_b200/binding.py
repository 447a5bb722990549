"""ctypes binding of the Muon C ABI (include/muon.h).

Argument marshalling only: every step of the optimizer runs in the CUDA
kernels of libmuon_b200.so.  PyTorch supplies device memory and streams.
The functions carry the C names; :class:`MuonContext` bundles them for the
usual init / step / status / destroy life cycle.
"""

from __future__ import annotations

import contextlib
import ctypes as C
import os
from dataclasses import dataclass
from typing import List, NamedTuple, Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmuon_b200.so")

MUON_OK = 0
MUON_ERR_INVALID_ARG = -1
MUON_ERR_UNSUPPORTED = -2
MUON_ERR_ALIGNMENT = -3
MUON_ERR_WORKSPACE = -4
MUON_ERR_CUDA = -5
MUON_ERR_TIMEOUT = -6
MUON_ERR_NONFINITE = -7
MUON_DTYPE_BF16 = 0
MUON_DTYPE_FP32 = 1
MUON_TAP_X0, MUON_TAP_A, MUON_TAP_B, MUON_TAP_X = 0, 1, 2, 3
MUON_SCALE_ADJUSTED_LR, MUON_SCALE_FIXED_DIM, MUON_SCALE_UPDATE_NORM = 0, 1, 2

EXPORTED = [
    "muon_workspace_bytes", "muon_partition", "muon_partition_slots", "muon_plan_buckets", "muon_plan_flops", "muon_plan_work", "muon_debug_tile_table", "muon_init", "muon_step", "muon_step_bucket",
    "muon_step_host", "muon_status",
    "muon_get_norms", "muon_get_update_rms", "muon_destroy", "muon_last_error", "muon_last_launch_count",
    "muon_debug_keep", "muon_debug_read", "muon_debug_set_chunk_bytes", "muon_debug_set_pair_fold", "muon_debug_set_tile_mode",
    "muon_debug_wait_expiry",
    "muon_profile_enable", "muon_profile_read", "muon_debug_tmem_bases",
    "muon_momentum_norm_static", "muon_adamw_step",
    "muon_head_workspace_bytes", "muon_head_xent", "muon_head_distill", "muon_head_status",
    "muon_debug_set_head_piece_bytes", "muon_debug_set_head_codes",
]
MUON_STATIC_MAX_TILES = 65536
KERNEL_KINDS = ["momentum", "norm", "gram", "poly", "comb", "update"]


class muon_group(C.Structure):
    _fields_ = [
        ("rows", C.c_int32), ("cols", C.c_int32), ("count", C.c_int32),
        ("w_dtype", C.c_int32), ("g_dtype", C.c_int32), ("reserved", C.c_int32),
        ("w", C.POINTER(C.c_void_p)), ("g", C.POINTER(C.c_void_p)), ("m", C.POINTER(C.c_void_p)),
        ("ld_w", C.c_int64), ("ld_g", C.c_int64), ("ld_m", C.c_int64),
        ("w_shadow", C.POINTER(C.c_void_p)), ("ld_shadow", C.c_int64),
    ]


class muon_hparams(C.Structure):
    _fields_ = [
        ("lr", C.c_float), ("wd", C.c_float), ("mu", C.c_float),
        ("nesterov", C.c_int32), ("ns_steps", C.c_int32),
        ("a", C.c_float), ("b", C.c_float), ("c", C.c_float),
        ("eps", C.c_float), ("rms_scale", C.c_float),
        ("scale_mode", C.c_int32), ("scale_dim", C.c_float),
        ("coeffs", C.POINTER(C.c_float)), ("protect_momentum", C.c_int32),
    ]


class muon_adamw_tensor(C.Structure):
    _fields_ = [("p", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("numel", C.c_int64), ("p_dtype", C.c_int32), ("g_dtype", C.c_int32)]


class muon_adamw_hparams(C.Structure):
    _fields_ = [("lr", C.c_float), ("wd", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("eps", C.c_float), ("step", C.c_int32)]


class muon_head_args(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("dim", C.c_int32), ("vocab", C.c_int32), ("mean", C.c_int32),
                ("x", C.c_void_p), ("w", C.c_void_p), ("ld_x", C.c_int64), ("ld_w", C.c_int64),
                ("x_dtype", C.c_int32), ("w_dtype", C.c_int32), ("weight", C.c_void_p),
                ("scale", C.c_float), ("logit_scale", C.c_float),
                ("loss", C.c_void_p), ("lse", C.c_void_p), ("total", C.c_void_p),
                ("dx", C.c_void_p), ("dw", C.c_void_p), ("ld_dx", C.c_int64), ("ld_dw", C.c_int64),
                ("dx_dtype", C.c_int32), ("dw_dtype", C.c_int32), ("dw_accumulate", C.c_int32),
                ("reserved", C.c_int32)]


class muon_head_teacher(C.Structure):
    _fields_ = [("top_ids", C.c_void_p), ("top_logits", C.c_void_p), ("ld_ids", C.c_int64),
                ("ld_logits", C.c_int64), ("teacher_lse", C.c_void_p), ("top", C.c_int32),
                ("logits_dtype", C.c_int32), ("temperature", C.c_float), ("reserved", C.c_int32)]


class MuonError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("muon error %d: %s" % (code, msg))
        self.code = code


_lib = None


def lib():
    """Load libmuon_b200.so (once).  There is no fallback: a missing library
    is an error."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libmuon_b200.so is not built (%s); run `python -m paper_2502_16982_b200.build`" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    L.muon_workspace_bytes.argtypes = [C.POINTER(muon_group), C.c_int, C.POINTER(C.c_size_t)]
    L.muon_partition.argtypes = [C.POINTER(muon_group), C.c_int, C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_double)]
    L.muon_partition_slots.argtypes = [C.POINTER(muon_group), C.c_int, C.c_int, C.POINTER(C.c_int),
                                       C.POINTER(C.c_int), C.POINTER(C.c_int), C.POINTER(C.c_double)]
    L.muon_init.argtypes = [C.POINTER(C.c_void_p), C.POINTER(muon_group), C.c_int, C.c_void_p, C.c_size_t, C.c_int]
    L.muon_step.argtypes = [C.c_void_p, C.POINTER(muon_hparams), C.c_void_p]
    L.muon_plan_buckets.argtypes = [C.POINTER(muon_group), C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int)]
    L.muon_plan_flops.argtypes = [C.POINTER(muon_group), C.c_int, C.c_int, C.POINTER(C.c_double),
                                  C.POINTER(C.c_double)]
    L.muon_plan_work.argtypes = [C.POINTER(muon_group), C.c_int, C.c_int, C.POINTER(C.c_double),
                                 C.POINTER(C.c_double)]
    L.muon_debug_tile_table.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int16), C.c_int,
                                        C.POINTER(C.c_int), C.POINTER(C.c_int)]
    L.muon_step_bucket.argtypes = [C.c_void_p, C.POINTER(muon_hparams), C.c_int, C.c_void_p]
    L.muon_step_host.argtypes = [C.c_void_p, C.POINTER(muon_hparams), C.POINTER(C.POINTER(C.c_void_p)),
                                 C.POINTER(C.POINTER(C.c_void_p)), C.c_void_p]
    L.muon_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int), C.POINTER(C.c_int)]
    L.muon_get_norms.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_float), C.c_int]
    L.muon_get_update_rms.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_float), C.c_int]
    L.muon_destroy.argtypes = [C.c_void_p]
    L.muon_last_error.restype = C.c_char_p
    L.muon_last_launch_count.argtypes = [C.c_void_p]
    L.muon_debug_keep.argtypes = [C.c_void_p, C.c_int]
    L.muon_debug_read.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_size_t]
    L.muon_debug_tmem_bases.argtypes = [C.c_void_p, C.POINTER(C.c_uint), C.c_int]
    L.muon_profile_enable.argtypes = [C.c_void_p, C.c_int]
    L.muon_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_int)]
    L.muon_momentum_norm_static.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int64, C.c_int64,
                                            C.c_int, C.c_float, C.c_int, C.c_void_p, C.c_int, C.c_void_p]
    L.muon_debug_set_chunk_bytes.argtypes = [C.c_size_t]
    L.muon_debug_set_pair_fold.argtypes = [C.c_int]
    L.muon_debug_set_tile_mode.argtypes = [C.c_int]
    L.muon_debug_wait_expiry.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_uint]
    L.muon_adamw_step.argtypes = [C.POINTER(muon_adamw_tensor), C.c_int, C.POINTER(muon_adamw_hparams), C.c_int,
                                  C.c_void_p]
    L.muon_head_workspace_bytes.argtypes = [C.POINTER(muon_head_args), C.c_int, C.POINTER(C.c_size_t),
                                            C.POINTER(C.c_size_t)]
    L.muon_debug_set_head_piece_bytes.argtypes = [C.c_size_t]
    L.muon_debug_set_head_codes.argtypes = [C.c_int]
    L.muon_head_xent.argtypes = [C.POINTER(muon_head_args), C.c_void_p, C.c_float, C.c_void_p, C.c_size_t, C.c_int,
                                 C.c_void_p]
    L.muon_head_distill.argtypes = [C.POINTER(muon_head_args), C.POINTER(muon_head_teacher), C.c_void_p, C.c_size_t,
                                    C.c_int, C.c_void_p]
    L.muon_head_status.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.POINTER(C.c_int)]
    for name in EXPORTED:
        if name in ("muon_debug_set_chunk_bytes", "muon_debug_set_head_piece_bytes"):
            getattr(L, name).restype = C.c_size_t
        elif name != "muon_last_error":
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _check(rc):
    if rc != 0:
        raise MuonError(rc, lib().muon_last_error().decode())


def muon_last_error() -> str:
    return lib().muon_last_error().decode()


@dataclass
class Hyper:
    """Hyper-parameters of one step; defaults are the paper's."""
    lr: float = 2e-2
    wd: float = 0.1
    mu: float = 0.95
    nesterov: bool = True
    ns_steps: int = 5
    a: float = 3.4445
    b: float = -4.7750
    c: float = 2.0315
    eps: float = 1e-7
    rms_scale: float = 0.2
    scale_mode: int = MUON_SCALE_ADJUSTED_LR
    scale_dim: float = 0.0
    coeffs: Optional[Sequence] = None  # one (a, b, c) per Newton-Schulz step
    protect_momentum: bool = False  # a matrix with a non-finite gradient keeps its momentum too

    def to_c(self) -> muon_hparams:
        hp = muon_hparams(self.lr, self.wd, self.mu, int(bool(self.nesterov)), int(self.ns_steps),
                          self.a, self.b, self.c, self.eps, self.rms_scale, int(self.scale_mode),
                          float(self.scale_dim), None, int(bool(self.protect_momentum)))
        if self.coeffs is not None:
            flat = [float(v) for triple in self.coeffs for v in triple]
            if len(flat) != 3 * int(self.ns_steps):
                raise MuonError(MUON_ERR_INVALID_ARG, "coeffs must hold one (a, b, c) per Newton-Schulz step")
            self._coeffs_c = (C.c_float * len(flat))(*flat)  # kept alive by the Hyper object
            hp.coeffs = C.cast(self._coeffs_c, C.POINTER(C.c_float))
        return hp


_dtype_codes = {}


def _dtype_code(t):
    code = _dtype_codes.get(t.dtype)
    if code is not None:
        return code
    import torch
    _dtype_codes.update({torch.bfloat16: MUON_DTYPE_BF16, torch.float32: MUON_DTYPE_FP32})
    if t.dtype in _dtype_codes:
        return _dtype_codes[t.dtype]
    raise MuonError(MUON_ERR_UNSUPPORTED, "dtype %s" % t.dtype)


class _GroupArrays:
    """Keeps the ctypes arrays of one param group alive."""

    def __init__(self, ws, gs, ms, shadows=None):
        w0, g0, m0 = ws[0], gs[0], ms[0]
        n = len(ws)
        if shadows is not None:
            import torch
            for t in shadows:
                if t.shape != w0.shape or t.dtype != torch.bfloat16 or t.stride(1) != 1 or t.stride(0) != shadows[0].stride(0):
                    raise MuonError(MUON_ERR_INVALID_ARG, "shadow copies must be bf16, shaped like W, with one row stride")
        for t in list(ws) + list(gs) + list(ms):
            if t.dim() != 2 or t.shape != w0.shape or t.stride(1) != 1:
                raise MuonError(MUON_ERR_INVALID_ARG, "matrices of a group must be 2-D, equal-shaped, rows contiguous")
        for seq, ref in ((ws, w0), (gs, g0), (ms, m0)):
            for t in seq:
                if t.dtype != ref.dtype or t.stride(0) != ref.stride(0):
                    raise MuonError(MUON_ERR_INVALID_ARG, "dtype and row stride must be uniform within a group")
        self.w = (C.c_void_p * n)(*[t.data_ptr() for t in ws])
        self.g = (C.c_void_p * n)(*[t.data_ptr() for t in gs])
        self.m = (C.c_void_p * n)(*[t.data_ptr() for t in ms])
        self.desc = muon_group(
            w0.shape[0], w0.shape[1], n, _dtype_code(w0), _dtype_code(g0), 0,
            C.cast(self.w, C.POINTER(C.c_void_p)), C.cast(self.g, C.POINTER(C.c_void_p)),
            C.cast(self.m, C.POINTER(C.c_void_p)),
            w0.stride(0) if w0.shape[0] > 1 else max(w0.stride(0), w0.shape[1]),
            g0.stride(0) if g0.shape[0] > 1 else max(g0.stride(0), g0.shape[1]),
            m0.stride(0) if m0.shape[0] > 1 else max(m0.stride(0), m0.shape[1]),
            None, 0)
        if shadows is not None:
            s0 = shadows[0]
            self.s = (C.c_void_p * n)(*[t.data_ptr() for t in shadows])
            self.desc.w_shadow = C.cast(self.s, C.POINTER(C.c_void_p))
            self.desc.ld_shadow = s0.stride(0) if s0.shape[0] > 1 else max(s0.stride(0), s0.shape[1])


def shape_only_groups(shapes) -> "C.Array":
    """muon_group array carrying only (rows, cols, count, w_dtype, g_dtype)
    for muon_workspace_bytes."""
    arr = (muon_group * len(shapes))()
    for i, (rows, cols, count, wd, gd) in enumerate(shapes):
        arr[i].rows, arr[i].cols, arr[i].count, arr[i].w_dtype, arr[i].g_dtype = rows, cols, count, wd, gd
    return arr


def muon_workspace_bytes(groups_c, n_groups) -> int:
    out = C.c_size_t(0)
    _check(lib().muon_workspace_bytes(groups_c, n_groups, C.byref(out)))
    return out.value


def muon_momentum_norm_static(g, m, mu: float, nesterov: bool, norm_out, stream=None):
    """M <- mu*M + G in place and ``norm_out[0] = ||U||_F`` for one 2-D CUDA
    matrix, through the entry point that needs no workspace: the library's
    built-in scratch array is used, so nothing is allocated here either
    (``norm_out`` is a one-element fp32 CUDA tensor the caller already owns).
    Meant for callers that cannot get device memory of their own, e.g. because
    the framework's pool has reserved the whole GPU.  Calls on one GPU share
    the scratch: keep them on one stream."""
    import torch
    if g.dim() != 2 or m.shape != g.shape or g.stride(1) != 1 or m.stride(1) != 1:
        raise MuonError(MUON_ERR_INVALID_ARG, "g and m must be equal-shaped 2-D tensors with contiguous rows")
    if m.dtype != torch.float32 or norm_out.dtype != torch.float32:
        raise MuonError(MUON_ERR_INVALID_ARG, "m and norm_out must be fp32")
    dev = g.device.index
    s = torch.cuda.current_stream(dev) if stream is None else stream
    rows, cols = g.shape
    ld_g = g.stride(0) if rows > 1 else max(g.stride(0), cols)
    ld_m = m.stride(0) if rows > 1 else max(m.stride(0), cols)
    _check(lib().muon_momentum_norm_static(
        C.c_void_p(g.data_ptr()), C.c_void_p(m.data_ptr()), rows, cols, ld_g, ld_m, _dtype_code(g),
        float(mu), int(bool(nesterov)), C.c_void_p(norm_out.data_ptr()), dev, C.c_void_p(s.cuda_stream)))


def muon_adamw_step(params, grads, exp_avgs, exp_avg_sqs, step: int, lr: float, wd: float,
                    beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, stream=None):
    """AdamW step over lists of contiguous CUDA tensors (p bf16/fp32, g bf16/fp32,
    m and v fp32), in place; argument marshalling only."""
    import torch
    n = len(params)
    arr = (muon_adamw_tensor * n)()
    for i, (p, g, m, v) in enumerate(zip(params, grads, exp_avgs, exp_avg_sqs)):
        for t in (p, g, m, v):
            if not t.is_contiguous() or t.numel() != p.numel():
                raise MuonError(MUON_ERR_INVALID_ARG, "AdamW tensors must be contiguous and equally sized")
        if m.dtype != torch.float32 or v.dtype != torch.float32:
            raise MuonError(MUON_ERR_INVALID_ARG, "AdamW moments must be fp32")
        arr[i] = muon_adamw_tensor(p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr(), p.numel(),
                                   _dtype_code(p), _dtype_code(g))
    dev = params[0].device.index
    s = torch.cuda.current_stream(dev) if stream is None else stream
    hp = muon_adamw_hparams(lr, wd, beta1, beta2, eps, int(step))
    _check(lib().muon_adamw_step(arr, n, C.byref(hp), dev, C.c_void_p(s.cuda_stream)))


_no_context = contextlib.nullcontext()


class HeadLoss(NamedTuple):
    """What a head loss gives: per-token ``loss`` and ``lse`` (fp32), ``total`` (one
    fp32 element) and the gradients of ``total`` (None where not asked for)."""
    loss: "torch.Tensor"
    lse: "torch.Tensor"
    total: "torch.Tensor"
    dx: Optional["torch.Tensor"]
    dw: Optional["torch.Tensor"]


def _row_stride(t):
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])


_head_bytes = {}  # workspace bytes of a plan, by everything the plan depends on


def _raw_stream(stream, dev):
    import torch
    if stream is not None:
        return stream.cuda_stream
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # a tenth of the cost of building a Stream object
    return get(dev) if get is not None else torch.cuda.current_stream(dev).cuda_stream


def _past_32_bits():
    raise MuonError(MUON_ERR_UNSUPPORTED, "a size past 32 bits")  # ctypes would keep its low 32 bits


def _head_vector(t, what, n, dev):
    import torch
    if t is None:
        return torch.empty(n, dtype=torch.float32, device=dev)
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous() or t.device != dev:
        raise MuonError(MUON_ERR_INVALID_ARG, "%s must be %d contiguous fp32 values on x's device" % (what, n))
    return t


def _head_matrix(t, what, shape, dev):
    if t.shape != shape or (shape[1] > 1 and t.stride(1) != 1) or t.device != dev:
        raise MuonError(MUON_ERR_INVALID_ARG, "%s must be shaped like its tensor, with contiguous rows, on x's device" % what)
    return t


def _head_call(x, w, top, loss, lse, total, dx, dw, weight, mean, scale, logit_scale, accumulate_dw, workspace, stream,
               least_workspace, call):
    """Checks, outputs and workspace shared by the head losses; ``call(args,
    workspace address, bytes, device, stream)`` makes the C call."""
    import torch
    if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1] or x.shape[1] < 1 or w.shape[0] < 1:
        raise MuonError(MUON_ERR_INVALID_ARG, "x must be [tokens, dim] and w [vocab, dim]")
    (tokens, dim), vocab = x.shape, w.shape[0]
    if (tokens | dim | vocab | top) >> 31:
        _past_32_bits()
    dev = x.device
    if dev.type != "cuda" or w.device != dev:
        raise MuonError(MUON_ERR_INVALID_ARG, "x and w must be on one CUDA device")
    if dim > 1 and (x.stride(1) != 1 or w.stride(1) != 1):
        raise MuonError(MUON_ERR_INVALID_ARG, "x and w must have contiguous rows")
    if accumulate_dw and not isinstance(dw, torch.Tensor):
        raise MuonError(MUON_ERR_INVALID_ARG, "accumulate_dw needs the dw to add to")
    empty = torch.empty
    # allocated for the stream the kernels run on
    with torch.cuda.stream(stream) if stream is not None else _no_context:
        if loss is None and lse is None and total is None:
            loss, lse, total = empty(2 * tokens + 1, dtype=torch.float32, device=dev).split_with_sizes((tokens, tokens, 1))
        else:
            loss = _head_vector(loss, "loss", tokens, dev)
            lse = _head_vector(lse, "lse", tokens, dev)
            total = _head_vector(total, "total", 1, dev)
        if dx is False:
            dx = None
        elif dx is not None:
            dx = torch.empty_like(x) if dx is True else _head_matrix(dx, "dx", x.shape, dev)
        if dw is False:
            dw = None
        elif dw is not None:
            dw = torch.empty_like(w) if dw is True else _head_matrix(dw, "dw", w.shape, dev)
        ld_w, w_ptr = _row_stride(w), w.data_ptr()
        a = muon_head_args(tokens, dim, vocab, 1 if mean else 0, x.data_ptr(), w_ptr, _row_stride(x) if tokens else dim, ld_w,
                           _dtype_code(x), _dtype_code(w),
                           None if weight is None else _head_vector(weight, "weight", tokens, dev).data_ptr(), scale,
                           logit_scale, loss.data_ptr(), lse.data_ptr(), total.data_ptr())
        if dx is not None:
            a.dx, a.ld_dx, a.dx_dtype = dx.data_ptr(), _row_stride(dx) if tokens else dim, _dtype_code(dx)
        if dw is not None:
            a.dw, a.ld_dw, a.dw_dtype, a.dw_accumulate = dw.data_ptr(), _row_stride(dw), _dtype_code(dw), 1 if accumulate_dw else 0
        if workspace is None:
            key = (tokens, dim, vocab, top, dx is None, dw is None, ld_w & 7, w_ptr & 15, least_workspace)
            need = _head_bytes.get(key)
            if need is None:
                out = C.c_size_t(0)
                _check(lib().muon_head_workspace_bytes(C.byref(a), top, None if least_workspace else C.byref(out),
                                                       C.byref(out) if least_workspace else None))
                if len(_head_bytes) >= 1024:
                    _head_bytes.clear()
                need = _head_bytes[key] = out.value + 1024
            workspace = empty(need, dtype=torch.uint8, device=dev)
        elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != dev:
            raise MuonError(MUON_ERR_WORKSPACE, "workspace must be a contiguous uint8 tensor on x's device")
    first = workspace.data_ptr()
    base = (first + 1023) // 1024 * 1024
    _check(call(C.byref(a), base, max(first + workspace.numel() - base, 0), dev.index, _raw_stream(stream, dev.index)))
    return HeadLoss(loss, lse, total, dx, dw)


def muon_head_workspace_bytes(tokens: int, dim: int, vocab: int, top: int = 0, dx: bool = True, dw: bool = True,
                              packed_head: bool = True, least: bool = False) -> int:
    """Workspace bytes of one head-loss call (``top``: teacher entries per token, 0
    for cross entropy), 1024 for aligning a tensor's start included.  ``least``: the
    smallest workspace a call accepts instead of the one it makes full use of.
    ``packed_head``: the head's rows are 16-byte aligned."""
    if any(C.c_int32(v).value != v for v in (tokens, dim, vocab, top)):
        _past_32_bits()
    ld = (dim + 7) // 8 * 8 if packed_head else dim | 1
    a = muon_head_args(tokens, dim, vocab, 1, None, None, dim, ld, MUON_DTYPE_BF16, MUON_DTYPE_BF16)
    a.dx, a.dw = (1024 if dx else None), (1024 if dw else None)  # only whether they are there counts
    out, low = C.c_size_t(0), C.c_size_t(0)
    _check(lib().muon_head_workspace_bytes(C.byref(a), int(top), C.byref(out), C.byref(low)))
    return (low if least else out).value + 1024


def muon_debug_set_head_piece_bytes(nbytes: int) -> int:
    _head_bytes.clear()
    return lib().muon_debug_set_head_piece_bytes(int(nbytes))


def muon_debug_set_head_codes(mode: int) -> int:
    _head_bytes.clear()
    return lib().muon_debug_set_head_codes(int(mode))


def muon_head_xent(x, w, targets, loss=None, lse=None, total=None, dx=None, dw=None, weight=None, mean=True,
                   scale=1.0, logit_scale=1.0, z_loss=0.0, accumulate_dw=False, workspace=None, stream=None,
                   least_workspace=False) -> HeadLoss:
    """Softmax cross entropy of ``x w^T`` over the vocabulary, with its gradients.
    ``x`` [tokens, dim] and ``w`` [vocab, dim] are bf16, ``targets`` int64 [tokens]
    (outside [0, vocab): the token is masked).
    ``dx`` / ``dw``: a bf16 or fp32 tensor to write, True to allocate one like x / w,
    None to leave the gradient out.  Other outputs and the workspace are allocated
    unless given; a workspace of :func:`muon_head_workspace_bytes` that is kept can be
    asked for the call's status.  By default a workspace with room for up to 3 GiB of
    logits as 16-bit codes is allocated, for speed; ``least_workspace``: the smallest
    that does, with one piece of the vocabulary's logits at a time.  Argument
    marshalling only; the formulas are in include/muon.h.
    Tensors used on another stream than the one they were allocated on are the
    caller's to keep alive (``record_stream``)."""
    import torch
    if targets.dtype != torch.int64 or targets.dim() != 1 or targets.shape[0] != x.shape[0] or not targets.is_contiguous() or targets.device != x.device:
        raise MuonError(MUON_ERR_INVALID_ARG, "targets must be contiguous int64 [tokens] on x's device")

    def call(a, ws, nbytes, dev, s):
        return lib().muon_head_xent(a, targets.data_ptr(), z_loss, ws, nbytes, dev, s)

    return _head_call(x, w, 0, loss, lse, total, dx, dw, weight, mean, scale, logit_scale, accumulate_dw, workspace,
                      stream, bool(least_workspace), call)


def muon_head_distill(x, w, top_ids, top_logits, temperature=1.0, teacher_lse=None, loss=None, lse=None, total=None,
                      dx=None, dw=None, weight=None, mean=True, scale=1.0, logit_scale=1.0, accumulate_dw=False,
                      workspace=None, stream=None, least_workspace=False) -> HeadLoss:
    """Distillation from a teacher's top logits: ``top_ids`` int64 and ``top_logits``
    bf16 or fp32, both [tokens, top], ``teacher_lse`` fp32 [tokens] or None.
    Everything else as :func:`muon_head_xent`."""
    import torch
    for t, what in ((top_ids, "top_ids"), (top_logits, "top_logits")):
        if t.dim() != 2 or t.shape != top_ids.shape or t.shape[0] != x.shape[0] or t.device != x.device or (t.shape[1] > 1 and t.stride(1) != 1):
            raise MuonError(MUON_ERR_INVALID_ARG, "%s must be [tokens, top] on x's device, rows contiguous" % what)
    if top_ids.dtype != torch.int64:
        raise MuonError(MUON_ERR_INVALID_ARG, "top_ids must be int64")
    if teacher_lse is not None and (teacher_lse.dtype != torch.float32 or teacher_lse.dim() != 1 or teacher_lse.numel() != x.shape[0]
                                    or not teacher_lse.is_contiguous() or teacher_lse.device != x.device):
        raise MuonError(MUON_ERR_INVALID_ARG, "teacher_lse must be contiguous fp32 [tokens] on x's device")
    top = top_ids.shape[1]
    if top < 1:
        raise MuonError(MUON_ERR_INVALID_ARG, "at least one teacher entry per token")
    t = muon_head_teacher(top_ids.data_ptr(), top_logits.data_ptr(), _row_stride(top_ids) if x.shape[0] else top,
                          _row_stride(top_logits) if x.shape[0] else top,
                          None if teacher_lse is None else teacher_lse.data_ptr(), top, _dtype_code(top_logits),
                          float(temperature), 0)

    def call(a, ws, nbytes, dev, s):
        return lib().muon_head_distill(a, C.byref(t), ws, nbytes, dev, s)

    return _head_call(x, w, top, loss, lse, total, dx, dw, weight, mean, scale, logit_scale, accumulate_dw, workspace,
                      stream, bool(least_workspace), call)


def muon_head_status(workspace, stream=None) -> int:
    """Synchronises the stream; 0, or MUON_ERR_TIMEOUT if a device-side wait of the
    last head-loss call that was given this workspace tensor expired."""
    import torch
    s = torch.cuda.current_stream(workspace.device) if stream is None else stream
    st = C.c_int(0)
    _check(lib().muon_head_status(C.c_void_p((workspace.data_ptr() + 1023) // 1024 * 1024), workspace.device.index,
                                  C.c_void_p(s.cuda_stream), C.byref(st)))
    return st.value


def muon_partition(shapes, world: int):
    """Owner rank of every matrix for `world` data-parallel ranks.  ``shapes``
    is a list of (rows, cols, count); returns (owners, loads)."""
    arr = shape_only_groups([(r, c, n, MUON_DTYPE_BF16, MUON_DTYPE_BF16) for (r, c, n) in shapes])
    total = sum(n for (_, _, n) in shapes)
    owners = (C.c_int * total)()
    loads = (C.c_double * world)()
    _check(lib().muon_partition(arr, len(shapes), int(world), owners, loads))
    return list(owners), list(loads)


def muon_partition_slots(shapes, world: int):
    """Slot partition for in-place collectives.  ``shapes`` is a list of (rows,
    cols, count, w_dtype code, g_dtype code); returns (owner per matrix, position
    in the owner's slot per matrix, slot capacity per bucket, load per rank)."""
    arr = shape_only_groups(shapes)
    total = sum(sh[2] for sh in shapes)
    _, n_buckets = muon_plan_buckets(shapes)
    owners = (C.c_int * total)()
    pos = (C.c_int * total)()
    share = (C.c_int * n_buckets)()
    loads = (C.c_double * world)()
    _check(lib().muon_partition_slots(arr, len(shapes), int(world), owners, pos, share, loads))
    return list(owners), list(pos), list(share), list(loads)


def muon_plan_flops(shapes, ns_steps: int = 5):
    """(algorithmic, planned) Newton-Schulz FLOPs of one step; ``shapes`` is a
    list of (rows, cols, count)."""
    arr = shape_only_groups([(r, c, n, MUON_DTYPE_BF16, MUON_DTYPE_BF16) for (r, c, n) in shapes])
    alg, planned = C.c_double(0), C.c_double(0)
    _check(lib().muon_plan_flops(arr, len(shapes), int(ns_steps), C.byref(alg), C.byref(planned)))
    return alg.value, planned.value


def muon_plan_work(shapes, ns_steps: int = 5):
    """({kind: planned FLOPs}, {kind: executed FLOPs}) of one step per kernel
    kind; ``shapes`` is a list of (rows, cols, count).  Executed counts whole
    tiles: padding and dropped blocks included."""
    arr = shape_only_groups([(r, c, n, MUON_DTYPE_BF16, MUON_DTYPE_BF16) for (r, c, n) in shapes])
    planned = (C.c_double * len(KERNEL_KINDS))()
    executed = (C.c_double * len(KERNEL_KINDS))()
    _check(lib().muon_plan_work(arr, len(shapes), int(ns_steps), planned, executed))
    return ({k: planned[i] for i, k in enumerate(KERNEL_KINDS)},
            {k: executed[i] for i, k in enumerate(KERNEL_KINDS)})


def muon_debug_tile_table(rows: int, cols: int, which: int, count: int = 4096):
    """(tiles, matrices per unit) of a bucket of ``count`` matrices (few small
    matrices are cut into finer tiles): every tile is a dict with the row blocks
    ``i`` and matrices ``dm`` of the two CTAs, the column blocks ``j`` of the
    two accumulator halves, the width ``nbw`` and the ``keep`` masks."""
    n, unit = C.c_int(0), C.c_int(0)
    _check(lib().muon_debug_tile_table(rows, cols, count, which, None, 0, C.byref(n), C.byref(unit)))
    buf = (C.c_int16 * (10 * max(1, n.value)))()
    _check(lib().muon_debug_tile_table(rows, cols, count, which, buf, n.value, C.byref(n), C.byref(unit)))
    tiles = []
    for k in range(n.value):
        v = buf[10 * k:10 * k + 10]
        tiles.append({"i": (v[0], v[1]), "j": (v[2], v[3]), "nbw": v[4], "dm": (v[5], v[6]), "keep": (v[7], v[8]),
                      "half": v[9]})
    return tiles, unit.value


def muon_debug_set_tile_mode(mode: int) -> int:
    """How tiles are cut where row blocks do not pair up (bit 0: half-height
    tiles for a row block without a partner, bit 1: for lone diagonal blocks of
    symmetric products; default 1).  Returns the previous mode."""
    return lib().muon_debug_set_tile_mode(int(mode))


def muon_debug_set_pair_fold(mode: int) -> int:
    """Where two iterations are taken per pass over X: 0 = the first two, by
    shape (default), 1 = never, 2 = the first two whenever the short side is at
    least 16, 3 = every pair for wide matrices, 4 = every pair whenever the
    short side is at least 16.  Returns the previous mode."""
    return lib().muon_debug_set_pair_fold(int(mode))


def muon_plan_buckets(shapes):
    """Bucket of every matrix.  ``shapes`` is a list of (rows, cols, count,
    w_dtype code, g_dtype code); returns (bucket per matrix, number of buckets)."""
    arr = shape_only_groups(shapes)
    total = sum(sh[2] for sh in shapes)
    out = (C.c_int * total)()
    n = C.c_int(0)
    _check(lib().muon_plan_buckets(arr, len(shapes), out, C.byref(n)))
    return list(out), n.value


def muon_debug_set_chunk_bytes(nbytes: int) -> int:
    """Test knob: bound on the Newton-Schulz operand bytes of one bucket chunk
    (0 = default).  Returns the previous value."""
    return lib().muon_debug_set_chunk_bytes(int(nbytes))


class MuonContext:
    """One initialised set of param groups.

    ``groups`` is a list of (weights, grads, momenta) triples, or
    (weights, grads, momenta, shadows) with bf16 copies of fp32 weights; each
    entry is a list of equal-shaped 2-D CUDA tensors (bf16 or fp32 weights and
    gradients, fp32 momenta).  Tensors must outlive the context.
    """

    def __init__(self, groups: Sequence[Sequence[Sequence["torch.Tensor"]]], device: Optional[int] = None,
                 workspace: Optional["torch.Tensor"] = None):
        """``workspace``: an optional uint8 CUDA tensor to carve the library's
        workspace from (at least ``muon_workspace_bytes`` + 1023 bytes, so that a
        1024-byte aligned start fits); by default one is allocated here."""
        import torch
        if not torch.cuda.is_available():
            raise MuonError(MUON_ERR_CUDA, "no CUDA device: this library has no CPU path")
        L = lib()
        self._arrays: List[_GroupArrays] = [_GroupArrays(*g) for g in groups]
        self._tensors = groups
        n = len(self._arrays)
        self._groups_c = (muon_group * n)(*[a.desc for a in self._arrays])
        self.n_groups = n
        self.n_matrices = sum(a.desc.count for a in self._arrays)
        dev = groups[0][0][0].device
        self.device = dev.index if device is None else device
        nbytes = muon_workspace_bytes(self._groups_c, n)
        self.workspace_bytes = nbytes
        if workspace is None:
            workspace = torch.empty(nbytes + 1024, dtype=torch.uint8, device=dev)
        elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != dev:
            raise MuonError(MUON_ERR_WORKSPACE, "workspace must be a contiguous uint8 tensor on the matrices' device")
        self.workspace = workspace
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 1023) // 1024 * 1024
        if self._ws_ptr + nbytes > base + workspace.numel():
            raise MuonError(MUON_ERR_WORKSPACE, "workspace too small: need %d bytes after alignment" % nbytes)
        ctx = C.c_void_p()
        _check(L.muon_init(C.byref(ctx), self._groups_c, n, C.c_void_p(self._ws_ptr), nbytes, self.device))
        self._ctx = ctx

    # -- the C calls -------------------------------------------------------
    def muon_step(self, hp: Hyper, stream=None):
        import torch
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        c_hp = hp.to_c()
        _check(lib().muon_step(self._ctx, C.byref(c_hp), C.c_void_p(s.cuda_stream)))

    def muon_step_bucket(self, hp: Hyper, bucket: int, stream=None):
        import torch
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        c_hp = hp.to_c()
        _check(lib().muon_step_bucket(self._ctx, C.byref(c_hp), int(bucket), C.c_void_p(s.cuda_stream)))

    def muon_step_host(self, hp: Hyper, g_host, w_host=None, stream=None):
        """g_host / w_host: per group, a list of pinned CPU tensors (dense)."""
        import torch
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        c_hp = hp.to_c()

        def table(host):
            rows = [(C.c_void_p * len(ts))(*[t.data_ptr() for t in ts]) for ts in host]
            tab = (C.POINTER(C.c_void_p) * len(rows))(*[C.cast(r, C.POINTER(C.c_void_p)) for r in rows])
            return rows, tab

        g_rows, g_tab = table(g_host)
        w_tab = None
        if w_host is not None:
            w_rows, w_tab = table(w_host)
        _check(lib().muon_step_host(self._ctx, C.byref(c_hp), g_tab, w_tab, C.c_void_p(s.cuda_stream)))

    def muon_status(self, stream=None):
        """Synchronises the stream; returns (status_code, matrix_index)."""
        import torch
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        st, mi = C.c_int(0), C.c_int(-1)
        _check(lib().muon_status(self._ctx, C.c_void_p(s.cuda_stream), C.byref(st), C.byref(mi)))
        return st.value, mi.value

    def muon_get_norms(self, stream=None):
        import torch
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        out = (C.c_float * self.n_matrices)()
        _check(lib().muon_get_norms(self._ctx, C.c_void_p(s.cuda_stream), out, self.n_matrices))
        return list(out)

    def muon_get_update_rms(self, stream=None):
        import torch
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        out = (C.c_float * self.n_matrices)()
        _check(lib().muon_get_update_rms(self._ctx, C.c_void_p(s.cuda_stream), out, self.n_matrices))
        return list(out)

    def muon_last_launch_count(self) -> int:
        return lib().muon_last_launch_count(self._ctx)

    def muon_profile_enable(self, enable: bool):
        _check(lib().muon_profile_enable(self._ctx, int(enable)))

    def muon_profile_read(self):
        """Returns {kernel kind: (milliseconds, launches)} since the last read."""
        n = len(KERNEL_KINDS)
        ms = (C.c_double * n)()
        cnt = (C.c_int * n)()
        _check(lib().muon_profile_read(self._ctx, ms, cnt))
        return {k: (ms[i], cnt[i]) for i, k in enumerate(KERNEL_KINDS)}

    def muon_debug_tmem_bases(self, n: int = 296):
        out = (C.c_uint * n)()
        _check(lib().muon_debug_tmem_bases(self._ctx, out, n))
        return list(out)

    def muon_debug_wait_expiry(self, matrix_index: int, limit_ms: int = 20, stream=None):
        import torch
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        _check(lib().muon_debug_wait_expiry(self._ctx, C.c_void_p(s.cuda_stream), int(matrix_index), int(limit_ms)))

    def muon_debug_keep(self, keep: bool):
        _check(lib().muon_debug_keep(self._ctx, int(keep)))

    def muon_debug_read(self, matrix_index: int, which: int, rows: int, cols: int):
        """Returns a CPU bf16 tensor rows x cols (short side first)."""
        import torch
        out = torch.empty((rows, cols), dtype=torch.bfloat16)
        _check(lib().muon_debug_read(self._ctx, matrix_index, which, C.c_void_p(out.data_ptr()), out.numel() * 2))
        return out

    def muon_destroy(self):
        if getattr(self, "_ctx", None) is not None and self._ctx:
            lib().muon_destroy(self._ctx)
            self._ctx = None

    def __del__(self):
        try:
            self.muon_destroy()
        except Exception:
            pass

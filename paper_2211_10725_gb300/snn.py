"""ctypes binding of libsnn (include/snn.h).

The functions named like the C entry points marshal torch tensors into
device pointers and call the library; every step of the scan runs in the
library's CUDA kernels.  PyTorch only allocates memory and supplies the
current stream.  If the library is missing the binding raises: there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import functools
import os
import re
import struct
from typing import Optional

import torch

from . import workloads as W

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "_lib", "libsnn.so")
HEADER = os.path.join(os.path.dirname(_PKG), "include", "snn.h")

SNN_OK = 0
STATUS_NAMES = {0: "SNN_OK", 1: "SNN_ERR_INVALID_ARG", 2: "SNN_ERR_ALIGNMENT",
                3: "SNN_ERR_UNSUPPORTED", 4: "SNN_ERR_WORKSPACE", 5: "SNN_ERR_CUDA",
                6: "SNN_ERR_TIMEOUT"}
DTYPE_CODE = {W.F32: 0, W.BF16: 1, W.F16: 2}
_TORCH_DTYPE_CODE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
GATE_CODE = {"none": 0, "sigmoid": 1, "silu": 2}
RESET_CODE = {"subtract": 0, "zero": 1, "none": 2}
SG_CODE = {"fast_sigmoid": 0, "atan": 1}
PMODE_CODE = {"scalar": 0, "per_neuron": 1, "per_channel": 2}
SAVE_CODE = {"mem": 0, "recompute": 1}
DEBUG_PRODUCER_IDLE = 1
DEBUG_FORCE_PLAIN = 2
DEBUG_NO_SEGMENT = 4


class SnnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}")


class ScanDesc(ctypes.Structure):
    """Mirror of snn_scan_desc."""
    _fields_ = [
        ("T", ctypes.c_int64), ("B", ctypes.c_int64), ("N", ctypes.c_int64),
        ("C", ctypes.c_int64), ("HW", ctypes.c_int64),
        ("in_dtype", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
        ("reset", ctypes.c_int32), ("detach_reset", ctypes.c_int32),
        ("surrogate", ctypes.c_int32), ("sg_param", ctypes.c_float),
        ("beta_mode", ctypes.c_int32), ("thr_mode", ctypes.c_int32),
        ("alpha_mode", ctypes.c_int32), ("save", ctypes.c_int32),
        ("ckpt_every", ctypes.c_int32), ("reserved0", ctypes.c_int32),
        ("wait_limit_ns", ctypes.c_int64), ("debug_flags", ctypes.c_uint32),
        ("reserved1", ctypes.c_uint32),
    ]


class AttnDesc(ctypes.Structure):
    """Mirror of snn_attn_desc."""
    _fields_ = [
        ("B", ctypes.c_int64), ("T", ctypes.c_int64), ("H", ctypes.c_int64),
        ("Hk", ctypes.c_int64), ("Dk", ctypes.c_int64), ("Dv", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_uint32 * 2),
    ]


class Bthd(ctypes.Structure):
    """Mirror of snn_bthd."""
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64),
                ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class NormDesc(ctypes.Structure):
    """Mirror of snn_norm_desc."""
    _fields_ = [
        ("M", ctypes.c_int64), ("N", ctypes.c_int64), ("group", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("res_dtype", ctypes.c_int32), ("gate", ctypes.c_int32),
        ("eps", ctypes.c_float), ("reserved", ctypes.c_uint32 * 2),
    ]


class Rows(ctypes.Structure):
    """Mirror of snn_rows."""
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64)]


class SscanDesc(ctypes.Structure):
    """Mirror of snn_sscan_desc."""
    _fields_ = [
        ("B", ctypes.c_int64), ("T", ctypes.c_int64), ("D", ctypes.c_int64),
        ("N", ctypes.c_int64), ("G", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("softplus", ctypes.c_int32), ("reserved", ctypes.c_uint32 * 2),
    ]


class ConvDesc(ctypes.Structure):
    """Mirror of snn_conv_desc."""
    _fields_ = [
        ("B", ctypes.c_int64), ("T", ctypes.c_int64), ("C", ctypes.c_int64), ("W", ctypes.c_int64),
        ("dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("reserved", ctypes.c_uint32 * 2),
    ]


class LayerNormDesc(ctypes.Structure):
    """Mirror of snn_layer_norm_desc."""
    _fields_ = [
        ("M", ctypes.c_int64), ("N", ctypes.c_int64), ("dtype", ctypes.c_int32),
        ("res_dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("reserved", ctypes.c_uint32),
    ]


class Btc(ctypes.Structure):
    """Mirror of snn_btc."""
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_t", ctypes.c_int64)]


_P = ctypes.c_void_p
_SIGS = {
    "snn_status_string": ([ctypes.c_int], ctypes.c_char_p),
    "snn_version": ([], ctypes.c_int),
    "snn_scan_desc_size": ([], ctypes.c_size_t),
    "snn_scan_workspace_bytes": ([ctypes.POINTER(ScanDesc)], ctypes.c_size_t),
    "snn_scan_ckpt_elems": ([ctypes.POINTER(ScanDesc), ctypes.c_int], ctypes.c_int64),
    "snn_workspace_init": ([_P, ctypes.c_size_t, _P], ctypes.c_int),
    "snn_workspace_status": ([_P, _P], ctypes.c_int),
    "snn_leaky_fwd": ([ctypes.POINTER(ScanDesc)] + [_P] * 9 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_leaky_bwd": ([ctypes.POINTER(ScanDesc)] + [_P] * 15 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_synaptic_fwd": ([ctypes.POINTER(ScanDesc)] + [_P] * 13 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_synaptic_bwd": ([ctypes.POINTER(ScanDesc)] + [_P] * 21 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_leaky_bwd_noalloc": ([ctypes.POINTER(ScanDesc)] + [_P] * 16, ctypes.c_int),
    "snn_rleaky_fwd": ([ctypes.POINTER(ScanDesc)] + [_P] * 10 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_rleaky_bwd": ([ctypes.POINTER(ScanDesc)] + [_P] * 17 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_dense_layer_fwd": ([ctypes.c_int64] * 3 + [_P] * 4 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_dense_workspace_bytes": ([ctypes.c_int64] * 3, ctypes.c_size_t),
    "snn_dense_layer_bwd": ([ctypes.c_int64] * 3 + [_P] * 6 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_rate_ce_workspace_bytes": ([ctypes.c_int64], ctypes.c_size_t),
    "snn_kernel_launches": ([], ctypes.c_uint64),
    "snn_dense_leaky_bwd": ([ctypes.POINTER(ScanDesc), ctypes.c_int64] + [_P] * 9
                            + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_dense_leaky_fwd": ([ctypes.POINTER(ScanDesc), ctypes.c_int64, ctypes.c_int64] + [_P] * 8
                            + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_conv2d_small_fwd_nhwc": ([ctypes.c_int64] * 8 + [_P] * 4, ctypes.c_int),
    "snn_conv2d_small_dw_workspace_bytes": ([ctypes.c_int64] * 7, ctypes.c_size_t),
    "snn_conv2d_small_dw_nhwc": ([ctypes.c_int64] * 8 + [_P] * 4 + [ctypes.c_size_t, _P],
                                 ctypes.c_int),
    "snn_im2col_nhwc": ([ctypes.c_int64] * 7 + [_P] * 3, ctypes.c_int),
    "snn_col2im_nhwc": ([ctypes.c_int64] * 7 + [_P] * 3, ctypes.c_int),
    "snn_maxpool2_fwd_nhwc": ([ctypes.c_int64] * 4 + [_P] * 4, ctypes.c_int),
    "snn_maxpool2_bwd_nhwc": ([ctypes.c_int64] * 4 + [_P] * 4, ctypes.c_int),
    "snn_rate_ce_loss": ([ctypes.c_int64] * 6 + [ctypes.c_int32] + [_P] * 5 + [ctypes.c_size_t, _P],
                         ctypes.c_int),
    "snn_rate_ce_leaky_bwd": ([ctypes.POINTER(ScanDesc)] + [ctypes.c_int64] * 3 + [_P] * 10
                              + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_attn_desc_size": ([], ctypes.c_size_t),
    "snn_leaky_attn_workspace_bytes": ([_P, ctypes.c_int], ctypes.c_size_t),
    "snn_leaky_attn_fwd": ([_P] * 9 + [ctypes.c_int64] + [_P] * 2 + [ctypes.c_size_t, _P],
                           ctypes.c_int),
    "snn_leaky_attn_bwd": ([_P] * 14 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_leaky_attn_step": ([_P] * 7 + [ctypes.c_int64, _P, _P], ctypes.c_int),
    "snn_norm_desc_size": ([], ctypes.c_size_t),
    "snn_block_norm_workspace_bytes": ([ctypes.c_int64] * 2, ctypes.c_size_t),
    "snn_block_norm_fwd": ([_P] * 10, ctypes.c_int),
    "snn_block_norm_bwd": ([_P] * 16 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_sscan_desc_size": ([], ctypes.c_size_t),
    "snn_selective_scan_workspace_bytes": ([_P, ctypes.c_int], ctypes.c_size_t),
    "snn_selective_scan_ckpt_elems": ([_P], ctypes.c_int64),
    "snn_selective_scan_fwd": ([_P] * 13 + [ctypes.c_int64] + [_P] * 3 + [ctypes.c_size_t, _P],
                               ctypes.c_int),
    "snn_selective_scan_bwd": ([_P] * 23 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_selective_scan_step": ([_P] * 11 + [ctypes.c_int64] + [_P] * 2, ctypes.c_int),
    "snn_conv_desc_size": ([], ctypes.c_size_t),
    "snn_causal_conv_workspace_bytes": ([_P], ctypes.c_size_t),
    "snn_causal_conv_fwd": ([_P] * 8 + [ctypes.c_int64] + [_P] * 2, ctypes.c_int),
    "snn_causal_conv_bwd": ([_P] * 13 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_causal_conv_step": ([_P] * 6 + [ctypes.c_int64] + [_P] * 2, ctypes.c_int),
    "snn_layer_norm_desc_size": ([], ctypes.c_size_t),
    "snn_layer_norm_workspace_bytes": ([ctypes.c_int64] * 2, ctypes.c_size_t),
    "snn_layer_norm_fwd": ([_P] * 7, ctypes.c_int),
    "snn_layer_norm_bwd": ([_P] * 9 + [ctypes.c_size_t, _P], ctypes.c_int),
    "snn_adamw_step": ([ctypes.c_int64] + [_P] * 5 + [ctypes.c_float] * 5 + [ctypes.c_int64] +
                       [_P, _P], ctypes.c_int),
}

_lib: Optional[ctypes.CDLL] = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libsnn.so (built by paper_2211_10725_gb300.build_lib); raise if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"libsnn.so not built ({path}); run __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    for name, (args, res) in _SIGS.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def header_functions(path: str = HEADER) -> list:
    """Names of the functions include/snn.h declares."""
    txt = open(path).read()
    txt = re.sub(r"/\*.*?\*/", "", txt, flags=re.S)
    return sorted(set(re.findall(r"\b(snn_[a-z0-9_]+)\s*\(", txt)))


def status_string(status: int) -> str:
    return load_library().snn_status_string(status).decode()


def _check(status: int, where: str):
    if status != SNN_OK:
        raise SnnError(status, where)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# handle of a device's current stream, without the Stream object around it
# (building one costs more than a small kernel takes)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream, device=None) -> Optional[int]:
    if stream is None:  # the current device's (`device`, where that is known)
        return _raw_stream(torch.cuda.current_device() if device is None else device.index)
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_desc(w: W.ScanWorkload, **over) -> ScanDesc:
    """Descriptor for a workload (fields can be overridden by keyword)."""
    d = ScanDesc()
    d.T, d.B, d.N, d.C, d.HW = w.T, w.B, w.N, w.C, w.HW
    d.in_dtype, d.io_dtype = DTYPE_CODE[w.in_dtype], DTYPE_CODE[w.io_dtype]
    d.reset = RESET_CODE[w.reset]
    d.detach_reset = 1 if w.detach_reset else 0
    d.surrogate = SG_CODE[w.surrogate]
    d.sg_param = w.sg_param
    d.beta_mode, d.thr_mode = PMODE_CODE[w.beta_mode], PMODE_CODE[w.thr_mode]
    d.alpha_mode = PMODE_CODE[w.v_mode if w.neuron == "rleaky" else w.alpha_mode]
    d.save = SAVE_CODE[w.save]
    d.ckpt_every = w.ckpt_every if w.save == "recompute" else 0
    for k, v in over.items():
        setattr(d, k, v)
    return d


# ---------------------------------------------------------------------------
# Thin wrappers with the C names (tensor -> pointer marshalling only)
# ---------------------------------------------------------------------------

def snn_scan_workspace_bytes(desc: ScanDesc) -> int:
    return load_library().snn_scan_workspace_bytes(ctypes.byref(desc))


def snn_scan_ckpt_elems(desc: ScanDesc, synaptic: bool) -> int:
    return load_library().snn_scan_ckpt_elems(ctypes.byref(desc), 1 if synaptic else 0)


def snn_workspace_init(ws: torch.Tensor, stream=None):
    _check(load_library().snn_workspace_init(_ptr(ws), ws.numel() * ws.element_size(),
                                             _stream(stream)), "snn_workspace_init")


def snn_workspace_status(ws: torch.Tensor, stream=None) -> int:
    return load_library().snn_workspace_status(_ptr(ws), _stream(stream))


def snn_leaky_fwd(desc, I, beta, thr, mem0, spk, mem, ckpt, mem_final, ws, stream=None):
    _check(load_library().snn_leaky_fwd(
        ctypes.byref(desc), _ptr(I), _ptr(beta), _ptr(thr), _ptr(mem0), _ptr(spk), _ptr(mem),
        _ptr(ckpt), _ptr(mem_final), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)), "snn_leaky_fwd")


def snn_leaky_bwd(desc, I, ckpt, mem, spk, beta, thr, mem0, grad_spk, grad_mem,
                  grad_mem_final, grad_I, grad_beta, grad_thr, grad_mem0, ws, stream=None):
    _check(load_library().snn_leaky_bwd(
        ctypes.byref(desc), _ptr(I), _ptr(ckpt), _ptr(mem), _ptr(spk), _ptr(beta), _ptr(thr),
        _ptr(mem0), _ptr(grad_spk), _ptr(grad_mem), _ptr(grad_mem_final), _ptr(grad_I),
        _ptr(grad_beta), _ptr(grad_thr), _ptr(grad_mem0), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)), "snn_leaky_bwd")


def snn_synaptic_fwd(desc, I, alpha, beta, thr, mem0, syn0, spk, mem, syn, ckpt, mem_final,
                     syn_final, ws, stream=None):
    _check(load_library().snn_synaptic_fwd(
        ctypes.byref(desc), _ptr(I), _ptr(alpha), _ptr(beta), _ptr(thr), _ptr(mem0),
        _ptr(syn0), _ptr(spk), _ptr(mem), _ptr(syn), _ptr(ckpt), _ptr(mem_final),
        _ptr(syn_final), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
        "snn_synaptic_fwd")


def snn_synaptic_bwd(desc, I, ckpt, mem, spk, syn, alpha, beta, thr, mem0, syn0, grad_spk,
                     grad_mem, grad_mem_final, grad_syn_final, grad_I, grad_alpha, grad_beta,
                     grad_thr, grad_mem0, grad_syn0, ws, stream=None):
    _check(load_library().snn_synaptic_bwd(
        ctypes.byref(desc), _ptr(I), _ptr(ckpt), _ptr(mem), _ptr(spk), _ptr(syn), _ptr(alpha),
        _ptr(beta), _ptr(thr), _ptr(mem0), _ptr(syn0), _ptr(grad_spk), _ptr(grad_mem),
        _ptr(grad_mem_final), _ptr(grad_syn_final), _ptr(grad_I), _ptr(grad_alpha),
        _ptr(grad_beta), _ptr(grad_thr), _ptr(grad_mem0), _ptr(grad_syn0), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)), "snn_synaptic_bwd")


def snn_rleaky_fwd(desc, I, v, beta, thr, mem0, spk, mem, ckpt, mem_final, ws, stream=None):
    _check(load_library().snn_rleaky_fwd(
        ctypes.byref(desc), _ptr(I), _ptr(v), _ptr(beta), _ptr(thr), _ptr(mem0), _ptr(spk),
        _ptr(mem), _ptr(ckpt), _ptr(mem_final), _ptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)), "snn_rleaky_fwd")


def snn_rleaky_bwd(desc, I, ckpt, mem, spk, v, beta, thr, mem0, grad_spk, grad_mem,
                   grad_mem_final, grad_I, grad_v, grad_beta, grad_thr, grad_mem0, ws,
                   stream=None):
    _check(load_library().snn_rleaky_bwd(
        ctypes.byref(desc), _ptr(I), _ptr(ckpt), _ptr(mem), _ptr(spk), _ptr(v), _ptr(beta),
        _ptr(thr), _ptr(mem0), _ptr(grad_spk), _ptr(grad_mem), _ptr(grad_mem_final),
        _ptr(grad_I), _ptr(grad_v), _ptr(grad_beta), _ptr(grad_thr), _ptr(grad_mem0), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)), "snn_rleaky_bwd")


def snn_leaky_bwd_noalloc(desc, I, ckpt, mem, spk, beta, thr, mem0, grad_spk, grad_mem,
                          grad_mem_final, grad_I, grad_beta, grad_thr, grad_mem0, status=None,
                          stream=None):
    """Leaky BPTT using the library's fixed device scratch instead of a
    workspace, for callers that cannot allocate device memory."""
    _check(load_library().snn_leaky_bwd_noalloc(
        ctypes.byref(desc), _ptr(I), _ptr(ckpt), _ptr(mem), _ptr(spk), _ptr(beta), _ptr(thr),
        _ptr(mem0), _ptr(grad_spk), _ptr(grad_mem), _ptr(grad_mem_final), _ptr(grad_I),
        _ptr(grad_beta), _ptr(grad_thr), _ptr(grad_mem0), _ptr(status), _stream(stream)),
        "snn_leaky_bwd_noalloc")


def snn_dense_workspace_bytes(M: int, K: int, N: int) -> int:
    return load_library().snn_dense_workspace_bytes(M, K, N)


def snn_dense_layer_fwd(X, W, I, ws, stream=None):
    """I[M, N] = X[M, K] @ W[N, K]^T on the tensor cores (bf16 in, fp32 out)."""
    M, K = X.shape[-2], X.shape[-1]
    N = W.shape[0]
    _check(load_library().snn_dense_layer_fwd(M, K, N, _ptr(X), _ptr(W), _ptr(I), _ptr(ws),
                                              ws.numel() * ws.element_size(), _stream(stream)),
           "snn_dense_layer_fwd")


def snn_dense_layer_bwd(X, W, dI, dX, dW, ws, stream=None):
    """dX = dI @ W (bf16) and dW = dI^T @ X (fp32); either output may be None."""
    M, K = X.shape[-2], X.shape[-1]
    N = W.shape[0]
    _check(load_library().snn_dense_layer_bwd(M, K, N, _ptr(X), _ptr(W), _ptr(dI), _ptr(dX),
                                              _ptr(dW), _ptr(ws), ws.numel() * ws.element_size(),
                                              _stream(stream)), "snn_dense_layer_bwd")


class SideStream:
    """A second stream for launches off a training step's critical path (the
    weight-gradient products, which nothing waits on until the optimiser):
    fork() queues a call on it behind the work already queued on the main
    stream, join() makes the main stream wait for every call forked since the
    last join.  Both are event records and waits, so a captured CUDA graph
    holds them as fork and join edges."""

    def __init__(self, device=None):
        self.stream = torch.cuda.Stream(device)
        self._done = []

    def fork(self, main, call):
        """call(stream) on the side stream, after main's queued work."""
        main = torch.cuda.current_stream() if main is None else main
        ready = torch.cuda.Event()
        ready.record(main)
        self.stream.wait_event(ready)
        call(self.stream)
        done = torch.cuda.Event()
        done.record(self.stream)
        self._done.append(done)

    def join(self, main):
        main = torch.cuda.current_stream() if main is None else main
        for done in self._done:
            main.wait_event(done)
        self._done = []


def dense_layer_bwd_split(X, W, dI, dX, dW, ws, stream=None, side: Optional[SideStream] = None):
    """snn_dense_layer_bwd with, given a side stream, the weight gradient
    forked onto it (issued first, so it runs beside the input gradient,
    which the rest of the reverse pass waits on)."""
    if side is None or dW is None:
        snn_dense_layer_bwd(X, W, dI, dX, dW, ws, stream)
        return
    side.fork(stream, lambda st: snn_dense_layer_bwd(X, W, dI, None, dW, ws, st))
    if dX is not None:
        snn_dense_layer_bwd(X, W, dI, dX, None, ws, stream)


def snn_rate_ce_workspace_bytes(B: int) -> int:
    return load_library().snn_rate_ce_workspace_bytes(B)


def snn_rate_ce_loss(spk, labels, C, loss, grad_spk, ws=None, stream=None, batch_total=None,
                     pop=1):
    """Cross-entropy on output spike counts; spk/grad_spk [T, B, ld], C
    classes of pop neurons each.  The mean is over batch_total samples
    (default B: this batch).  ws: a zeroed uint8 device tensor of
    snn_rate_ce_workspace_bytes(B) bytes (a fresh one when None)."""
    T, B, ld = spk.shape
    dt = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[spk.dtype]
    if ws is None:
        ws = torch.zeros(snn_rate_ce_workspace_bytes(B), dtype=torch.uint8, device=spk.device)
    _check(load_library().snn_rate_ce_loss(T, B, C, pop, ld, batch_total or 0, dt, _ptr(spk),
                                           _ptr(labels), _ptr(loss), _ptr(grad_spk), _ptr(ws),
                                           ws.numel() * ws.element_size(), _stream(stream)),
           "snn_rate_ce_loss")


def snn_rate_ce_leaky_bwd(desc, spk, labels, C, beta, thr, mem, ckpt, loss, grad_spk, grad_I,
                          ws, stream=None, batch_total=None, pop=1):
    """snn_rate_ce_loss with the readout layer's BPTT in the same launch:
    writes loss, grad_I [T, B, ld] and (unless None) grad_spk.  ckpt: the
    forward's spike bits, or None to take the spike decisions from spk."""
    _check(load_library().snn_rate_ce_leaky_bwd(ctypes.byref(desc), C, pop, batch_total or 0,
                                                _ptr(spk), _ptr(labels), _ptr(beta), _ptr(thr),
                                                _ptr(mem), _ptr(ckpt), _ptr(loss), _ptr(grad_spk),
                                                _ptr(grad_I), _ptr(ws),
                                                ws.numel() * ws.element_size(), _stream(stream)),
           "snn_rate_ce_leaky_bwd")


def snn_adamw_step(w, w_bf16, grad, m, v, lr, beta1=0.9, beta2=0.999, eps=1e-8,
                   weight_decay=1e-2, step=1, step_counter=None, stream=None):
    """AdamW update in place of fp32 w, m, v from grad (same numel); writes
    the bf16 copy of the new weights to w_bf16 unless it is None.  With a
    device int64 [2] step_counter the step number is read from (and advanced
    on) the device instead of taken from ``step``."""
    n = w.numel()
    for t in (grad, m, v) + ((w_bf16,) if w_bf16 is not None else ()):
        if t.numel() != n:
            raise ValueError("snn_adamw_step: tensors differ in size")
    _check(load_library().snn_adamw_step(n, _ptr(w), _ptr(w_bf16), _ptr(grad), _ptr(m), _ptr(v),
                                         lr, beta1, beta2, eps, weight_decay, step,
                                         _ptr(step_counter), _stream(stream)), "snn_adamw_step")


def snn_dense_leaky_fwd(desc, X, W, beta, thr, spk, mem, ckpt, ws, P=1, stream=None):
    """GEMM of X [T*B*P, K] with W [Nout, K] and the Leaky scan of its
    currents in one kernel; writes spk, mem (and the spike bits to ckpt)."""
    K = X.shape[-1]
    _check(load_library().snn_dense_leaky_fwd(ctypes.byref(desc), P, K, _ptr(X), _ptr(W),
                                              _ptr(beta), _ptr(thr), _ptr(spk), _ptr(mem),
                                              _ptr(ckpt), _ptr(ws), ws.numel() * ws.element_size(),
                                              _stream(stream)), "snn_dense_leaky_fwd")


def snn_dense_leaky_bwd(desc, dI_up, W, beta, thr, mem, spk, ckpt, grad_I, ws, stream=None):
    """dX = dI_up [T*B, K] @ W [K, N] on the tensor cores, and the Leaky BPTT
    of the layer below on it in the same kernel; writes that layer's grad_I."""
    K = dI_up.shape[-1]
    _check(load_library().snn_dense_leaky_bwd(ctypes.byref(desc), K, _ptr(dI_up), _ptr(W),
                                              _ptr(beta), _ptr(thr), _ptr(mem), _ptr(spk),
                                              _ptr(ckpt), _ptr(grad_I), _ptr(ws),
                                              ws.numel() * ws.element_size(), _stream(stream)),
           "snn_dense_leaky_bwd")


def snn_kernel_launches() -> int:
    """Kernels the library has launched (or captured) in this process."""
    return int(load_library().snn_kernel_launches())


def snn_conv2d_small_fwd_nhwc(X, Wt, I, KH, KW, stream=None):
    """I [M, Ho, Wo, Cout] fp32 = X [M, H, W, Cin] (*) filters Wt [Cout, ldw]
    on the CUDA cores (few input channels)."""
    M, H, W_, Cin = X.shape
    Cout, ldw = Wt.shape
    _check(load_library().snn_conv2d_small_fwd_nhwc(M, H, W_, Cin, Cout, KH, KW, ldw, _ptr(X),
                                                    _ptr(Wt), _ptr(I), _stream(stream)),
           "snn_conv2d_small_fwd_nhwc")


def snn_conv2d_small_dw_workspace_bytes(M, H, W_, Cin, Cout, KH, KW) -> int:
    return load_library().snn_conv2d_small_dw_workspace_bytes(M, H, W_, Cin, Cout, KH, KW)


def snn_conv2d_small_dw_nhwc(X, dI, dW, KH, KW, ws, stream=None):
    """dW [Cout, ldw] fp32 of snn_conv2d_small_fwd_nhwc from dI [M, Ho, Wo, Cout] bf16."""
    M, H, W_, Cin = X.shape
    Cout, ldw = dW.shape
    _check(load_library().snn_conv2d_small_dw_nhwc(M, H, W_, Cin, Cout, KH, KW, ldw, _ptr(X),
                                                   _ptr(dI), _ptr(dW), _ptr(ws),
                                                   ws.numel() * ws.element_size(),
                                                   _stream(stream)), "snn_conv2d_small_dw_nhwc")


def snn_im2col_nhwc(X, cols, KH, KW, stream=None):
    """Patch rows of channel-last X [M, H, W, Cin] into cols [M*Ho*Wo, Kpad]."""
    M, H, W_, Cin = X.shape
    _check(load_library().snn_im2col_nhwc(M, H, W_, Cin, KH, KW, cols.shape[-1], _ptr(X),
                                          _ptr(cols), _stream(stream)), "snn_im2col_nhwc")


def snn_col2im_nhwc(dcols, dX, KH, KW, stream=None):
    """Patch-row gradient dcols [M*Ho*Wo, Kpad] summed onto dX [M, H, W, Cin]."""
    M, H, W_, Cin = dX.shape
    _check(load_library().snn_col2im_nhwc(M, H, W_, Cin, KH, KW, dcols.shape[-1], _ptr(dcols),
                                          _ptr(dX), _stream(stream)), "snn_col2im_nhwc")


def snn_maxpool2_fwd_nhwc(X, Y, idx, stream=None):
    M, H, W_, C = X.shape
    _check(load_library().snn_maxpool2_fwd_nhwc(M, H, W_, C, _ptr(X), _ptr(Y), _ptr(idx),
                                                _stream(stream)), "snn_maxpool2_fwd_nhwc")


def snn_maxpool2_bwd_nhwc(dY, idx, dX, stream=None):
    M, H, W_, C = dX.shape
    _check(load_library().snn_maxpool2_bwd_nhwc(M, H, W_, C, _ptr(dY), _ptr(idx), _ptr(dX),
                                                _stream(stream)), "snn_maxpool2_bwd_nhwc")


@functools.lru_cache(maxsize=1024)
def _attn_desc(where, B, T, H, Hk, Dk, Dv, dtype, scale) -> AttnDesc:
    code = _TORCH_DTYPE_CODE.get(dtype)
    if code is None:
        raise ValueError(f"{where}: dtype {dtype}")
    return AttnDesc(B, T, H, Hk, Dk, Dv, code, scale)


def _bthd(where, name, t, shape, dtype):
    """The words of snn_bthd for a [B, T, heads, D] tensor (a [B, heads, D] one
    for a single token) with contiguous D."""
    if t.shape != shape or t.dtype != dtype or not t.is_cuda:
        raise ValueError(f"{where}: {name} must be a CUDA {dtype} tensor of shape {shape}")
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{where}: {name} must have a contiguous last dimension")
    return t.data_ptr(), st[0], st[1], st[-2]


def _rows(where, name, t, shape, dtype):
    """The words of snn_rows for an [M, N] matrix with contiguous rows, or for None."""
    if t is None:
        return 0, 0
    if t.shape != shape or t.dtype != dtype or not t.is_cuda:
        raise ValueError(f"{where}: {name} must be a CUDA {dtype} tensor of shape {shape}")
    ld, inner = t.stride()
    if inner != 1 and shape[1] > 1:
        raise ValueError(f"{where}: {name} must have contiguous rows")
    return t.data_ptr(), ld


# A call's snn_bthd or snn_rows structures (a pointer and 64-bit strides) lie in
# one array; the addresses of the structures in it.  (Packed first: filling a
# ctypes array element by element takes four times as long.)
_WORDS = {n: (struct.Struct(f"{n}q"), ctypes.c_int64 * n) for n in (10, 16, 28)}


def _places(words, each):
    pack, array = _WORDS[len(words)]
    array = array.from_buffer_copy(pack.pack(*words))
    at = ctypes.addressof(array)
    return array, range(at, at + 8 * len(words), 8 * each)


def _flat(where, name, t, shape, dtype):
    """Pointer of a contiguous tensor of the given shape and type, or None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{where}: {name} must be a contiguous CUDA {dtype} tensor of shape {shape}")
    return t.data_ptr()


@functools.lru_cache(maxsize=1024)
def snn_leaky_attn_workspace_bytes(B, T, H, Hk, Dk, Dv, backward=False) -> int:
    d = AttnDesc(B, T, H, Hk, Dk, Dv, 1, 1.0)
    return load_library().snn_leaky_attn_workspace_bytes(ctypes.byref(d), 1 if backward else 0)


def _state_places(where, slots, B, states):
    """(slots pointer, number of places) of the fp32 [places, H, Dk, Dv] states."""
    places = [s.shape[0] for s in states if s is not None]
    n = places[0] if places else B
    if slots is None:
        if n != B:
            raise ValueError(f"{where}: without slots the states have one place per sequence")
        return None, n
    return _flat(where, "slots", slots, (B,), torch.int32), n


def snn_leaky_attn_fwd(q, k, v, beta, o, ws, scale=1.0, seq_lens=None, state_in=None,
                       state_out=None, slots=None, stream=None):
    """Leaky attention over whole sequences, S_t = beta_h S_{t-1} + k_t v_t^T and
    o_t = scale S_t^T q_t: q [B, T, H, Dk], k [B, T, Hk, Dk], v [B, T, Hk, Dv],
    o [B, T, H, Dv] (bf16 or fp16, any strides with contiguous D), beta fp32
    [H].  seq_lens int32 [B]; state_in and state_out fp32 [places, H, Dk, Dv]
    with slots int32 [B] naming each sequence's place (default b; outside the
    range: no state).  ws: snn_leaky_attn_workspace_bytes of the shape."""
    w = "snn_leaky_attn_fwd"
    (B, T, H, Dk), Hk, Dv, dt = q.shape, k.shape[2], v.shape[-1], q.dtype
    d = _attn_desc(w, B, T, H, Hk, Dk, Dv, dt, float(scale))
    if state_in is not None and state_out is not None and len(state_in) != len(state_out):
        raise ValueError(f"{w}: state_in and state_out differ in places")
    ps, n = _state_places(w, slots, B, (state_in, state_out))
    array, (pq, pk, pv, po) = _places(
        _bthd(w, "q", q, (B, T, H, Dk), dt) + _bthd(w, "k", k, (B, T, Hk, Dk), dt)
        + _bthd(w, "v", v, (B, T, Hk, Dv), dt) + _bthd(w, "o", o, (B, T, H, Dv), dt), 4)
    _check(load_library().snn_leaky_attn_fwd(
        ctypes.byref(d), pq, pk, pv, _flat(w, "beta", beta, (H,), torch.float32),
        _flat(w, "seq_lens", seq_lens, (B,), torch.int32),
        _flat(w, "state_in", state_in, (n, H, Dk, Dv), torch.float32),
        _flat(w, "state_out", state_out, (n, H, Dk, Dv), torch.float32), ps, n, po, _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)), w)


def snn_leaky_attn_bwd(q, k, v, beta, grad_o, grad_q, grad_k, grad_v, ws, scale=1.0,
                       seq_lens=None, state_in=None, grad_state_out=None, grad_state_in=None,
                       stream=None):
    """Gradients of snn_leaky_attn_fwd (states [B, H, Dk, Dv], in sequence
    order); ws: snn_leaky_attn_workspace_bytes(..., backward=True)."""
    w = "snn_leaky_attn_bwd"
    (B, T, H, Dk), Hk, Dv, dt = q.shape, k.shape[2], v.shape[-1], q.dtype
    d = _attn_desc(w, B, T, H, Hk, Dk, Dv, dt, float(scale))
    qs, ks, vs, os = (B, T, H, Dk), (B, T, Hk, Dk), (B, T, Hk, Dv), (B, T, H, Dv)
    array, (pq, pk, pv, po, gq, gk, gv) = _places(
        _bthd(w, "q", q, qs, dt) + _bthd(w, "k", k, ks, dt) + _bthd(w, "v", v, vs, dt)
        + _bthd(w, "grad_o", grad_o, os, dt) + _bthd(w, "grad_q", grad_q, qs, dt)
        + _bthd(w, "grad_k", grad_k, ks, dt) + _bthd(w, "grad_v", grad_v, vs, dt), 4)
    state = lambda name, t: _flat(w, name, t, (B, H, Dk, Dv), torch.float32)
    _check(load_library().snn_leaky_attn_bwd(
        ctypes.byref(d), pq, pk, pv, _flat(w, "beta", beta, (H,), torch.float32),
        _flat(w, "seq_lens", seq_lens, (B,), torch.int32), state("state_in", state_in), po,
        state("grad_state_out", grad_state_out), gq, gk, gv, state("grad_state_in", grad_state_in),
        _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), w)


def snn_leaky_attn_step(q, k, v, beta, state, o, scale=1.0, slots=None, stream=None):
    """One token of each sequence (decoding): q [B, H, Dk], k [B, Hk, Dk],
    v [B, Hk, Dv], o [B, H, Dv]; state fp32 [places, H, Dk, Dv] is updated in
    place at slots (int32 [B]; default b; outside the range: an empty place of
    the batch, whose o is zero)."""
    w = "snn_leaky_attn_step"
    (B, H, Dk), Hk, Dv, dt = q.shape, k.shape[1], v.shape[-1], q.dtype
    d = _attn_desc(w, B, 1, H, Hk, Dk, Dv, dt, float(scale))
    n = state.shape[0]
    array, (pq, pk, pv, po) = _places(
        _bthd(w, "q", q, (B, H, Dk), dt) + _bthd(w, "k", k, (B, Hk, Dk), dt)
        + _bthd(w, "v", v, (B, Hk, Dv), dt) + _bthd(w, "o", o, (B, H, Dv), dt), 4)
    _check(load_library().snn_leaky_attn_step(
        ctypes.byref(d), pq, pk, pv, _flat(w, "beta", beta, (H,), torch.float32),
        _flat(w, "state", state, (n, H, Dk, Dv), torch.float32),
        _flat(w, "slots", slots, (B,), torch.int32), n, po, _stream(stream)), w)


@functools.lru_cache(maxsize=1024)
def snn_block_norm_workspace_bytes(M: int, N: int) -> int:
    return load_library().snn_block_norm_workspace_bytes(M, N)


@functools.lru_cache(maxsize=1024)
def _norm_desc(where, M, N, group, dtype, res_dtype, gate, eps) -> NormDesc:
    for dt in (dtype, res_dtype):
        if dt not in _TORCH_DTYPE_CODE:
            raise ValueError(f"{where}: dtype {dt}")
    if gate not in GATE_CODE:
        raise ValueError(f"{where}: gate {gate!r}")
    return NormDesc(M, N, group, _TORCH_DTYPE_CODE[dtype], _TORCH_DTYPE_CODE[res_dtype],
                    GATE_CODE[gate], eps)


def snn_block_norm_fwd(r, a, z, w_post, res_scale, w_pre, r_out, y, eps=1e-6, group=0,
                       gate="none", stream=None):
    """r_out = r + res_scale * norm(a) w_post * act(z) and y = norm(r_out)
    w_pre over the rows of [M, N] matrices (rows any stride apart).  a None:
    y = norm(r) w_pre alone; w_pre None: no y.  group: channels per norm of a
    (0: the row); gate: "none", "sigmoid" or "silu" of z."""
    w = "snn_block_norm_fwd"
    shape, res = r.shape, r.dtype
    io = a.dtype if a is not None else y.dtype if y is not None else res
    d = _norm_desc(w, *shape, int(group), io, res, gate, float(eps))
    array, (pr, pa, pz, po, py) = _places(
        _rows(w, "r", r, shape, res) + _rows(w, "a", a, shape, io) + _rows(w, "z", z, shape, io)
        + _rows(w, "r_out", r_out, shape, res) + _rows(w, "y", y, shape, io), 2)
    n = shape[1:]
    _check(load_library().snn_block_norm_fwd(
        ctypes.byref(d), pr, pa, pz, _flat(w, "w_post", w_post, n, torch.float32),
        _flat(w, "res_scale", res_scale, n, torch.float32),
        _flat(w, "w_pre", w_pre, n, torch.float32), po, py, _stream(stream)), w)


def snn_block_norm_bwd(r_out, a, z, w_post, res_scale, w_pre, grad_r_out, grad_y, grad_r, grad_a,
                       grad_z, grad_w_post, grad_scale, grad_w_pre, ws, eps=1e-6, group=0,
                       gate="none", stream=None):
    """Gradients of snn_block_norm_fwd from its stored r_out; grad_r_out or
    grad_y None stands for zeros, an output None is not computed.  ws:
    snn_block_norm_workspace_bytes(M, N) (None without parameter gradients)."""
    w = "snn_block_norm_bwd"
    of = r_out if r_out is not None else grad_r_out
    shape, res = of.shape, of.dtype
    io = a.dtype if a is not None else grad_y.dtype if grad_y is not None else res
    d = _norm_desc(w, *shape, int(group), io, res, gate, float(eps))
    array, (pr, pa, pz, gro, gy, gr, ga, gz) = _places(
        _rows(w, "r_out", r_out, shape, res) + _rows(w, "a", a, shape, io)
        + _rows(w, "z", z, shape, io) + _rows(w, "grad_r_out", grad_r_out, shape, res)
        + _rows(w, "grad_y", grad_y, shape, io) + _rows(w, "grad_r", grad_r, shape, res)
        + _rows(w, "grad_a", grad_a, shape, io) + _rows(w, "grad_z", grad_z, shape, io), 2)
    n = shape[1:]
    par = lambda name, t: _flat(w, name, t, n, torch.float32)
    _check(load_library().snn_block_norm_bwd(
        ctypes.byref(d), pr, pa, pz, par("w_post", w_post), par("res_scale", res_scale),
        par("w_pre", w_pre), gro, gy, gr, ga, gz, par("grad_w_post", grad_w_post),
        par("grad_scale", grad_scale), par("grad_w_pre", grad_w_pre), _ptr(ws),
        ws.numel() * ws.element_size() if ws is not None else 0, _stream(stream)), w)


# Tensors of the selective scan, the causal convolution and the layer norm: all on one
# device, which has to be the current one (its stream takes the launches).

def _device(where, t):
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"{where}: tensors must be on the current CUDA device, not {t.device}")
    return t.device


def _refuse(where, name, t, shape, dtype, device, last):
    """Why a tensor was refused (`last`: of the layout)."""
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise ValueError(f"{where}: {name} must be a {dtype} tensor of shape {shape} on {device}")
    raise ValueError(f"{where}: {name} must {last}")


# The checks stand in each function, not in one of their own: a call per tensor is
# a tenth of a small kernel's way through here.

def _btc(where, name, t, shape, dtype, device):
    """The words of snn_btc for a [B, T, C] tensor (a [B, C] one for a single
    token) with contiguous C, or for None."""
    if t is None:
        return 0, 0, 0
    st = t.stride()
    if t.shape != shape or t.dtype != dtype or t.device != device or (st[-1] != 1 and shape[-1] > 1):
        _refuse(where, name, t, shape, dtype, device, "have a contiguous last dimension")
    return t.data_ptr(), st[0], st[-2]


def _btgn(where, name, t, shape, dtype, device):
    """The words of snn_bthd for a [B, T, G, N] tensor (a [B, G, N] one for a single
    token) with contiguous N."""
    st = t.stride()
    if t.shape != shape or t.dtype != dtype or t.device != device or (st[-1] != 1 and shape[-1] > 1):
        _refuse(where, name, t, shape, dtype, device, "have a contiguous last dimension")
    return t.data_ptr(), st[0], st[1], st[-2]


def _whole(where, name, t, shape, dtype, device):
    """Pointer of a contiguous tensor, or None."""
    if t is None:
        return None
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        _refuse(where, name, t, shape, dtype, device, "be contiguous")
    return t.data_ptr()


@functools.lru_cache(maxsize=64)
def _layout(sizes):
    """(pack, array type, offsets) of structures of these many 64-bit words."""
    n, at = sum(sizes), [0]
    for k in sizes[:-1]:
        at.append(at[-1] + 8 * k)
    return struct.Struct(f"{n}q").pack, ctypes.c_int64 * n, tuple(at)


def _structs(*parts):
    """The parts' words in one array, and the address of each part (None for an
    absent tensor)."""
    pack, array, offsets = _layout(tuple(map(len, parts)))
    array = array.from_buffer_copy(pack(*[w for p in parts for w in p]))
    base = ctypes.addressof(array)
    return array, [base + o if p[0] else None for o, p in zip(offsets, parts)]


def _ws(where, ws, device):
    """(pointer, bytes) of a workspace, or of None."""
    if ws is None:
        return None, 0
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"{where}: ws must be a contiguous tensor on {device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


@functools.lru_cache(maxsize=1024)
def _sscan_desc(where, B, T, D, N, G, dtype, softplus):
    code = _TORCH_DTYPE_CODE.get(dtype)
    if code is None:
        raise ValueError(f"{where}: dtype {dtype}")
    d = SscanDesc(B, T, D, N, G, code, 1 if softplus else 0)
    return d, ctypes.addressof(d)


def _places_of(where, slots, B, states, device):
    """(slots pointer, number of places) of states whose first dimension is the places."""
    places = [s.shape[0] for s in states if s is not None]
    n = places[0] if places else B
    if any(p != n for p in places):
        raise ValueError(f"{where}: the states differ in places")
    if slots is None:
        if n != B:
            raise ValueError(f"{where}: without slots the states have one place per sequence")
        return None, n
    return _whole(where, "slots", slots, (B,), torch.int32, device), n


@functools.lru_cache(maxsize=1024)
def snn_selective_scan_workspace_bytes(B, T, D, N, G=1, backward=False) -> int:
    d = SscanDesc(B, T, D, N, G)
    return load_library().snn_selective_scan_workspace_bytes(ctypes.byref(d), 1 if backward else 0)


@functools.lru_cache(maxsize=1024)
def snn_selective_scan_ckpt_elems(B, T, D, N, G=1) -> int:
    d = SscanDesc(B, T, D, N, G)
    return load_library().snn_selective_scan_ckpt_elems(ctypes.byref(d))


def snn_selective_scan_fwd(u, delta, A, B, C, y, ws, D=None, z=None, delta_bias=None, softplus=True,
                           seq_lens=None, state_in=None, state_out=None, slots=None, ckpt=None,
                           stream=None):
    """Selective scan over whole sequences, s = softplus(delta + delta_bias), h_t =
    exp(s A) h_{t-1} + s u B and y = (C h + D u) silu(z): u, delta, z, y [B, T, D] and
    B, C [B, T, G, N] of one type (fp32, bf16 or fp16, any strides with a contiguous
    last dimension); A [D, N], D and delta_bias [D], states [places, D, N] fp32.
    seq_lens and slots: int32 [B].  ws: snn_selective_scan_workspace_bytes of the shape;
    ckpt: fp32, snn_selective_scan_ckpt_elems of the shape, for the backward."""
    w = "snn_selective_scan_fwd"
    dev, (nB, T, nD), (N, G), dt = _device(w, u), u.shape, (A.shape[-1], B.shape[2]), u.dtype
    _, d = _sscan_desc(w, nB, T, nD, N, G, dt, bool(softplus))
    ps, n = _places_of(w, slots, nB, (state_in, state_out), dev)
    seq, grp, f32 = (nB, T, nD), (nB, T, G, N), torch.float32
    keep, (pu, pd, pB, pC, pz, py) = _structs(
        _btc(w, "u", u, seq, dt, dev), _btc(w, "delta", delta, seq, dt, dev),
        _btgn(w, "B", B, grp, dt, dev), _btgn(w, "C", C, grp, dt, dev), _btc(w, "z", z, seq, dt, dev),
        _btc(w, "y", y, seq, dt, dev))
    if ckpt is not None and ckpt.numel() < snn_selective_scan_ckpt_elems(nB, T, nD, N, G):
        raise ValueError(f"{w}: ckpt is smaller than snn_selective_scan_ckpt_elems")
    pw, nw = _ws(w, ws, dev)
    _check(load_library().snn_selective_scan_fwd(
        d, pu, pd, _whole(w, "A", A, (nD, N), f32, dev), pB, pC, _whole(w, "D", D, (nD,), f32, dev), pz,
        _whole(w, "delta_bias", delta_bias, (nD,), f32, dev),
        _whole(w, "seq_lens", seq_lens, (nB,), torch.int32, dev),
        _whole(w, "state_in", state_in, (n, nD, N), f32, dev),
        _whole(w, "state_out", state_out, (n, nD, N), f32, dev), ps, n,
        None if ckpt is None else _whole(w, "ckpt", ckpt, ckpt.shape, f32, dev), py, pw, nw,
        _stream(stream, dev)), w)


def snn_selective_scan_bwd(u, delta, A, B, C, grad_y, ckpt, grad_u, grad_delta, grad_A, grad_B, grad_C,
                           ws, D=None, z=None, delta_bias=None, softplus=True, seq_lens=None,
                           grad_state_out=None, grad_D=None, grad_z=None, grad_delta_bias=None,
                           grad_state_in=None, stream=None):
    """Gradients of snn_selective_scan_fwd from the checkpoints that it left (states
    [B, D, N], in sequence order); grad_z is given exactly when z is.  ws:
    snn_selective_scan_workspace_bytes(..., backward=True)."""
    w = "snn_selective_scan_bwd"
    dev, (nB, T, nD), (N, G), dt = _device(w, u), u.shape, (A.shape[-1], B.shape[2]), u.dtype
    _, d = _sscan_desc(w, nB, T, nD, N, G, dt, bool(softplus))
    seq, grp, f32 = (nB, T, nD), (nB, T, G, N), torch.float32
    keep, (pu, pd, pB, pC, pz, pgy, pgu, pgd, pgB, pgC, pgz) = _structs(
        _btc(w, "u", u, seq, dt, dev), _btc(w, "delta", delta, seq, dt, dev),
        _btgn(w, "B", B, grp, dt, dev), _btgn(w, "C", C, grp, dt, dev), _btc(w, "z", z, seq, dt, dev),
        _btc(w, "grad_y", grad_y, seq, dt, dev), _btc(w, "grad_u", grad_u, seq, dt, dev),
        _btc(w, "grad_delta", grad_delta, seq, dt, dev), _btgn(w, "grad_B", grad_B, grp, dt, dev),
        _btgn(w, "grad_C", grad_C, grp, dt, dev), _btc(w, "grad_z", grad_z, seq, dt, dev))
    if ckpt.numel() < snn_selective_scan_ckpt_elems(nB, T, nD, N, G):
        raise ValueError(f"{w}: ckpt is smaller than snn_selective_scan_ckpt_elems")
    flat = lambda name, t, shape: _whole(w, name, t, shape, f32, dev)
    pw, nw = _ws(w, ws, dev)
    _check(load_library().snn_selective_scan_bwd(
        d, pu, pd, flat("A", A, (nD, N)), pB, pC, flat("D", D, (nD,)), pz,
        flat("delta_bias", delta_bias, (nD,)), _whole(w, "seq_lens", seq_lens, (nB,), torch.int32, dev),
        flat("ckpt", ckpt, ckpt.shape), pgy, flat("grad_state_out", grad_state_out, (nB, nD, N)), pgu, pgd,
        flat("grad_A", grad_A, (nD, N)), pgB, pgC, flat("grad_D", grad_D, (nD,)), pgz,
        flat("grad_delta_bias", grad_delta_bias, (nD,)),
        flat("grad_state_in", grad_state_in, (nB, nD, N)), pw, nw, _stream(stream, dev)), w)


def snn_selective_scan_step(u, delta, A, B, C, state, y, D=None, z=None, delta_bias=None, softplus=True,
                            slots=None, stream=None):
    """One token of each sequence (decoding): u, delta, z, y [B, D], B and C [B, G, N];
    state fp32 [places, D, N] is updated in place at slots (int32 [B]; default b; outside the
    range: an empty place of the batch, whose y is zero)."""
    w = "snn_selective_scan_step"
    dev, (nB, nD), (N, G), dt = _device(w, u), u.shape, (A.shape[-1], B.shape[1]), u.dtype
    _, d = _sscan_desc(w, nB, 1, nD, N, G, dt, bool(softplus))
    seq, grp, f32, n = (nB, nD), (nB, G, N), torch.float32, state.shape[0]
    keep, (pu, pd, pB, pC, pz, py) = _structs(
        _btc(w, "u", u, seq, dt, dev), _btc(w, "delta", delta, seq, dt, dev),
        _btgn(w, "B", B, grp, dt, dev), _btgn(w, "C", C, grp, dt, dev), _btc(w, "z", z, seq, dt, dev),
        _btc(w, "y", y, seq, dt, dev))
    _check(load_library().snn_selective_scan_step(
        d, pu, pd, _whole(w, "A", A, (nD, N), f32, dev), pB, pC, _whole(w, "D", D, (nD,), f32, dev), pz,
        _whole(w, "delta_bias", delta_bias, (nD,), f32, dev), _whole(w, "state", state, (n, nD, N), f32, dev),
        _whole(w, "slots", slots, (nB,), torch.int32, dev), n, py, _stream(stream, dev)), w)


@functools.lru_cache(maxsize=1024)
def _conv_desc(where, B, T, C, W, dtype, act):
    code = _TORCH_DTYPE_CODE.get(dtype)
    if code is None:
        raise ValueError(f"{where}: dtype {dtype}")
    if act not in GATE_CODE:
        raise ValueError(f"{where}: act {act!r}")
    d = ConvDesc(B, T, C, W, code, GATE_CODE[act])
    return d, ctypes.addressof(d)


@functools.lru_cache(maxsize=1024)
def snn_causal_conv_workspace_bytes(B, T, C, W) -> int:
    d = ConvDesc(B, T, C, W)
    return load_library().snn_causal_conv_workspace_bytes(ctypes.byref(d))


def snn_causal_conv_fwd(x, w, bias, y, act="none", seq_lens=None, state_in=None, state_out=None,
                        slots=None, stream=None):
    """Causal convolution of each channel over W = 2, 3 or 4 tokens, y_t = act(bias +
    sum_j w[j] x_{t-W+1+j}): x, y [B, T, C] (fp32, bf16 or fp16, any strides with contiguous C),
    w fp32 [C, W], bias fp32 [C] or None, act "none" or "silu".  states [places, W-1, C] of
    x's type hold the inputs before the sequence, with slots int32 [B] naming the places."""
    f = "snn_causal_conv_fwd"
    dev, (B, T, C), W, dt = _device(f, x), x.shape, w.shape[-1], x.dtype
    _, d = _conv_desc(f, B, T, C, W, dt, act)
    ps, n = _places_of(f, slots, B, (state_in, state_out), dev)
    keep, (px, py) = _structs(_btc(f, "x", x, (B, T, C), dt, dev), _btc(f, "y", y, (B, T, C), dt, dev))
    _check(load_library().snn_causal_conv_fwd(
        d, px, _whole(f, "w", w, (C, W), torch.float32, dev), _whole(f, "bias", bias, (C,), torch.float32, dev),
        _whole(f, "seq_lens", seq_lens, (B,), torch.int32, dev),
        _whole(f, "state_in", state_in, (n, W - 1, C), dt, dev),
        _whole(f, "state_out", state_out, (n, W - 1, C), dt, dev), ps, n, py, _stream(stream, dev)), f)


def snn_causal_conv_bwd(x, w, bias, grad_y, grad_x, grad_w, grad_bias, ws, act="none", seq_lens=None,
                        state_in=None, grad_state_out=None, grad_state_in=None, stream=None):
    """Gradients of snn_causal_conv_fwd (states [B, W-1, C], in sequence order); an output
    None is not computed.  ws: snn_causal_conv_workspace_bytes (None without grad_w and
    grad_bias)."""
    f = "snn_causal_conv_bwd"
    dev, (B, T, C), W, dt = _device(f, x), x.shape, w.shape[-1], x.dtype
    _, d = _conv_desc(f, B, T, C, W, dt, act)
    seq = (B, T, C)
    keep, (px, pgy, pgx) = _structs(_btc(f, "x", x, seq, dt, dev), _btc(f, "grad_y", grad_y, seq, dt, dev),
                                    _btc(f, "grad_x", grad_x, seq, dt, dev))
    f32 = lambda name, t, shape: _whole(f, name, t, shape, torch.float32, dev)
    state = lambda name, t: _whole(f, name, t, (B, W - 1, C), dt, dev)
    pw, nw = _ws(f, ws, dev)
    _check(load_library().snn_causal_conv_bwd(
        d, px, f32("w", w, (C, W)), f32("bias", bias, (C,)),
        _whole(f, "seq_lens", seq_lens, (B,), torch.int32, dev), state("state_in", state_in), pgy,
        state("grad_state_out", grad_state_out), pgx, f32("grad_w", grad_w, (C, W)),
        f32("grad_bias", grad_bias, (C,)), state("grad_state_in", grad_state_in), pw, nw,
        _stream(stream, dev)), f)


def snn_causal_conv_step(x, w, bias, state, y, act="none", slots=None, stream=None):
    """One token of each sequence (decoding): x, y [B, C]; state [places, W-1, C] of x's
    type loses its oldest input and takes x, at slots (int32 [B]; default b; outside the
    range: an empty place of the batch, whose y is zero)."""
    f = "snn_causal_conv_step"
    dev, (B, C), W, dt = _device(f, x), x.shape, w.shape[-1], x.dtype
    _, d = _conv_desc(f, B, 1, C, W, dt, act)
    n = state.shape[0]
    keep, (px, py) = _structs(_btc(f, "x", x, (B, C), dt, dev), _btc(f, "y", y, (B, C), dt, dev))
    _check(load_library().snn_causal_conv_step(
        d, px, _whole(f, "w", w, (C, W), torch.float32, dev), _whole(f, "bias", bias, (C,), torch.float32, dev),
        _whole(f, "state", state, (n, W - 1, C), dt, dev), _whole(f, "slots", slots, (B,), torch.int32, dev), n,
        py, _stream(stream, dev)), f)


@functools.lru_cache(maxsize=1024)
def snn_layer_norm_workspace_bytes(M: int, N: int) -> int:
    return load_library().snn_layer_norm_workspace_bytes(M, N)


@functools.lru_cache(maxsize=1024)
def _layer_norm_desc(where, M, N, dtype, res_dtype, eps):
    for dt in (dtype, res_dtype):
        if dt not in _TORCH_DTYPE_CODE:
            raise ValueError(f"{where}: dtype {dt}")
    d = LayerNormDesc(M, N, _TORCH_DTYPE_CODE[dtype], _TORCH_DTYPE_CODE[res_dtype], eps)
    return d, ctypes.addressof(d)


def _matrix(where, name, t, shape, dtype, device):
    """The words of snn_rows for an [M, N] matrix with contiguous rows, or for None."""
    if t is None:
        return 0, 0
    st = t.stride()
    if t.shape != shape or t.dtype != dtype or t.device != device or (st[-1] != 1 and shape[1] > 1):
        _refuse(where, name, t, shape, dtype, device, "have contiguous rows")
    return t.data_ptr(), st[0]


def snn_layer_norm_fwd(x, w, b, y, stats=None, eps=1e-5, stream=None):
    """y = (x - mean) rsqrt(var + eps) w + b over the rows of [M, N] matrices (rows any stride
    apart; y of x's type, or 16-bit of an fp32 x); w (None: ones) and b (None: zeros) fp32
    [N]; stats fp32 [2, M] for the backward, or None."""
    f = "snn_layer_norm_fwd"
    dev, (M, N) = _device(f, x), x.shape
    _, d = _layer_norm_desc(f, M, N, y.dtype, x.dtype, float(eps))
    keep, (px, py) = _structs(_matrix(f, "x", x, (M, N), x.dtype, dev), _matrix(f, "y", y, (M, N), y.dtype, dev))
    f32 = lambda name, t, shape: _whole(f, name, t, shape, torch.float32, dev)
    _check(load_library().snn_layer_norm_fwd(d, px, f32("w", w, (N,)), f32("b", b, (N,)), py,
                                             f32("stats", stats, (2, M)), _stream(stream, dev)), f)


def snn_layer_norm_bwd(x, w, stats, grad_y, grad_x, grad_w, grad_b, ws, stream=None):
    """Gradients of snn_layer_norm_fwd from its stats; an output None is not computed.  ws:
    snn_layer_norm_workspace_bytes(M, N) (None without grad_w and grad_b)."""
    f = "snn_layer_norm_bwd"
    dev, (M, N) = _device(f, x), x.shape
    _, d = _layer_norm_desc(f, M, N, grad_y.dtype, x.dtype, 1.0)
    keep, (px, pgy, pgx) = _structs(
        _matrix(f, "x", x, (M, N), x.dtype, dev), _matrix(f, "grad_y", grad_y, (M, N), grad_y.dtype, dev),
        _matrix(f, "grad_x", grad_x, (M, N), x.dtype, dev))
    f32 = lambda name, t, shape: _whole(f, name, t, shape, torch.float32, dev)
    pw, nw = _ws(f, ws, dev)
    _check(load_library().snn_layer_norm_bwd(
        d, px, f32("w", w, (N,)), f32("stats", stats, (2, M)), pgy, pgx, f32("grad_w", grad_w, (N,)),
        f32("grad_b", grad_b, (N,)), pw, nw, _stream(stream, dev)), f)


# ---------------------------------------------------------------------------
# A layer object: allocates the buffers of one scan workload on the device
# ---------------------------------------------------------------------------

class ScanLayer:
    """Device buffers plus forward/backward calls for one ScanWorkload.

    Inputs are taken as given (already on the device); outputs, checkpoints
    and the workspace are allocated once with torch and reused.
    """

    def __init__(self, w: W.ScanWorkload, device="cuda", want_syn: bool = False, **desc_over):
        self.w = w
        self.synaptic = w.neuron == "synaptic"
        self.recurrent = w.neuron == "rleaky"   # Eq. (7): v in the alpha slot
        self.desc = make_desc(w, **desc_over)
        self.device = torch.device(device)
        io = W.TORCH_DTYPE[w.io_dtype]
        shape = (w.T, w.B, w.N)
        dev = self.device
        self.spk = torch.empty(shape, dtype=io, device=dev)
        need_mem = w.want_mem or w.save == "mem"
        self.mem = torch.empty(shape, dtype=io, device=dev) if need_mem else None
        self.syn = torch.empty(shape, dtype=io, device=dev) if (self.synaptic and want_syn) else None
        nck = snn_scan_ckpt_elems(self.desc, self.synaptic)
        self.ckpt = torch.empty(max(nck, 1), dtype=torch.float32, device=dev) if nck > 0 else None
        self.mem_final = torch.empty((w.B, w.N), dtype=torch.float32, device=dev)
        self.syn_final = torch.empty((w.B, w.N), dtype=torch.float32, device=dev) if self.synaptic else None
        self.grad_I = torch.empty(shape, dtype=io, device=dev)
        plen = {"scalar": 1, "per_neuron": w.N, "per_channel": w.C}
        self.grad_beta = torch.empty(plen[w.beta_mode], dtype=torch.float32, device=dev)
        self.grad_thr = torch.empty(plen[w.thr_mode], dtype=torch.float32, device=dev)
        self.grad_alpha = torch.empty(plen[w.alpha_mode], dtype=torch.float32, device=dev) \
            if self.synaptic else None
        self.grad_v = torch.empty(plen[w.v_mode], dtype=torch.float32, device=dev) \
            if self.recurrent else None
        self.grad_mem0 = torch.empty((w.B, w.N), dtype=torch.float32, device=dev)
        self.grad_syn0 = torch.empty((w.B, w.N), dtype=torch.float32, device=dev) \
            if self.synaptic else None
        nws = snn_scan_workspace_bytes(self.desc)
        if nws == 0:
            raise SnnError(1, "snn_scan_workspace_bytes")
        self.ws = torch.empty(nws, dtype=torch.uint8, device=dev)
        snn_workspace_init(self.ws)

    def forward(self, I, beta, thr, alpha=None, mem0=None, syn0=None, stream=None, v=None):
        if self.recurrent:
            snn_rleaky_fwd(self.desc, I, v, beta, thr, mem0, self.spk, self.mem, self.ckpt,
                           self.mem_final, self.ws, stream)
        elif self.synaptic:
            snn_synaptic_fwd(self.desc, I, alpha, beta, thr, mem0, syn0, self.spk, self.mem,
                             self.syn, self.ckpt, self.mem_final, self.syn_final, self.ws, stream)
        else:
            snn_leaky_fwd(self.desc, I, beta, thr, mem0, self.spk, self.mem, self.ckpt,
                          self.mem_final, self.ws, stream)
        return self.spk

    def backward(self, I, beta, thr, grad_spk, alpha=None, mem0=None, syn0=None, grad_mem=None,
                 grad_mem_final=None, grad_syn_final=None, want_param_grads=True,
                 want_state_grads=True, stream=None, v=None):
        gb = self.grad_beta if want_param_grads else None
        gt = self.grad_thr if want_param_grads else None
        gm0 = self.grad_mem0 if want_state_grads else None
        recompute = self.w.save == "recompute"
        if self.recurrent:
            snn_rleaky_bwd(self.desc, I if recompute else None, self.ckpt, self.mem, self.spk, v,
                           beta, thr, mem0, grad_spk, grad_mem, grad_mem_final, self.grad_I,
                           self.grad_v if want_param_grads else None, gb, gt, gm0, self.ws,
                           stream)
        elif self.synaptic:
            ga = self.grad_alpha if (want_param_grads and (recompute or self.syn is not None)) else None
            gs0 = self.grad_syn0 if want_state_grads else None
            snn_synaptic_bwd(self.desc, I if recompute else None, self.ckpt, self.mem, self.spk,
                             self.syn, alpha, beta, thr, mem0, syn0, grad_spk, grad_mem,
                             grad_mem_final, grad_syn_final, self.grad_I, ga, gb, gt, gm0, gs0,
                             self.ws, stream)
        else:
            snn_leaky_bwd(self.desc, I if recompute else None, self.ckpt, self.mem, self.spk,
                          beta, thr, mem0, grad_spk, grad_mem, grad_mem_final, self.grad_I, gb,
                          gt, gm0, self.ws, stream)
        return self.grad_I

    def status(self, stream=None) -> int:
        return snn_workspace_status(self.ws, stream)

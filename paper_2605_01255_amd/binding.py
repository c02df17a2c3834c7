"""ctypes binding of libacc.so: same names as include/acc.h, argument marshalling only.

PyTorch appears here only as the owner of device memory and of the HIP stream; every step of
the layer runs inside the library's kernels.  There is no CPU fallback: if the library is not
built, importing this module raises.
"""
from __future__ import annotations

import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libacc.so")

ACC_F32, ACC_BF16 = 0, 1
ACC_FLAG_SKIP_SKETCH = 1
ACC_FLAG_ONE_LAUNCH = 2
ACC_FLAG_W_OUT_IN = 4
ACC_FLAG_DW_ACCUMULATE = 8
ACC_FLAG_RSVD_POWER_SHIFT = 8   # flags bits 8..9: rounds of subspace iteration of the RSVD forward

ACC_STATIC_SCRATCH_BYTES = 32 << 20
ACC_FP8_E4M3, ACC_FP8_E5M2 = 0, 1
ACC_ACT8_BLOCK = 32
ACC_ACT8_E4M3, ACC_ACT8_INT8 = 0, 1
ACC_ATTN_CAUSAL = 1

EXPORTS = ("acc_linear_workspace_bytes", "acc_linear_fwd", "acc_linear_fwd_static", "acc_linear_bwd", "acc_linear_dw",
           "acc_linear_fwd_fp8", "acc_linear_bwd_fp8",
           "acc_linear_bias_grad",
           "acc_rsvd_workspace_bytes", "acc_linear_fwd_rsvd", "acc_linear_bwd_rsvd", "acc_lowrank_workspace_bytes",
           "acc_lowrank_projector", "acc_lowrank_adamw_step",
           "acc_act8_pack", "acc_act8_unpack", "acc_linear_fwd_act8", "acc_linear_act8_workspace_bytes",
           "acc_linear_bwd_act8", "acc_gated_fwd_act8", "acc_gated_bwd_act8",
           "acc_linear_ce_workspace_bytes", "acc_linear_ce_fwd", "acc_linear_ce_bwd",
           "acc_attn_workspace_bytes", "acc_attn_fwd", "acc_attn_bwd",
           "acc_embed_fwd", "acc_embed_workspace_bytes", "acc_embed_bwd",
           "acc_grad_norm_workspace_bytes", "acc_grad_norm", "acc_grad_scale",
           "acc_philox_dump_u32", "acc_probe_mfma",
           "acc_sketch_dump", "acc_status_string", "acc_version")


class AccLinearDesc(ctypes.Structure):
    """Mirror of `acc_linear_desc`."""
    _fields_ = [("n", ctypes.c_int64), ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
                ("r", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldw", ctypes.c_int64),
                ("ldy", ctypes.c_int64), ("seed", ctypes.c_uint64), ("row_offset", ctypes.c_uint64),
                ("io_dtype", ctypes.c_int32), ("factor_dtype", ctypes.c_int32),
                ("dw_dtype", ctypes.c_int32), ("flags", ctypes.c_uint32), ("ldf", ctypes.c_int64)]


class AccAdamwHyper(ctypes.Structure):
    """Mirror of `acc_adamw_hyper`."""
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float), ("scale", ctypes.c_float),
                ("step", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class AccAct8Desc(ctypes.Structure):
    """Mirror of `acc_act8_desc`."""
    _fields_ = [("n", ctypes.c_int64), ("c", ctypes.c_int64), ("ldx", ctypes.c_int64), ("io_dtype", ctypes.c_int32),
                ("format", ctypes.c_int32)]


class AccGatedDesc(ctypes.Structure):
    """Mirror of `acc_gated_desc`."""
    _fields_ = [("n", ctypes.c_int64), ("f", ctypes.c_int64), ("ldg", ctypes.c_int64), ("ldh", ctypes.c_int64),
                ("io_dtype", ctypes.c_int32), ("format", ctypes.c_int32)]


class AccCeDesc(ctypes.Structure):
    """Mirror of `acc_ce_desc`."""
    _fields_ = [("n", ctypes.c_int64), ("d", ctypes.c_int64), ("v", ctypes.c_int64), ("ldx", ctypes.c_int64),
                ("ldw", ctypes.c_int64), ("piece", ctypes.c_int64), ("io_dtype", ctypes.c_int32),
                ("dw_dtype", ctypes.c_int32), ("flags", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class AccAttnDesc(ctypes.Structure):
    """Mirror of `acc_attn_desc`."""
    _fields_ = [("n", ctypes.c_int64), ("heads", ctypes.c_int64), ("kv_heads", ctypes.c_int64), ("d", ctypes.c_int64),
                ("ldq", ctypes.c_int64), ("ldk", ctypes.c_int64), ("ldv", ctypes.c_int64), ("ldo", ctypes.c_int64),
                ("docs", ctypes.c_int64), ("seq", ctypes.c_int64), ("window", ctypes.c_int64), ("scale", ctypes.c_float),
                ("cap", ctypes.c_float), ("io_dtype", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class AccEmbedDesc(ctypes.Structure):
    """Mirror of `acc_embed_desc`."""
    _fields_ = [("n", ctypes.c_int64), ("d", ctypes.c_int64), ("v", ctypes.c_int64), ("ldw", ctypes.c_int64), ("ldy", ctypes.c_int64),
                ("scale", ctypes.c_float), ("io_dtype", ctypes.c_int32), ("dw_dtype", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32)]


class AccGradTensor(ctypes.Structure):
    """Mirror of `acc_grad_tensor`."""
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("count", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("dst_dtype", ctypes.c_int32)]


class AccGradFactors(ctypes.Structure):
    """Mirror of `acc_grad_factors`."""
    _fields_ = [("left", ctypes.c_void_p), ("gr", ctypes.c_void_p), ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64), ("r", ctypes.c_int64),
                ("ldl", ctypes.c_int64), ("ldg", ctypes.c_int64), ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class AccError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"libacc status {status}: {status_string(status)}")


# torch first: libacc.so must bind to the HIP runtime torch has loaded, so that torch's device
# pointers and streams are valid inside the library.
import torch  # noqa: E402,F401

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'` "
                      "(there is no fallback path)")
_lib = ctypes.CDLL(LIB_PATH)

_vp, _sz, _dp = ctypes.c_void_p, ctypes.c_size_t, ctypes.POINTER(AccLinearDesc)
_lib.acc_linear_workspace_bytes.restype = _sz
_lib.acc_linear_workspace_bytes.argtypes = [_dp, ctypes.c_int]
_lib.acc_linear_fwd.restype = ctypes.c_int
_lib.acc_linear_fwd.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_linear_fwd_static.restype = ctypes.c_int
_lib.acc_linear_fwd_static.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp]
_lib.acc_linear_bwd.restype = ctypes.c_int
_lib.acc_linear_bwd.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_linear_fwd_fp8.restype = ctypes.c_int
_lib.acc_linear_fwd_fp8.argtypes = [_dp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _sz, _vp]
_lib.acc_linear_bwd_fp8.restype = ctypes.c_int
_lib.acc_linear_bwd_fp8.argtypes = [_dp, _vp, _vp, ctypes.c_int, _vp, ctypes.c_float, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_linear_dw.restype = ctypes.c_int
_lib.acc_linear_dw.argtypes = [_dp, _vp, _vp, _vp, _vp]
_lib.acc_linear_bias_grad.restype = ctypes.c_int
_lib.acc_linear_bias_grad.argtypes = [_dp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_rsvd_workspace_bytes.restype = _sz
_lib.acc_rsvd_workspace_bytes.argtypes = [_dp, ctypes.c_int]
_lib.acc_linear_fwd_rsvd.restype = ctypes.c_int
_lib.acc_linear_fwd_rsvd.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_linear_bwd_rsvd.restype = ctypes.c_int
_lib.acc_linear_bwd_rsvd.argtypes = [_dp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_lowrank_adamw_step.restype = ctypes.c_int
_lib.acc_lowrank_adamw_step.argtypes = [_dp, ctypes.POINTER(AccAdamwHyper), _vp, ctypes.c_int64, _vp, _vp, _vp, _vp,
                                        _vp, _vp, _sz, _vp]
_lib.acc_lowrank_workspace_bytes.restype = _sz
_lib.acc_lowrank_workspace_bytes.argtypes = [_dp, ctypes.c_int64]
_lib.acc_lowrank_projector.restype = ctypes.c_int
_lib.acc_lowrank_projector.argtypes = [_dp, ctypes.c_int64, _vp, _vp, _vp, _vp, _sz, _vp]
_adp, _gdp = ctypes.POINTER(AccAct8Desc), ctypes.POINTER(AccGatedDesc)
_lib.acc_act8_pack.restype = ctypes.c_int
_lib.acc_act8_pack.argtypes = [_adp, _vp, _vp, _vp, _vp]
_lib.acc_act8_unpack.restype = ctypes.c_int
_lib.acc_act8_unpack.argtypes = [_adp, _vp, _vp, _vp, _vp]
_lib.acc_linear_fwd_act8.restype = ctypes.c_int
_lib.acc_linear_fwd_act8.argtypes = [_dp, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.acc_linear_act8_workspace_bytes.restype = _sz
_lib.acc_linear_act8_workspace_bytes.argtypes = [_dp]
_lib.acc_linear_bwd_act8.restype = ctypes.c_int
_lib.acc_linear_bwd_act8.argtypes = [_dp, ctypes.c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_gated_fwd_act8.restype = ctypes.c_int
_lib.acc_gated_fwd_act8.argtypes = [_gdp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.acc_gated_bwd_act8.restype = ctypes.c_int
_lib.acc_gated_bwd_act8.argtypes = [_gdp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]
_cdp = ctypes.POINTER(AccCeDesc)
_lib.acc_linear_ce_workspace_bytes.restype = _sz
_lib.acc_linear_ce_workspace_bytes.argtypes = [_cdp, ctypes.c_int]
_lib.acc_linear_ce_fwd.restype = ctypes.c_int
_lib.acc_linear_ce_fwd.argtypes = [_cdp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_linear_ce_bwd.restype = ctypes.c_int
_lib.acc_linear_ce_bwd.argtypes = [_cdp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_tdp = ctypes.POINTER(AccAttnDesc)
_lib.acc_attn_workspace_bytes.restype = _sz
_lib.acc_attn_workspace_bytes.argtypes = [_tdp, ctypes.c_int]
_lib.acc_attn_fwd.restype = ctypes.c_int
_lib.acc_attn_fwd.argtypes = [_tdp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_attn_bwd.restype = ctypes.c_int
_lib.acc_attn_bwd.argtypes = [_tdp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]
_edp, _gtp, _gfp = ctypes.POINTER(AccEmbedDesc), ctypes.POINTER(AccGradTensor), ctypes.POINTER(AccGradFactors)
_lib.acc_embed_fwd.restype = ctypes.c_int
_lib.acc_embed_fwd.argtypes = [_edp, _vp, _vp, _vp, _vp]
_lib.acc_embed_workspace_bytes.restype = _sz
_lib.acc_embed_workspace_bytes.argtypes = [_edp]
_lib.acc_embed_bwd.restype = ctypes.c_int
_lib.acc_embed_bwd.argtypes = [_edp, _vp, _vp, _vp, _vp, _sz, _vp]
_lib.acc_grad_norm_workspace_bytes.restype = _sz
_lib.acc_grad_norm_workspace_bytes.argtypes = [_gtp, ctypes.c_int64, _gfp, ctypes.c_int64]
_lib.acc_grad_norm.restype = ctypes.c_int
_lib.acc_grad_norm.argtypes = [_gtp, ctypes.c_int64, _gfp, ctypes.c_int64, ctypes.c_float, _vp, _vp, _sz, _vp]
_lib.acc_grad_scale.restype = ctypes.c_int
_lib.acc_grad_scale.argtypes = [_gtp, ctypes.c_int64, _vp, _vp]
_lib.acc_philox_dump_u32.restype = ctypes.c_int
_lib.acc_philox_dump_u32.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int64, ctypes.c_int64, _vp, _vp]
_lib.acc_sketch_dump.restype = ctypes.c_int
_lib.acc_sketch_dump.argtypes = [_dp, _vp, _vp]
_lib.acc_probe_mfma.restype = ctypes.c_int
_lib.acc_probe_mfma.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int64, _vp, _sz,
                                ctypes.POINTER(ctypes.c_double), _vp]
_lib.acc_status_string.restype = ctypes.c_char_p
_lib.acc_status_string.argtypes = [ctypes.c_int]
_lib.acc_version.restype = ctypes.c_int
_lib.acc_version.argtypes = []


def status_string(status: int) -> str:
    return _lib.acc_status_string(int(status)).decode()


def acc_probe_mfma(shape, waves_per_simd, random_data, iters, sink, stream=None) -> float:
    """Enqueue one launch of the register-only MFMA loop; returns the flops of the launch."""
    flops = ctypes.c_double(0.0)
    _check(_lib.acc_probe_mfma(shape, waves_per_simd, 1 if random_data else 0, iters, _ptr(sink),
                               sink.numel() * sink.element_size(), ctypes.byref(flops), _stream(stream)))
    return flops.value


def acc_version() -> int:
    return int(_lib.acc_version())


def make_desc(n, d_in, d_out, r, seed=0, io_dtype=ACC_BF16, factor_dtype=None, dw_dtype=None,
              row_offset=0, ldx=0, ldw=0, ldy=0, flags=0, ldf=0) -> AccLinearDesc:
    if factor_dtype is None:
        factor_dtype = io_dtype
    if dw_dtype is None:
        dw_dtype = io_dtype
    return AccLinearDesc(n, d_in, d_out, r, ldx, ldw, ldy, seed, row_offset, io_dtype, factor_dtype,
                         dw_dtype, flags, ldf)


def _ptr(t):
    """Device pointer of a torch tensor (or None -> NULL, or a raw int)."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# The handle of the current stream without a Stream object around it: 0.3 us against 3, and 14 in autograd's thread,
# where a backward pass asks for it twice.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int):
    if status != 0:
        raise AccError(status)


def acc_linear_workspace_bytes(desc: AccLinearDesc, is_backward: bool) -> int:
    return int(_lib.acc_linear_workspace_bytes(ctypes.byref(desc), 1 if is_backward else 0))


def acc_linear_fwd(desc, X, W, Y, Xs, workspace, stream=None, ws_bytes=None):
    """Enqueue Y = X.W and Xs = X^T.S.  All tensors are caller-allocated device tensors."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_fwd(ctypes.byref(desc), _ptr(X), _ptr(W), _ptr(Y), _ptr(Xs),
                               _ptr(workspace), ws_bytes, _stream(stream)))


def acc_linear_fwd_static(desc, X, W, Y, Xs, stream=None):
    """acc_linear_fwd with the partial tiles in the library's static device array (nothing is allocated)."""
    _check(_lib.acc_linear_fwd_static(ctypes.byref(desc), _ptr(X), _ptr(W), _ptr(Y), _ptr(Xs), _stream(stream)))


def acc_linear_bwd(desc, dY, W, Xs, dX, Gr, dW, workspace, stream=None, ws_bytes=None):
    """Enqueue dX = dY.W^T, Gr = S^T.dY and (dW is not None) dW = Xs.Gr."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_bwd(ctypes.byref(desc), _ptr(dY), _ptr(W), _ptr(Xs), _ptr(dX), _ptr(Gr),
                               _ptr(dW), _ptr(workspace), ws_bytes, _stream(stream)))


def acc_linear_fwd_fp8(desc, X, X8, W8, scale, Y, Xs, workspace, stream=None, ws_bytes=None):
    """Enqueue Y = scale * (X8.W8) on 8-bit operands (uint8 tensors of fp8 e4m3 bits) and Xs = X^T.S from the bf16 X."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_fwd_fp8(ctypes.byref(desc), _ptr(X), _ptr(X8), _ptr(W8), float(scale), _ptr(Y), _ptr(Xs),
                                   _ptr(workspace), ws_bytes, _stream(stream)))


def acc_linear_bwd_fp8(desc, dY, dY8, dy8_format, W8, scale, Xs, dX, Gr, dW, workspace, stream=None, ws_bytes=None):
    """Enqueue dX = scale * (dY8.W8^T) on 8-bit operands, Gr = S^T.dY from the bf16 dY and (dW is not None) dW."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_bwd_fp8(ctypes.byref(desc), _ptr(dY), _ptr(dY8), int(dy8_format), _ptr(W8), float(scale),
                                   _ptr(Xs), _ptr(dX), _ptr(Gr), _ptr(dW), _ptr(workspace), ws_bytes,
                                   _stream(stream)))


def acc_linear_dw(desc, Xs, Gr, dW, stream=None):
    """Enqueue dW = Xs.Gr (+= with ACC_FLAG_DW_ACCUMULATE) from the two factors alone."""
    _check(_lib.acc_linear_dw(ctypes.byref(desc), _ptr(Xs), _ptr(Gr), _ptr(dW), _stream(stream)))


def acc_linear_bias_grad(desc, dY, dB, workspace, stream=None, ws_bytes=None):
    """Enqueue dB = column sums of dY (workspace: the backward one)."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_bias_grad(ctypes.byref(desc), _ptr(dY), _ptr(dB), _ptr(workspace), ws_bytes,
                                     _stream(stream)))


def acc_rsvd_workspace_bytes(desc: AccLinearDesc, is_backward: bool) -> int:
    return int(_lib.acc_rsvd_workspace_bytes(ctypes.byref(desc), 1 if is_backward else 0))


def acc_linear_fwd_rsvd(desc, X, W, Y, U, V, workspace, stream=None, ws_bytes=None):
    """Enqueue Y = X.W and the RSVD factors U [n, r], V [d_in, r] of X."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_fwd_rsvd(ctypes.byref(desc), _ptr(X), _ptr(W), _ptr(Y), _ptr(U), _ptr(V),
                                    _ptr(workspace), ws_bytes, _stream(stream)))


def acc_linear_bwd_rsvd(desc, dY, W, U, V, dX, Gr, dW, workspace, stream=None, ws_bytes=None):
    """Enqueue dX = dY.W^T, Gr = U^T.dY and (dW is not None) dW = V.Gr."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_bwd_rsvd(ctypes.byref(desc), _ptr(dY), _ptr(W), _ptr(U), _ptr(V), _ptr(dX),
                                    _ptr(Gr), _ptr(dW), _ptr(workspace), ws_bytes, _stream(stream)))


def make_hyper(step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, scale=1.0) -> AccAdamwHyper:
    return AccAdamwHyper(lr, beta1, beta2, eps, weight_decay, scale, step, 0)


def acc_lowrank_workspace_bytes(desc: AccLinearDesc, k: int) -> int:
    return int(_lib.acc_lowrank_workspace_bytes(ctypes.byref(desc), int(k)))


def acc_lowrank_projector(desc, k, left, Gr, P, workspace, stream=None, ws_bytes=None):
    """Enqueue P [d_in, k] = orthonormal basis of a k-dimensional subspace of range(left . Gr)."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_lowrank_projector(ctypes.byref(desc), int(k), _ptr(left), _ptr(Gr), _ptr(P), _ptr(workspace),
                                      ws_bytes, _stream(stream)))


def acc_lowrank_adamw_step(desc, hyper, P, k, left, Gr, M, V, W, workspace, stream=None, ws_bytes=None):
    """Enqueue one AdamW update of W from the gradient factors left [d_in, r] and Gr, through the projector
    P [d_in, k] (None: the left factor is the projector, k = r); M, V fp32 [k, d_out]."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_lowrank_adamw_step(ctypes.byref(desc), ctypes.byref(hyper), _ptr(P), int(k), _ptr(left),
                                       _ptr(Gr), _ptr(M), _ptr(V), _ptr(W), _ptr(workspace), ws_bytes,
                                       _stream(stream)))


def alloc_lowrank_workspace(desc, k: int, device="cuda:0"):
    import torch
    return torch.empty(max(acc_lowrank_workspace_bytes(desc, k), 16), dtype=torch.uint8, device=device)


def make_act8_desc(n, c, ldx=0, io_dtype=ACC_BF16, format=ACC_ACT8_E4M3) -> AccAct8Desc:
    return AccAct8Desc(n, c, ldx, io_dtype, format)


def alloc_act8(desc: AccAct8Desc, device="cuda:0"):
    """The two buffers of a checkpoint: its bytes [n, c] and its blocks' exponents (uint8 tensors)."""
    return (torch.empty(desc.n, desc.c, dtype=torch.uint8, device=device),
            torch.empty((desc.n + ACC_ACT8_BLOCK - 1) // ACC_ACT8_BLOCK, desc.c, dtype=torch.uint8, device=device))


def acc_act8_pack(desc, X, Q, E, stream=None):
    """Enqueue Q, E = the 8-bit checkpoint of X."""
    _check(_lib.acc_act8_pack(ctypes.byref(desc), _ptr(X), _ptr(Q), _ptr(E), _stream(stream)))


def acc_act8_unpack(desc, Q, E, X, stream=None):
    """Enqueue X = the values that the checkpoint stands for."""
    _check(_lib.acc_act8_unpack(ctypes.byref(desc), _ptr(Q), _ptr(E), _ptr(X), _stream(stream)))


def acc_linear_fwd_act8(desc, format, X, W, Y, Q, E, stream=None):
    """Enqueue Y = X.W and the 8-bit checkpoint of X."""
    _check(_lib.acc_linear_fwd_act8(ctypes.byref(desc), int(format), _ptr(X), _ptr(W), _ptr(Y), _ptr(Q), _ptr(E),
                                    _stream(stream)))


def acc_linear_act8_workspace_bytes(desc: AccLinearDesc) -> int:
    return int(_lib.acc_linear_act8_workspace_bytes(ctypes.byref(desc)))


def acc_linear_bwd_act8(desc, format, dY, W, Q, E, dX, dW, workspace, stream=None, ws_bytes=None):
    """Enqueue dX = dY.W^T (dX is not None) and dW = X^^T.dY from the checkpoint (dW is not None)."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_bwd_act8(ctypes.byref(desc), int(format), _ptr(dY), _ptr(W), _ptr(Q), _ptr(E), _ptr(dX),
                                    _ptr(dW), _ptr(workspace), ws_bytes, _stream(stream)))


def make_gated_desc(n, f, ldg=0, ldh=0, io_dtype=ACC_BF16, format=ACC_ACT8_E4M3) -> AccGatedDesc:
    return AccGatedDesc(n, f, ldg, ldh, io_dtype, format)


def alloc_gated_act8(desc: AccGatedDesc, device="cuda:0"):
    """Qg, Eg, Qu, Eu of acc_gated_fwd_act8."""
    one = make_act8_desc(desc.n, desc.f, io_dtype=desc.io_dtype, format=desc.format)
    return (*alloc_act8(one, device), *alloc_act8(one, device))


def acc_gated_fwd_act8(desc, G, U, H, Qg, Eg, Qu, Eu, stream=None):
    """Enqueue H = silu(G) o U and the 8-bit checkpoints of G and U."""
    _check(_lib.acc_gated_fwd_act8(ctypes.byref(desc), _ptr(G), _ptr(U), _ptr(H), _ptr(Qg), _ptr(Eg), _ptr(Qu), _ptr(Eu),
                                   _stream(stream)))


def acc_gated_bwd_act8(desc, dH, Qg, Eg, Qu, Eu, dG, dU, H=None, stream=None):
    """Enqueue dG and dU from the checkpoints and (H is not None) the activation again."""
    _check(_lib.acc_gated_bwd_act8(ctypes.byref(desc), _ptr(dH), _ptr(Qg), _ptr(Eg), _ptr(Qu), _ptr(Eu), _ptr(dG),
                                   _ptr(dU), _ptr(H), _stream(stream)))


def make_ce_desc(n, d, v, ldx=0, ldw=0, piece=0, io_dtype=ACC_BF16, dw_dtype=None, flags=0) -> AccCeDesc:
    return AccCeDesc(n, d, v, ldx, ldw, piece, io_dtype, io_dtype if dw_dtype is None else dw_dtype, flags, 0)


def acc_linear_ce_workspace_bytes(desc: AccCeDesc, is_backward: bool) -> int:
    return int(_lib.acc_linear_ce_workspace_bytes(ctypes.byref(desc), 1 if is_backward else 0))


def acc_linear_ce_fwd(desc, X, W, targets, loss, stats, workspace, stream=None, ws_bytes=None):
    """Enqueue the per-token losses of X.W^T against `targets` (int64) and what the backward call reads of them."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_ce_fwd(ctypes.byref(desc), _ptr(X), _ptr(W), _ptr(targets), _ptr(loss), _ptr(stats),
                                  _ptr(workspace), ws_bytes, _stream(stream)))


def acc_linear_ce_bwd(desc, X, W, targets, stats, dloss, dX, dW, workspace, stream=None, ws_bytes=None):
    """Enqueue dX and dW of sum(dloss * loss); either may be None."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_linear_ce_bwd(ctypes.byref(desc), _ptr(X), _ptr(W), _ptr(targets), _ptr(stats), _ptr(dloss),
                                  _ptr(dX), _ptr(dW), _ptr(workspace), ws_bytes, _stream(stream)))


def make_attn_desc(n, heads, kv_heads, d, ldq=0, ldk=0, ldv=0, ldo=0, docs=0, seq=0, window=0, scale=0.0, cap=0.0, io_dtype=ACC_BF16,
                   flags=ACC_ATTN_CAUSAL) -> AccAttnDesc:
    return AccAttnDesc(n, heads, kv_heads, d, ldq, ldk, ldv, ldo, docs, seq, window, scale, cap, io_dtype, flags)


def acc_attn_workspace_bytes(desc: AccAttnDesc, is_backward: bool) -> int:
    return int(_lib.acc_attn_workspace_bytes(ctypes.byref(desc), 1 if is_backward else 0))


def acc_attn_fwd(desc, Q, K, V, starts, prefix, slopes, O, lse, workspace, stream=None, ws_bytes=None):
    """Enqueue O and lse of attention over the documents of `starts` (int64; None: sequences of desc.seq rows); prefix (int64) and
    slopes (float32) may be None."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_attn_fwd(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), _ptr(starts), _ptr(prefix), _ptr(slopes), _ptr(O), _ptr(lse),
                             _ptr(workspace), ws_bytes, _stream(stream)))


def acc_attn_bwd(desc, Q, K, V, starts, prefix, slopes, O, lse, dO, dQ, dK, dV, workspace, stream=None, ws_bytes=None):
    """Enqueue dQ, dK and dV from what acc_attn_fwd read and wrote, and the gradient of O."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_attn_bwd(ctypes.byref(desc), _ptr(Q), _ptr(K), _ptr(V), _ptr(starts), _ptr(prefix), _ptr(slopes), _ptr(O), _ptr(lse),
                             _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(workspace), ws_bytes, _stream(stream)))


def make_embed_desc(n, d, v, ldw=0, ldy=0, scale=1.0, io_dtype=ACC_BF16, dw_dtype=None, flags=0) -> AccEmbedDesc:
    return AccEmbedDesc(n, d, v, ldw, ldy, scale, io_dtype, io_dtype if dw_dtype is None else dw_dtype, flags, 0)


def acc_embed_fwd(desc, W, ids, Y, stream=None):
    """Enqueue Y = scale W[ids] (ids int64)."""
    _check(_lib.acc_embed_fwd(ctypes.byref(desc), _ptr(W), _ptr(ids), _ptr(Y), _stream(stream)))


def acc_embed_workspace_bytes(desc: AccEmbedDesc) -> int:
    return int(_lib.acc_embed_workspace_bytes(ctypes.byref(desc)))


def acc_embed_bwd(desc, ids, dY, dW, workspace, stream=None, ws_bytes=None):
    """Enqueue dW (+)= scale times the sums of dY over the tokens of a word."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_embed_bwd(ctypes.byref(desc), _ptr(ids), _ptr(dY), _ptr(dW), _ptr(workspace), ws_bytes, _stream(stream)))


_GRAD_CODES = {torch.bfloat16: ACC_BF16, torch.float32: ACC_F32}


def make_grad_list(tensors, outs=None):
    """The table of acc_grad_norm and acc_grad_scale: dense tensors and where they go when scaled (None: in place)."""
    # Filled as one array of AccGradTensor's words (src, dst, count, both types), column by column: 0.7 us a tensor, 1.3 row by row.
    tensors = list(tensors)
    count, of = list(map(torch.Tensor.numel, tensors)), torch.Tensor.data_ptr
    src = dst = list(map(of, tensors))
    whole = all(map(torch.Tensor.is_contiguous, tensors))
    try:
        code = out = [_GRAD_CODES[t.dtype] for t in tensors]
        if outs is not None:
            outs = list(outs)
            whole = whole and all(map(torch.Tensor.is_contiguous, outs)) and count == list(map(torch.Tensor.numel, outs))
            dst, out = list(map(of, outs)), [_GRAD_CODES[t.dtype] for t in outs]
    except KeyError:
        raise TypeError("gradients are bfloat16 or float32") from None
    if not whole:
        raise ValueError("gradients and their outputs must be contiguous and of one size")
    if not tensors:
        return (AccGradTensor * 0)()
    words = [0] * (4 * len(tensors))
    words[0::4], words[1::4], words[2::4], words[3::4] = src, dst, count, [a | b << 32 for a, b in zip(code, out)]
    return (AccGradTensor * len(tensors)).from_buffer_copy(struct.pack(f"{len(words)}q", *words))


def make_factor_list(left, gr, flags=0):
    """The table of factored gradients: left [d_in, r] and gr [r, d_out] ([d_out, r] with ACC_FLAG_W_OUT_IN), rows of any stride."""
    rows = []
    for x, g in zip(left, gr, strict=True):
        d_out, r = g.shape if flags & ACC_FLAG_W_OUT_IN else g.shape[::-1]
        code = _GRAD_CODES.get(x.dtype)
        if code is None or x.dtype != g.dtype or x.shape[1] != r:
            raise ValueError("the factors of a gradient have one type (bfloat16 or float32) and one rank")
        if x.stride(1) != 1 or g.stride(1) != 1:
            raise ValueError("the factors' rows must be contiguous")
        rows.append((x.data_ptr(), g.data_ptr(), x.shape[0], d_out, r, x.stride(0) if x.shape[0] > 1 else 0, g.stride(0) if g.shape[0] > 1 else 0,
                     code, flags))
    return (AccGradFactors * len(rows))(*rows)


def acc_grad_norm_workspace_bytes(tensors, factors) -> int:
    return int(_lib.acc_grad_norm_workspace_bytes(tensors, len(tensors), factors, len(factors)))


def acc_grad_norm(tensors, factors, max_norm, out, workspace, stream=None, ws_bytes=None):
    """Enqueue out[0] = the norm over the tables' gradients and out[1] = min(1, max_norm / (norm + 1e-6)) (float32)."""
    if ws_bytes is None:
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_lib.acc_grad_norm(tensors, len(tensors), factors, len(factors), float(max_norm), _ptr(out), _ptr(workspace), ws_bytes, _stream(stream)))


def acc_grad_scale(tensors, factor, stream=None):
    """Enqueue the table's outputs = its gradients times factor[0] (float32)."""
    _check(_lib.acc_grad_scale(tensors, len(tensors), _ptr(factor), _stream(stream)))


def acc_philox_dump_u32(seed, row_offset, n, r, out, stream=None):
    _check(_lib.acc_philox_dump_u32(seed, row_offset, n, r, _ptr(out), _stream(stream)))


def acc_sketch_dump(desc, S, stream=None):
    _check(_lib.acc_sketch_dump(ctypes.byref(desc), _ptr(S), _stream(stream)))


# ---------------------------------------------------------------------------------------------
# convenience for tests / bench: allocation helpers (torch owns the memory, nothing is computed)
# ---------------------------------------------------------------------------------------------
def torch_dtype(code: int):
    import torch
    return torch.bfloat16 if code == ACC_BF16 else torch.float32


def to_device(arr, device="cuda:0"):
    """numpy float32 array or uint16 bf16-bit array -> device tensor of the matching dtype."""
    import numpy as np
    import torch
    if arr.dtype == np.uint16:
        return torch.from_numpy(arr.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(arr).to(device)


def to_host_f64(t):
    """device tensor -> numpy float64 (exact widening)."""
    import torch
    return t.detach().to("cpu").to(torch.float64).numpy()


def alloc_workspace(desc, is_backward: bool, device="cuda:0", rsvd: bool = False):
    import torch
    nbytes = (acc_rsvd_workspace_bytes if rsvd else acc_linear_workspace_bytes)(desc, is_backward)
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)

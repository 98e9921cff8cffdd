"""Thin ctypes binding of liblrnnx.so: argument marshalling only.

Every function here has the name of the C entry point it calls (include/lrnnx.h) and
does nothing but check tensor dtypes/devices, allocate the outputs and the workspace
with torch, fill the args struct with data pointers, strides and the current HIP
stream, and call into the library.  Calls in their usual form take the same steps in
csrc/binding.cpp.  There is no CPU or PyTorch fallback: if the
library has not been built, importing the entry points raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblrnnx.so")
BINDING_PATH = os.path.join(_HERE, "_binding.so")

F32, BF16, C64 = 0, 1, 2
DISC = {"zoh_s6": 0, "zoh": 1, "bilinear": 2, "dirac": 3}
PATH = {"auto": 0, "single_pass": 1, "chunk_carry": 2}
WS_FWD, WS_BWD, WS_LTI, WS_LTI_BWD, WS_DIAG, WS_DIAG_BWD, WS_BWD_COMPLEX, WS_BWD_CARRY, WS_FWD_COMPLEX, WS_BWD_SUMS = 0, 1, 2, 3, 4, 5, 6, 7, 8, 9
STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported", 3: "workspace", 4: "launch"}

_vp, _i32, _i64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t


_SEL_HEAD = [("struct_size", _sz), ("B", _i32), ("D", _i32), ("N", _i32), ("bc_groups", _i32), ("L", _i64),
             ("io_dtype", _i32), ("disc", _i32), ("delta_softplus", _i32), ("path", _i32), ("cu_seqlens", _vp)]
_SEL_INPUTS = [("u", _vp), ("u_stride_b", _i64), ("u_stride_d", _i64),
               ("delta", _vp), ("delta_stride_b", _i64), ("delta_stride_d", _i64),
               ("A", _vp), ("Bm", _vp), ("Cm", _vp), ("Dskip", _vp), ("delta_bias", _vp),
               ("z", _vp), ("z_stride_b", _i64), ("z_stride_d", _i64),
               ("x0", _vp)]
_SEL_FWD_TAIL = [("y", _vp), ("y_stride_b", _i64), ("y_stride_d", _i64), ("x_last", _vp), ("ckpt", _vp),
                 ("workspace", _vp), ("workspace_bytes", _sz), ("stream", _vp)]
_SEL_BWD_TAIL = [("dy", _vp), ("dy_stride_b", _i64), ("dy_stride_d", _i64), ("ckpt", _vp),
                 ("du", _vp), ("du_stride_b", _i64), ("du_stride_d", _i64),
                 ("ddelta", _vp), ("ddelta_stride_b", _i64), ("ddelta_stride_d", _i64),
                 ("dz", _vp), ("dz_stride_b", _i64), ("dz_stride_d", _i64),
                 ("dA", _vp), ("dBm", _vp), ("dCm", _vp), ("dD", _vp), ("dbias", _vp), ("dx0", _vp),
                 ("workspace", _vp), ("workspace_bytes", _sz), ("stream", _vp)]


class FwdArgs(ctypes.Structure):                  # lrnnx_ss_fwd_args
    _fields_ = _SEL_HEAD + _SEL_INPUTS + _SEL_FWD_TAIL


class FwdComplexArgs(ctypes.Structure):           # lrnnx_ss_fwd_complex_args (same layout, complex pointers)
    _fields_ = _SEL_HEAD + _SEL_INPUTS + _SEL_FWD_TAIL


class BwdArgs(ctypes.Structure):                  # lrnnx_ss_bwd_args
    _fields_ = _SEL_HEAD + [("max_seqlen", _i64)] + _SEL_INPUTS + _SEL_BWD_TAIL


class BwdComplexArgs(ctypes.Structure):           # lrnnx_ss_bwd_complex_args
    _fields_ = _SEL_HEAD + [("max_seqlen", _i64)] + _SEL_INPUTS + _SEL_BWD_TAIL


class LtiArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", _sz), ("B", _i32), ("P", _i32), ("L", _i64), ("path", _i32), ("reserved", _i32),
        ("lambda_", _vp), ("v", _vp), ("x0", _vp), ("x", _vp), ("x_last", _vp), ("chain_status", _vp),
        ("workspace", _vp), ("workspace_bytes", _sz), ("stream", _vp),
    ]


class LtiBwdArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", _sz), ("B", _i32), ("P", _i32), ("L", _i64),
        ("lambda_", _vp), ("x", _vp), ("x0", _vp), ("gx", _vp), ("dv", _vp), ("dlambda", _vp), ("dx0", _vp),
        ("chain_status", _vp), ("workspace", _vp), ("workspace_bytes", _sz), ("stream", _vp),
    ]


class DiagScanArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", _sz), ("B", _i32), ("P", _i32), ("L", _i64), ("dtype", _i32), ("reserved", _i32),
        ("a", _vp), ("b", _vp), ("x0", _vp), ("x", _vp), ("x_last", _vp), ("chain_status", _vp),
        ("workspace", _vp), ("workspace_bytes", _sz), ("stream", _vp),
    ]


class DiagScanBwdArgs(ctypes.Structure):
    _fields_ = [
        ("struct_size", _sz), ("B", _i32), ("P", _i32), ("L", _i64), ("dtype", _i32), ("reserved", _i32),
        ("a", _vp), ("x", _vp), ("x0", _vp), ("gx", _vp), ("da", _vp), ("db", _vp), ("dx0", _vp),
        ("chain_status", _vp), ("workspace", _vp), ("workspace_bytes", _sz), ("stream", _vp),
    ]


_STEP_FIELDS = [
    ("struct_size", _sz), ("B", _i32), ("D", _i32), ("N", _i32), ("bc_groups", _i32),
    ("io_dtype", _i32), ("disc", _i32), ("delta_softplus", _i32), ("reserved", _i32),
    ("x", _vp),
    ("u", _vp), ("u_stride_b", _i64), ("u_stride_d", _i64),
    ("delta", _vp), ("delta_stride_b", _i64), ("delta_stride_d", _i64),
    ("A", _vp), ("Bm", _vp), ("Cm", _vp), ("Dskip", _vp), ("delta_bias", _vp),
    ("z", _vp), ("z_stride_b", _i64), ("z_stride_d", _i64),
    ("y", _vp), ("y_stride_b", _i64), ("y_stride_d", _i64),
    ("stream", _vp),
]


class StepArgs(ctypes.Structure):                 # lrnnx_ss_step_args
    _fields_ = _STEP_FIELDS


class StepComplexArgs(ctypes.Structure):          # lrnnx_ss_step_complex_args
    _fields_ = _STEP_FIELDS


class LtiStepArgs(ctypes.Structure):
    _fields_ = [("struct_size", _sz), ("B", _i32), ("P", _i32), ("lambda_", _vp), ("x", _vp), ("v", _vp), ("stream", _vp)]


def _strided(name, axes):
    return [(name, _vp)] + [(f"{name}_stride_{x}", _i64) for x in axes]


_DELTA_HEAD = [("struct_size", _sz), ("B", _i32), ("Hk", _i32), ("Hv", _i32), ("dk", _i32), ("dv", _i32),
               ("io_dtype", _i32), ("gate_dtype", _i32), ("scale", ctypes.c_float)]
_DELTA_INPUTS = [("L", _i64), ("cu_seqlens", _vp), *_strided("q", "blh"), *_strided("k", "blh"), *_strided("v", "blh"),
                 *_strided("g", "blh"), *_strided("beta", "blh"), ("s0", _vp)]
_SCRATCH = [("workspace", _vp), ("workspace_bytes", _sz), ("stream", _vp)]


class DeltaFwdArgs(ctypes.Structure):             # lrnnx_delta_fwd_args
    _fields_ = _DELTA_HEAD + _DELTA_INPUTS + _strided("o", "blh") + [("s_last", _vp), ("saved", _vp), ("saved_bytes", _sz)] + _SCRATCH


class DeltaBwdArgs(ctypes.Structure):             # lrnnx_delta_bwd_args
    _fields_ = (_DELTA_HEAD + _DELTA_INPUTS + _strided("dout", "blh") + [("ds_last", _vp), ("saved", _vp), ("saved_bytes", _sz)]
                + [(n, _vp) for n in ("dq", "dkey", "dval", "dg", "dbeta", "ds0")] + _SCRATCH)


class DeltaStepArgs(ctypes.Structure):            # lrnnx_delta_step_args
    _fields_ = (_DELTA_HEAD + _strided("q", "bh") + _strided("k", "bh") + _strided("v", "bh") + _strided("g", "bh")
                + _strided("beta", "bh") + [("state", _vp)] + _strided("o", "bh") + [("stream", _vp)])


_NORM_HEAD = [("struct_size", _sz), ("M", _i64), ("D", _i32), ("groups", _i32), ("post_shared", _i32), ("gate_act", _i32),
              ("io_dtype", _i32), ("res_dtype", _i32), ("eps", ctypes.c_float), ("reserved", _i32),
              ("x", _vp), ("x_stride", _i64), ("post_weight", _vp), ("gate", _vp), ("gate_stride", _i64),
              ("residual", _vp), ("residual_stride", _i64), ("res_scale", _vp), ("pre_weight", _vp)]


class NormFwdArgs(ctypes.Structure):              # lrnnx_norm_fwd_args
    _fields_ = _NORM_HEAD + [("h", _vp), ("y", _vp), ("stream", _vp)]


class NormBwdArgs(ctypes.Structure):              # lrnnx_norm_bwd_args
    _fields_ = (_NORM_HEAD + [("dh", _vp), ("dh_stride", _i64), ("dy", _vp), ("dy_stride", _i64)]
                + [(n, _vp) for n in ("dx", "dgate", "dresidual", "dpost_weight", "dres_scale", "dpre_weight")] + _SCRATCH)


_CONV_HEAD = [("struct_size", _sz), ("B", _i32), ("D", _i32), ("W", _i32), ("time_last", _i32), ("act", _i32), ("io_dtype", _i32),
              ("L", _i64), ("cu_seqlens", _vp), *_strided("x", "bs"), ("weight", _vp), ("bias", _vp), ("x0", _vp)]


class ConvFwdArgs(ctypes.Structure):              # lrnnx_conv_fwd_args
    _fields_ = _CONV_HEAD + _strided("y", "bs") + [("x_last", _vp), ("stream", _vp)]


class ConvBwdArgs(ctypes.Structure):              # lrnnx_conv_bwd_args
    _fields_ = (_CONV_HEAD + _strided("dy", "bs") + [("dx_last", _vp)] + _strided("dx", "bs")
                + [(n, _vp) for n in ("dweight", "dbias", "dx0")] + _SCRATCH)


class ConvStepArgs(ctypes.Structure):             # lrnnx_conv_step_args
    _fields_ = [("struct_size", _sz), ("B", _i32), ("D", _i32), ("W", _i32), ("act", _i32), ("io_dtype", _i32), ("reserved", _i32),
                *_strided("x", "bd"), ("weight", _vp), ("bias", _vp), ("state", _vp), *_strided("y", "bd"), ("stream", _vp)]


_VOCAB_HEAD = [("struct_size", _sz), ("T", _i64), ("V", _i64), ("K", _i32), ("io_dtype", _i32), ("h", _vp), ("h_stride", _i64),
               ("weight", _vp), ("weight_stride", _i64), ("target", _vp)]


class VocabFwdArgs(ctypes.Structure):             # lrnnx_vocab_fwd_args
    _fields_ = _VOCAB_HEAD + [("loss", _vp), ("lse", _vp)] + _SCRATCH


class VocabBwdArgs(ctypes.Structure):             # lrnnx_vocab_bwd_args
    _fields_ = _VOCAB_HEAD + [("lse", _vp), ("dloss", _vp), ("dloss_stride", _i64), ("dh", _vp), ("dweight", _vp)] + _SCRATCH


_GRAD_HEAD = [("struct_size", _sz), ("count", _i64), ("grads", _vp), ("numel", _vp), ("dtype", _vp)]


class GradNormArgs(ctypes.Structure):             # lrnnx_grad_norm_args
    _fields_ = _GRAD_HEAD + [("norm", _vp)] + _SCRATCH


class GradClipArgs(ctypes.Structure):             # lrnnx_grad_clip_args
    _fields_ = _GRAD_HEAD + [("out", _vp), ("out_dtype", _vp), ("norm", _vp), ("max_norm", ctypes.c_float), ("eps", ctypes.c_float),
                             ("stream", _vp)]


def _packer(cls):
    """Packs the values of an argument struct's fields in order (0, not None, stands for NULL).  One call of 0.6 us, where 34
    attributes set one by one take 3.7: the general path of the forward call of 16 rows of 256 steps takes 15.3 us, of a generated
    token of 64 x 1536 channels 11.0 (csrc/binding.cpp: 6.6 and 5.0)."""
    code = {_vp: "Q", _i32: "i", _i64: "q", _sz: "Q", ctypes.c_float: "f"}
    p = struct.Struct("=" + "".join(code[t] for _, t in cls._fields_))
    assert p.size == ctypes.sizeof(cls), f"{cls.__name__}: padded"
    return p.pack


_pack_fwd, _pack_bwd, _pack_step = _packer(FwdArgs), _packer(BwdArgs), _packer(StepArgs)
_pack_delta_fwd, _pack_delta_bwd, _pack_delta_step = _packer(DeltaFwdArgs), _packer(DeltaBwdArgs), _packer(DeltaStepArgs)
_pack_norm_fwd, _pack_norm_bwd = _packer(NormFwdArgs), _packer(NormBwdArgs)
_pack_conv_fwd, _pack_conv_bwd, _pack_conv_step = _packer(ConvFwdArgs), _packer(ConvBwdArgs), _packer(ConvStepArgs)
_pack_vocab_fwd, _pack_vocab_bwd = _packer(VocabFwdArgs), _packer(VocabBwdArgs)
_pack_grad_norm, _pack_grad_clip = _packer(GradNormArgs), _packer(GradClipArgs)
_FWD_SIZE, _BWD_SIZE, _STEP_SIZE = ctypes.sizeof(FwdArgs), ctypes.sizeof(BwdArgs), ctypes.sizeof(StepArgs)

_lib = None
_native = None                                    # entry points that csrc/binding.cpp takes in their usual form
_packed = {}                                      # the entry points that are called with a packed struct


def lib():
    """The loaded C library.  Raises if it was not built (no fallback exists)."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH) or not os.path.exists(BINDING_PATH):
            raise RuntimeError(f"{LIB_PATH} or {BINDING_PATH} is missing: run `python -m paper_2602_08810_amd.build` "
                               "(the scan has no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB_PATH)
        L.lrnnx_selective_scan_fwd.argtypes = [ctypes.POINTER(FwdArgs)]
        L.lrnnx_selective_scan_bwd.argtypes = [ctypes.POINTER(BwdArgs)]
        L.lrnnx_selective_scan_bwd_workspace_bytes.argtypes = [ctypes.POINTER(BwdArgs)]
        L.lrnnx_selective_scan_bwd_workspace_bytes.restype = _sz
        L.lrnnx_selective_scan_fwd_complex.argtypes = [ctypes.POINTER(FwdComplexArgs)]
        L.lrnnx_selective_scan_fwd_complex.restype = ctypes.c_int
        L.lrnnx_selective_scan_bwd_complex.argtypes = [ctypes.POINTER(BwdComplexArgs)]
        L.lrnnx_selective_scan_bwd_complex.restype = ctypes.c_int
        L.lrnnx_lti_diag_scan.argtypes = [ctypes.POINTER(LtiArgs)]
        L.lrnnx_lti_diag_scan_static.argtypes = [ctypes.POINTER(LtiArgs)]
        L.lrnnx_lti_diag_scan_static.restype = ctypes.c_int
        L.lrnnx_static_scratch_bytes.restype = _sz
        L.lrnnx_lti_diag_scan_bwd.argtypes = [ctypes.POINTER(LtiBwdArgs)]
        L.lrnnx_lti_diag_scan_bwd.restype = ctypes.c_int
        L.lrnnx_diag_scan.argtypes = [ctypes.POINTER(DiagScanArgs)]
        L.lrnnx_diag_scan.restype = ctypes.c_int
        L.lrnnx_diag_scan_bwd.argtypes = [ctypes.POINTER(DiagScanBwdArgs)]
        L.lrnnx_diag_scan_bwd.restype = ctypes.c_int
        L.lrnnx_selective_step.argtypes = [ctypes.POINTER(StepArgs)]
        L.lrnnx_selective_step_complex.argtypes = [ctypes.POINTER(StepComplexArgs)]
        L.lrnnx_selective_step_complex.restype = ctypes.c_int
        L.lrnnx_lti_step.argtypes = [ctypes.POINTER(LtiStepArgs)]
        L.lrnnx_selective_step.restype = ctypes.c_int
        L.lrnnx_lti_step.restype = ctypes.c_int
        for f in (L.lrnnx_selective_scan_fwd, L.lrnnx_selective_scan_bwd, L.lrnnx_lti_diag_scan, L.lrnnx_version):
            f.restype = ctypes.c_int
        L.lrnnx_workspace_bytes.argtypes = [ctypes.c_int, _i64, _i64, _i64, _i64, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.lrnnx_workspace_bytes.restype = _sz
        L.lrnnx_selective_scan_bwd_chunks.argtypes = [_i64, _i64, _i64, _i64, ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.lrnnx_selective_scan_bwd_chunks.restype = ctypes.c_int
        L.lrnnx_selective_scan_fwd_complex_chunks.argtypes = [_i64, _i64, _i64, _i64, ctypes.c_int, ctypes.c_int]
        L.lrnnx_selective_scan_fwd_complex_chunks.restype = ctypes.c_int
        L.lrnnx_ckpt_interval.restype = _i64
        L.lrnnx_status_string.argtypes = [ctypes.c_int]
        L.lrnnx_status_string.restype = ctypes.c_char_p
        of_bytes, size_of_bytes = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_char_p), ctypes.CFUNCTYPE(_sz, ctypes.c_char_p)
        for n in ("lrnnx_selective_scan_fwd", "lrnnx_selective_scan_bwd", "lrnnx_selective_step", "lrnnx_gated_delta_fwd",
                  "lrnnx_gated_delta_bwd", "lrnnx_gated_delta_step", "lrnnx_block_norm_fwd", "lrnnx_block_norm_bwd",
                  "lrnnx_short_conv_fwd", "lrnnx_short_conv_bwd", "lrnnx_short_conv_step", "lrnnx_vocab_loss_fwd", "lrnnx_vocab_loss_bwd",
                  "lrnnx_grad_norm", "lrnnx_grad_clip"):
            _packed[n] = of_bytes((n, L))
        for n in ("lrnnx_selective_scan_bwd_workspace_bytes", "lrnnx_gated_delta_fwd_workspace_bytes",
                  "lrnnx_gated_delta_saved_bytes", "lrnnx_gated_delta_bwd_workspace_bytes", "lrnnx_short_conv_bwd_workspace_bytes",
                  "lrnnx_vocab_loss_fwd_workspace_bytes", "lrnnx_vocab_loss_bwd_workspace_bytes", "lrnnx_grad_norm_workspace_bytes"):
            _packed[n] = size_of_bytes((n, L))
        L.lrnnx_block_norm_bwd_workspace_bytes.argtypes = [_i64, _i64]
        L.lrnnx_block_norm_bwd_workspace_bytes.restype = _sz
        from . import _binding
        _binding.bind(_check, L.lrnnx_ckpt_interval(), tuple(ctypes.cast(getattr(L, "lrnnx_" + n), _vp).value for n in (
            "selective_scan_fwd", "selective_scan_bwd", "selective_scan_bwd_workspace_bytes", "selective_scan_fwd_complex",
            "selective_scan_bwd_complex", "selective_step", "selective_step_complex", "lti_diag_scan", "lti_diag_scan_bwd",
            "diag_scan", "diag_scan_bwd", "workspace_bytes", "gated_delta_fwd", "gated_delta_fwd_workspace_bytes", "gated_delta_saved_bytes",
            "gated_delta_bwd", "gated_delta_bwd_workspace_bytes", "gated_delta_step", "block_norm_fwd", "block_norm_bwd",
            "block_norm_bwd_workspace_bytes", "short_conv_fwd", "short_conv_bwd", "short_conv_bwd_workspace_bytes", "short_conv_step",
            "vocab_loss_fwd", "vocab_loss_fwd_workspace_bytes", "vocab_loss_bwd", "vocab_loss_bwd_workspace_bytes", "grad_norm",
            "grad_norm_workspace_bytes", "grad_clip")))
        _lib = L
        _native = _binding
    return _lib


def _call(name, args):
    """An entry point on a packed argument struct."""
    if _lib is None:
        lib()
    return _packed[name](args)


class LrnnxError(RuntimeError):
    def __init__(self, code):
        self.code = code
        super().__init__(f"lrnnx status {code}: {lib().lrnnx_status_string(code).decode()}")


def _check(code):
    if code != 0:
        raise LrnnxError(code)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _io_dtype(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"I/O dtype must be float32 or bfloat16, got {t.dtype}")


def _bdl(t, name, io=None, shape=None, out=False):
    """(ptr, stride_b, stride_d) of a [B,D,L] tensor whose last axis is contiguous.  `shape`: the (B, D, L) every
    per-channel tensor of the call must have (the kernels index all of them with the same b, d, l; only a stride of
    0 may broadcast an input).  `out`: an output, whose rows must not overlap."""
    if t is None:
        return 0, 0, 0
    if t.shape == shape and t.dtype == io and t.is_contiguous():     # the common form, without a look at each axis
        s0, s1, _ = t.stride()
        return t.data_ptr(), s0, s1
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"{name}: expected [B,D,L] with contiguous time axis")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if out:
        # rows (b, d) of L elements at b * stride_b + d * stride_d: the axis with the smaller stride must step over a
        # whole row, the other one over all rows of the first (either axis may be the inner one)
        axes = sorted((t.stride(i), t.shape[i]) for i in (0, 1) if t.shape[i] > 1)
        need = t.shape[2]
        for stride, count in axes:
            if stride < need:
                raise ValueError(f"{name}: output rows overlap")
            need = stride * count
    if io is not None and t.dtype != io:
        raise TypeError(f"{name}: dtype {t.dtype} differs from the I/O dtype {io}")
    return t.data_ptr(), t.stride(0), t.stride(1)


def _f32c(t, name, shape):
    """Pointer of an optional contiguous float32 tensor."""
    if t is None:
        return 0
    if t.dtype != torch.float32 or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous float32 tensor")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _code(v, names):
    """A mode given by name or number; a number becomes 32 bits as the struct's field does."""
    return names[v] if isinstance(v, str) else _i32(int(v)).value


def _status_word(t):
    """Device pointer of an optional int32 status word (a one-element tensor the caller has cleared)."""
    if t is None:
        return None
    if t.dtype != torch.int32 or t.numel() != 1 or not t.is_cuda:
        raise ValueError("chain_status: expected a one-element int32 device tensor")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    """The current stream of the current device."""
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


def _entry(fn, native):
    name = fn.__name__
    Tensor = torch.Tensor

    def bad(v, dev):
        if not v.is_cuda:
            return TypeError(f"{name}: a tensor argument is on {v.device}; the scan library needs GPU tensors")
        return TypeError(f"{name}: tensors on different devices (cuda:{dev} and {v.device})")

    @functools.wraps(fn)
    def wrapper(*args, **kwargs):
        if native and _native is not None:
            res = getattr(_native, name)(args, kwargs)
            if res is not None:
                return res
        dev = -1
        for v in (*args, *kwargs.values()) if args else kwargs.values():
            if v is None or v.__class__ is str:
                continue
            if isinstance(v, Tensor):
                d = v.get_device()                    # -1 for a host tensor
                if d < 0 or (dev >= 0 and d != dev):
                    raise bad(v, dev)
                dev = d
            elif isinstance(v, dict):
                for t in v.values():
                    if isinstance(t, Tensor):
                        d = t.get_device()
                        if d < 0 or (dev >= 0 and d != dev):
                            raise bad(t, dev)
                        dev = d
        return fn(*args, **kwargs)
    return wrapper


def _device_checked(fn):
    """Every tensor argument of a compute entry point must live on ONE GPU: the library takes device pointers and
    has no CPU path, so a host tensor is refused here, before anything is launched.  (Kept cheap: the single-token
    step is called once per generated token.)"""
    return _entry(fn, native=False)


def _native_first(fn):
    """Calls in their usual form are taken by csrc/binding.cpp, without the checks and the marshalling below; everything
    else (None: nothing done) goes the general way, which is `__wrapped__`.  (One wrapper for both: with one around the other
    the trial cost a call that is not taken 0.3 to 0.7 us, 2 to 4 %, so 0.1 to 0.5.)"""
    wrapper = _entry(fn, native=True)
    wrapper.__wrapped__ = _device_checked(fn)
    return wrapper


def lrnnx_ckpt_interval() -> int:
    return int(lib().lrnnx_ckpt_interval())


def lrnnx_workspace_bytes(which, B, D, N, L, io_dtype, bc_groups=1, packed=False) -> int:
    return int(lib().lrnnx_workspace_bytes(which, B, D, N, L, io_dtype, bc_groups, int(bool(packed))))


def _check_cu(cu):
    """Number of sequences of a packed batch; cu is int64 [S+1] on the device."""
    if cu.dtype != torch.int64 or cu.dim() != 1 or not cu.is_contiguous() or not cu.is_cuda or cu.numel() < 2:
        raise ValueError("cu_seqlens: expected a contiguous int64 device tensor [S+1]")
    return cu.numel() - 1


def _bc_groups(Bm, Cm, io, Bsz, D, L, N):
    """Number of groups of the maps: [B,L,N] -> 1, [B,G,L,N] -> G (channel d reads group d // (D/G))."""
    one = (Bsz, L, N)
    if Bm.shape == one and Cm.shape == one and Bm.dtype == io and Cm.dtype == io and Bm.is_contiguous() and Cm.is_contiguous():
        return 1
    for name, t in (("Bm", Bm), ("Cm", Cm)):
        ok = t.dtype == io and t.is_contiguous() and t.shape == Bm.shape and (
            tuple(t.shape) == (Bsz, L, N) or (t.dim() == 4 and t.shape[0] == Bsz and tuple(t.shape[2:]) == (L, N)))
        if not ok:
            raise ValueError(f"{name}: expected contiguous [B,L,N] or [B,G,L,N] of dtype {io}")
    G = Bm.shape[1] if Bm.dim() == 4 else 1
    if D % G:
        raise ValueError("D must be a multiple of the number of Bm/Cm groups")
    return G


@_native_first
def lrnnx_selective_scan_fwd(u, delta, A, Bm, Cm, Dskip=None, delta_bias=None, z=None, x0=None,
                             disc="zoh_s6", delta_softplus=True, path="auto",
                             return_last_state=False, return_ckpt=False, out=None, ckpt_out=None, workspace=None,
                             cu_seqlens=None):
    """y (and optionally x_last, ckpt) of the forward selective scan; see lrnnx_ss_fwd_args.

    `out`, `ckpt_out` and `workspace` may supply preallocated buffers (ckpt_out implies return_ckpt).
    With `cu_seqlens` (int64 [S+1] on the device) the call is in packed variable-length mode: u, delta, z, y are
    [D,L], Bm and Cm [L,N] or [G,L,N], x0 and x_last [S,D,N]."""
    io = u.dtype
    packed = cu_seqlens is not None
    if packed:
        Bsz = _check_cu(cu_seqlens)
        u, delta, z, out = (None if t is None else t.unsqueeze(0) for t in (u, delta, z, out))
        Bm, Cm = Bm.unsqueeze(0), Cm.unsqueeze(0)
    Bio = 1 if packed else u.shape[0]                   # leading dimension of the I/O tensors and of the maps
    if not packed:
        Bsz = Bio
    _, D, L = u.shape
    N = A.shape[1]
    io_code = _io_dtype(u)
    disc, path = _code(disc, DISC), _code(path, PATH)
    bdl = (Bio, D, L)
    pu, u_sb, u_sd = _bdl(u, "u", io, bdl)
    pdelta, dl_sb, dl_sd = _bdl(delta, "delta", io, bdl)
    pz, z_sb, z_sd = _bdl(z, "z", io, bdl)
    pA = _f32c(A, "A", (D, N))
    groups = _bc_groups(Bm, Cm, io, Bio, D, L, N)
    pD, pbias = _f32c(Dskip, "Dskip", (D,)), _f32c(delta_bias, "delta_bias", (D,))
    px0 = _f32c(x0, "x0", (Bsz, D, N))
    y = out if out is not None else torch.empty(bdl, dtype=io, device=u.device)
    py, y_sb, y_sd = _bdl(y, "y", io, bdl, out=True)
    x_last = torch.empty((Bsz, D, N), dtype=torch.float32, device=u.device) if return_last_state else None
    ckpt, pck = ckpt_out, 0
    return_ckpt = return_ckpt or ckpt_out is not None
    if return_ckpt:
        I = lrnnx_ckpt_interval()
        ck_shape = (D, L // I + Bsz, N) if packed else (Bsz, D, (L + I - 1) // I, N)
        if ckpt is None:
            ckpt = torch.empty(ck_shape, dtype=torch.float32, device=u.device)
        pck = _f32c(ckpt, "ckpt_out", ck_shape)
    if workspace is None:
        nbytes = lrnnx_workspace_bytes(WS_FWD, Bsz, D, N, L, io_code, groups, packed)
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=u.device) if nbytes else None
    ws, ws_bytes = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())
    _check(_call("lrnnx_selective_scan_fwd", _pack_fwd(
        _FWD_SIZE, Bsz, D, N, groups, L, io_code, disc, bool(delta_softplus), path, cu_seqlens.data_ptr() if packed else 0,
        pu, u_sb, u_sd, pdelta, dl_sb, dl_sd, pA, Bm.data_ptr(), Cm.data_ptr(), pD, pbias, pz, z_sb, z_sd, px0,
        py, y_sb, y_sd, 0 if x_last is None else x_last.data_ptr(), pck, ws, ws_bytes, _stream())))
    res = (y[0] if packed else y,)
    if return_last_state:
        res += (x_last,)
    if return_ckpt:
        res += (ckpt,)
    return res[0] if len(res) == 1 else res


@_native_first
def lrnnx_selective_scan_fwd_complex(u, delta, A, Bm, Cm, Dskip=None, delta_bias=None, z=None, x0=None,
                                     disc="zoh_s6", delta_softplus=True, return_last_state=False, out=None,
                                     return_ckpt=False, ckpt_out=None, cu_seqlens=None, path="auto", workspace=None):
    """y (and optionally x_last, ckpt) of the forward selective scan with complex A, Bm, Cm; see
    lrnnx_ss_fwd_complex_args.  `ckpt_out`: a preallocated checkpoint array to fill (implies return_ckpt).

    A [D,N] complex64.  Bm, Cm [B,L,N]: complex64 for float32 I/O; for bfloat16 I/O a bfloat16 tensor [B,L,N,2]
    of (re, im) pairs.  x0, x_last [B,D,N] complex64; ckpt [B,D,ceil(L/interval),N] complex64.
    With `cu_seqlens` (int64 [S+1] on the device) the call is in packed variable-length mode: u, delta, z, y are
    [D,L], Bm and Cm [L,N] or [G,L,N] (plus the pair axis for bfloat16), x0 and x_last [S,D,N], ckpt
    [D, L // interval + S, N].  `path`: "auto", "single_pass" or "chunk_carry" (few rows, long sequences); `workspace`
    may supply the scratch buffer of the latter."""
    io = u.dtype
    packed = cu_seqlens is not None
    if packed:
        Bsz = _check_cu(cu_seqlens)
        u, delta, z, out = (None if t is None else t.unsqueeze(0) for t in (u, delta, z, out))
        Bm, Cm = Bm.unsqueeze(0), Cm.unsqueeze(0)
    Bio = 1 if packed else u.shape[0]                   # leading dimension of the I/O tensors and of the maps
    if not packed:
        Bsz = Bio
    _, D, L = u.shape
    N, G = _check_complex_maps(A, Bm, Cm, io, Bio, D, L)
    a = FwdComplexArgs()
    a.struct_size = ctypes.sizeof(FwdComplexArgs)
    a.B, a.D, a.N, a.L = Bsz, D, N, L
    a.bc_groups = G
    a.cu_seqlens = _ptr(cu_seqlens)
    a.io_dtype = _io_dtype(u)
    a.disc = DISC[disc] if isinstance(disc, str) else int(disc)
    a.delta_softplus = int(bool(delta_softplus))
    bdl = (Bio, D, L)
    a.u, a.u_stride_b, a.u_stride_d = _bdl(u, "u", io, bdl)
    a.delta, a.delta_stride_b, a.delta_stride_d = _bdl(delta, "delta", io, bdl)
    a.z, a.z_stride_b, a.z_stride_d = _bdl(z, "z", io, bdl)
    a.A, a.Bm, a.Cm = A.data_ptr(), Bm.data_ptr(), Cm.data_ptr()
    a.Dskip = _f32c(Dskip, "Dskip", (D,))
    a.delta_bias = _f32c(delta_bias, "delta_bias", (D,))
    if x0 is not None:
        if x0.dtype != torch.complex64 or not x0.is_contiguous() or tuple(x0.shape) != (Bsz, D, N):
            raise ValueError("x0: expected contiguous complex64 [B,D,N]")
        a.x0 = x0.data_ptr()
    y = out if out is not None else torch.empty((Bio, D, L), dtype=io, device=u.device)
    a.y, a.y_stride_b, a.y_stride_d = _bdl(y, "y", io, bdl, out=True)
    x_last = torch.empty((Bsz, D, N), dtype=torch.complex64, device=u.device) if return_last_state else None
    a.x_last = _ptr(x_last)
    ckpt = None
    if return_ckpt or ckpt_out is not None:
        I = lrnnx_ckpt_interval()
        shape = (D, L // I + Bsz, N) if packed else (Bsz, D, -(-L // I), N)
        ckpt = ckpt_out if ckpt_out is not None else torch.empty(shape, dtype=torch.complex64, device=u.device)
        if ckpt.dtype != torch.complex64 or not ckpt.is_contiguous() or tuple(ckpt.shape) != shape:
            raise ValueError(f"ckpt_out: expected contiguous complex64 {shape}")
        a.ckpt = ckpt.data_ptr()
        return_ckpt = True
    a.path = PATH[path] if isinstance(path, str) else int(path)
    if workspace is None:
        nbytes = lrnnx_workspace_bytes(WS_FWD_COMPLEX, Bsz, D, N, L, a.io_dtype, G, packed)
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=u.device)
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    a.stream = _stream()
    _check(lib().lrnnx_selective_scan_fwd_complex(ctypes.byref(a)))
    res = (y[0] if packed else y,) + ((x_last,) if return_last_state else ()) + ((ckpt,) if return_ckpt else ())
    return res if len(res) > 1 else y


def _check_complex_maps(A, Bm, Cm, io, Bsz, D, L):
    """Validate A [D,N] complex64 and the complex maps for this I/O type ([B,L,N], or [B,G,L,N] with G groups; the
    bfloat16 form has a trailing axis of (re, im) pairs); returns (N, G)."""
    if A.dtype != torch.complex64 or A.dim() != 2 or A.shape[0] != D or not A.is_contiguous():
        raise ValueError("A: expected contiguous complex64 [D,N]")
    N = A.shape[1]
    G = None
    for name, t in (("Bm", Bm), ("Cm", Cm)):
        shape = tuple(t.shape)
        if io == torch.bfloat16:
            ok = t.dtype == torch.bfloat16 and shape[-1:] == (2,)
            shape = shape[:-1]
        else:
            ok = io == torch.float32 and t.dtype == torch.complex64
        ok = ok and t.is_contiguous() and (shape == (Bsz, L, N) or (len(shape) == 4 and shape[0] == Bsz and shape[2:] == (L, N)))
        g = shape[1] if ok and len(shape) == 4 else 1
        if not ok or (G is not None and g != G):
            raise ValueError(f"{name}: expected contiguous complex64 [B,L,N] or [B,G,L,N] (float32 I/O), or bfloat16 "
                             "with a trailing (re, im) axis")
        G = g
    if D % G:
        raise ValueError("D must be a multiple of the number of Bm/Cm groups")
    return N, G


@_native_first
def lrnnx_selective_scan_bwd_complex(u, delta, A, Bm, Cm, dy, Dskip=None, delta_bias=None, z=None, x0=None,
                                     ckpt=None, disc="zoh_s6", delta_softplus=True, want_dx0=False, outs=None,
                                     workspace=None, cu_seqlens=None, path="auto", max_seqlen=None):
    """Gradients of sum(dy*y) of the complex-A selective scan as a dict; see lrnnx_ss_bwd_complex_args.
    dA [D,N], dBm, dCm [B,L,N], dx0 [B,D,N] are complex64 (dLoss/dRe + i dLoss/dIm); du, ddelta, dz in the I/O
    type; dD, dbias float32.  `ckpt`: the checkpoints a forward call returned (else they are recomputed).
    `cu_seqlens`: packed variable-length mode as in the forward call (du, ddelta, dz are [D,L]; dBm, dCm [L,N] or
    [G,L,N]; dx0 [S,D,N]).  `path`: "auto", "single_pass" or "chunk_carry" as for the real scan.  `max_seqlen`: as
    for the real scan."""
    io = u.dtype
    packed = cu_seqlens is not None
    if packed:
        Bsz = _check_cu(cu_seqlens)
        u, delta, z, dy = (None if t is None else t.unsqueeze(0) for t in (u, delta, z, dy))
        Bm, Cm = Bm.unsqueeze(0), Cm.unsqueeze(0)
    Bio = 1 if packed else u.shape[0]
    if not packed:
        Bsz = Bio
    _, D, L = u.shape
    N, G = _check_complex_maps(A, Bm, Cm, io, Bio, D, L)
    dev = u.device
    outs = dict(outs or {})
    if packed:                                          # caller-supplied outputs are in the packed shapes
        outs = {k: (v.unsqueeze(0) if k in ("du", "ddelta", "dz", "dBm", "dCm") else v) for k, v in outs.items()}

    def new(name, shape, dtype):
        if name not in outs:
            outs[name] = torch.empty(shape, dtype=dtype, device=dev)
        t = outs[name]
        strided_ok = name in ("du", "ddelta", "dz")          # [B,D,L] outputs are passed with their strides
        if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not (strided_ok or t.is_contiguous()):
            raise ValueError(f"{name}: expected {dtype} {tuple(shape)}" + ("" if strided_ok else ", contiguous"))
        return t

    a = BwdComplexArgs()
    a.struct_size = ctypes.sizeof(BwdComplexArgs)
    a.B, a.D, a.N, a.L = Bsz, D, N, L
    a.bc_groups = G
    a.cu_seqlens = _ptr(cu_seqlens)
    a.max_seqlen = 0 if max_seqlen is None else int(max_seqlen)
    a.path = PATH[path] if isinstance(path, str) else int(path)
    a.io_dtype = _io_dtype(u)
    a.disc = DISC[disc] if isinstance(disc, str) else int(disc)
    a.delta_softplus = int(bool(delta_softplus))
    bdl = (Bio, D, L)
    a.u, a.u_stride_b, a.u_stride_d = _bdl(u, "u", io, bdl)
    a.delta, a.delta_stride_b, a.delta_stride_d = _bdl(delta, "delta", io, bdl)
    a.z, a.z_stride_b, a.z_stride_d = _bdl(z, "z", io, bdl)
    a.dy, a.dy_stride_b, a.dy_stride_d = _bdl(dy, "dy", io, bdl)
    a.A, a.Bm, a.Cm = A.data_ptr(), Bm.data_ptr(), Cm.data_ptr()
    a.Dskip = _f32c(Dskip, "Dskip", (D,))
    a.delta_bias = _f32c(delta_bias, "delta_bias", (D,))
    I = lrnnx_ckpt_interval()
    ck_shape = (D, L // I + Bsz, N) if packed else (Bsz, D, -(-L // I), N)
    for name, t, shape in (("x0", x0, (Bsz, D, N)), ("ckpt", ckpt, ck_shape)):
        if t is not None:
            if t.dtype != torch.complex64 or not t.is_contiguous() or tuple(t.shape) != shape:
                raise ValueError(f"{name}: expected contiguous complex64 {shape}")
            setattr(a, name, t.data_ptr())
    a.du, a.du_stride_b, a.du_stride_d = _bdl(new("du", bdl, io), "du", io, bdl, out=True)
    a.ddelta, a.ddelta_stride_b, a.ddelta_stride_d = _bdl(new("ddelta", bdl, io), "ddelta", io, bdl, out=True)
    if z is not None:
        a.dz, a.dz_stride_b, a.dz_stride_d = _bdl(new("dz", bdl, io), "dz", io, bdl, out=True)
    c64 = torch.complex64
    a.dA = new("dA", (D, N), c64).data_ptr()
    map_shape = (Bio, L, N) if (Bm.dim() == 3 + (io == torch.bfloat16)) else (Bio, G, L, N)
    a.dBm = new("dBm", map_shape, c64).data_ptr()
    a.dCm = new("dCm", map_shape, c64).data_ptr()
    if Dskip is not None:
        a.dD = new("dD", (D,), torch.float32).data_ptr()
    if delta_bias is not None:
        a.dbias = new("dbias", (D,), torch.float32).data_ptr()
    if want_dx0:
        a.dx0 = new("dx0", (Bsz, D, N), c64).data_ptr()
    if workspace is None:
        # with the forward's checkpoints only the chunk aggregates (or the launch order of a packed batch) and the sums of
        # dBm and dCm are needed
        nbytes = lrnnx_workspace_bytes(WS_BWD_COMPLEX, Bsz, D, N, L, a.io_dtype, G, packed)
        if ckpt is not None:
            nbytes -= (ckpt.numel() * 8 + 255) // 256 * 256
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    if workspace is not None:
        a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    a.stream = _stream()
    _check(lib().lrnnx_selective_scan_bwd_complex(ctypes.byref(a)))
    if packed:
        outs = {k: (v[0] if k in ("du", "ddelta", "dz", "dBm", "dCm") else v) for k, v in outs.items()}
    return outs


@_native_first
def lrnnx_selective_scan_bwd(u, delta, A, Bm, Cm, dy, Dskip=None, delta_bias=None, z=None, x0=None,
                             ckpt=None, disc="zoh_s6", delta_softplus=True, want_dx0=False,
                             outs=None, workspace=None, cu_seqlens=None, path="auto", max_seqlen=None):
    """Gradients of sum(dy*y) as a dict; see lrnnx_ss_bwd_args.  `outs` may supply preallocated outputs.
    `cu_seqlens`: packed variable-length mode as in the forward call (du, ddelta, dz are [D,L]; dBm, dCm as Bm).
    `path`: "auto", "single_pass" or "chunk_carry" (time axis cut into chunks that run side by side).
    `max_seqlen`: packed mode, the longest sequence of the batch if the host knows it (a hint for the launch shape
    that keeps one long sequence from setting the time of the whole launch, and lets "auto" cut a few long sequences
    into chunks; the lengths themselves stay on the device)."""
    io = u.dtype
    packed = cu_seqlens is not None
    if packed:
        Bsz = _check_cu(cu_seqlens)
        u, delta, z, dy = (None if t is None else t.unsqueeze(0) for t in (u, delta, z, dy))
        Bm, Cm = Bm.unsqueeze(0), Cm.unsqueeze(0)
    Bio = 1 if packed else u.shape[0]
    if not packed:
        Bsz = Bio
    _, D, L = u.shape
    N = A.shape[1]
    dev = u.device
    outs = dict(outs or {})
    if packed:                                          # caller-supplied outputs are in the packed shapes
        outs = {k: (v.unsqueeze(0) if k in ("du", "ddelta", "dz", "dBm", "dCm") else v) for k, v in outs.items()}

    def new(name, shape, dtype):
        if name not in outs:
            outs[name] = torch.empty(shape, dtype=dtype, device=dev)
        t = outs[name]
        strided_ok = name in ("du", "ddelta", "dz")          # [B,D,L] outputs are passed with their strides
        if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not (strided_ok or t.is_contiguous()):
            raise ValueError(f"{name}: expected {dtype} {tuple(shape)}" + ("" if strided_ok else ", contiguous"))
        return t

    io_code = _io_dtype(u)
    max_seqlen = 0 if max_seqlen is None else _i64(int(max_seqlen)).value
    path, disc = _code(path, PATH), _code(disc, DISC)
    bdl = (Bio, D, L)
    pu, u_sb, u_sd = _bdl(u, "u", io, bdl)
    pdelta, dl_sb, dl_sd = _bdl(delta, "delta", io, bdl)
    pz, z_sb, z_sd = _bdl(z, "z", io, bdl)
    pdy, dy_sb, dy_sd = _bdl(dy, "dy", io, bdl)
    pA = _f32c(A, "A", (D, N))
    groups = _bc_groups(Bm, Cm, io, Bio, D, L, N)
    pD, pbias = _f32c(Dskip, "Dskip", (D,)), _f32c(delta_bias, "delta_bias", (D,))
    px0 = _f32c(x0, "x0", (Bsz, D, N))
    I = lrnnx_ckpt_interval()
    pck = _f32c(ckpt, "ckpt", (D, L // I + Bsz, N) if packed else (Bsz, D, -(-L // I), N))
    pdu, du_sb, du_sd = _bdl(new("du", bdl, io), "du", io, bdl, out=True)
    pdd, dd_sb, dd_sd = _bdl(new("ddelta", bdl, io), "ddelta", io, bdl, out=True)
    pdz, dz_sb, dz_sd = _bdl(new("dz", bdl, io), "dz", io, bdl, out=True) if z is not None else (0, 0, 0)
    f32 = torch.float32
    pdA = new("dA", (D, N), f32).data_ptr()
    pdB, pdC = new("dBm", Bm.shape, f32).data_ptr(), new("dCm", Cm.shape, f32).data_ptr()
    pdD = new("dD", (D,), f32).data_ptr() if Dskip is not None else 0
    pdbias = new("dbias", (D,), f32).data_ptr() if delta_bias is not None else 0
    pdx0 = new("dx0", (Bsz, D, N), f32).data_ptr() if want_dx0 else 0

    def args(ws, ws_bytes, stream):
        return _pack_bwd(
            _BWD_SIZE, Bsz, D, N, groups, L, io_code, disc, bool(delta_softplus), path, cu_seqlens.data_ptr() if packed else 0,
            max_seqlen, pu, u_sb, u_sd, pdelta, dl_sb, dl_sd, pA, Bm.data_ptr(), Cm.data_ptr(), pD, pbias, pz, z_sb, z_sd, px0,
            pdy, dy_sb, dy_sd, pck, pdu, du_sb, du_sd, pdd, dd_sb, dd_sd, pdz, dz_sb, dz_sd,
            pdA, pdB, pdC, pdD, pdbias, pdx0, ws, ws_bytes, stream)

    if workspace is None:
        nbytes = _call("lrnnx_selective_scan_bwd_workspace_bytes", args(0, 0, 0))
        if nbytes:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    ws, ws_bytes = (0, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())
    _check(_call("lrnnx_selective_scan_bwd", args(ws, ws_bytes, _stream())))
    if packed:
        outs = {k: (v[0] if k in ("du", "ddelta", "dz", "dBm", "dCm") else v) for k, v in outs.items()}
    return outs


@_native_first
def lrnnx_lti_diag_scan(lam, v, x0=None, return_last_state=False, out=None, workspace=None, path="auto",
                        chain_status=None):
    """x [B,L,P] complex64 of x_k = lam * x_{k-1} + v_k; see lrnnx_lti_args.  `chain_status`: an int32 device word the
    library sets to 1 should a bounded wait between workgroups ever run out (clear it first)."""
    if v.dtype != torch.complex64 or lam.dtype != torch.complex64:
        raise TypeError("lam and v must be complex64")
    if not v.is_contiguous() or not lam.is_contiguous():
        raise ValueError("lam and v must be contiguous")
    Bsz, L, P = v.shape
    if tuple(lam.shape) != (P,):
        raise ValueError(f"lam: expected shape ({P},), got {tuple(lam.shape)}")
    if out is not None and (out.dtype != torch.complex64 or not out.is_contiguous() or out.shape != v.shape):
        raise ValueError("out: expected a contiguous complex64 tensor of the shape of v")
    a = LtiArgs()
    a.struct_size = ctypes.sizeof(LtiArgs)
    a.B, a.P, a.L = Bsz, P, L
    a.path = PATH[path] if isinstance(path, str) else int(path)
    a.lambda_, a.v = lam.data_ptr(), v.data_ptr()
    if x0 is not None:
        if x0.dtype != torch.complex64 or not x0.is_contiguous() or tuple(x0.shape) != (Bsz, P):
            raise ValueError("x0: expected contiguous complex64 [B,P]")
        a.x0 = x0.data_ptr()
    x = out if out is not None else torch.empty_like(v)
    a.x = x.data_ptr()
    x_last = torch.empty((Bsz, P), dtype=torch.complex64, device=v.device) if return_last_state else None
    a.x_last = _ptr(x_last)
    a.chain_status = _status_word(chain_status)
    if workspace is None:
        nbytes = lrnnx_workspace_bytes(WS_LTI, Bsz, P, 0, L, 0)
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=v.device)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    a.stream = _stream()
    _check(lib().lrnnx_lti_diag_scan(ctypes.byref(a)))
    return (x, x_last) if return_last_state else x


@_device_checked
def lrnnx_lti_diag_scan_static(lam, v, out, x0=None, x_last_out=None):
    """The LTI scan on the library's own static scratch array: no workspace is passed and the C call allocates
    nothing; see lrnnx_lti_diag_scan_static.  The caller supplies every buffer: `out` [B,L,P] complex64 (may be v
    itself) and optionally `x_last_out` [B,P].  Returns `out`."""
    for name, t in (("lam", lam), ("v", v), ("out", out)):
        if t.dtype != torch.complex64 or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous complex64")
    Bsz, L, P = v.shape
    if tuple(out.shape) != (Bsz, L, P) or tuple(lam.shape) != (P,):
        raise ValueError("shape mismatch between lam [P], v and out [B,L,P]")
    a = LtiArgs()
    a.struct_size = ctypes.sizeof(LtiArgs)
    a.B, a.P, a.L = Bsz, P, L
    a.path = PATH["auto"]
    a.lambda_, a.v, a.x = lam.data_ptr(), v.data_ptr(), out.data_ptr()
    for name, t in (("x0", x0), ("x_last_out", x_last_out)):
        if t is not None and (t.dtype != torch.complex64 or not t.is_contiguous() or tuple(t.shape) != (Bsz, P)):
            raise ValueError(f"{name}: expected contiguous complex64 [B,P]")
    a.x0, a.x_last = _ptr(x0), _ptr(x_last_out)
    a.stream = _stream()
    _check(lib().lrnnx_lti_diag_scan_static(ctypes.byref(a)))
    return out


@_native_first
def lrnnx_lti_diag_scan_bwd(lam, x, gx, x0=None, want_dx0=True, out=None, workspace=None, chain_status=None):
    """(dv [B,L,P], dlam [P], dx0 [B,P] or None) from the saved states x and the incoming gradient gx;
    see lrnnx_lti_bwd_args."""
    for t, name in ((lam, "lam"), (x, "x"), (gx, "gx")):
        if t.dtype != torch.complex64 or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous complex64")
    Bsz, L, P = x.shape
    if tuple(gx.shape) != (Bsz, L, P) or tuple(lam.shape) != (P,):
        raise ValueError("shape mismatch between lam [P], x and gx [B,L,P]")
    a = LtiBwdArgs()
    a.struct_size = ctypes.sizeof(LtiBwdArgs)
    a.B, a.P, a.L = Bsz, P, L
    a.lambda_, a.x, a.gx = lam.data_ptr(), x.data_ptr(), gx.data_ptr()
    if x0 is not None:
        if x0.dtype != torch.complex64 or not x0.is_contiguous() or tuple(x0.shape) != (Bsz, P):
            raise ValueError("x0: expected contiguous complex64 [B,P]")
        a.x0 = x0.data_ptr()
    if out is not None and (out.dtype != torch.complex64 or not out.is_contiguous() or out.shape != gx.shape):
        raise ValueError("out: expected a contiguous complex64 tensor of the shape of gx")
    dv = out if out is not None else torch.empty_like(gx)
    dlam = torch.empty(P, dtype=torch.complex64, device=x.device)
    dx0 = torch.empty((Bsz, P), dtype=torch.complex64, device=x.device) if want_dx0 else None
    a.dv, a.dlambda, a.dx0 = dv.data_ptr(), dlam.data_ptr(), _ptr(dx0)
    a.chain_status = _status_word(chain_status)
    if workspace is None:
        nbytes = lrnnx_workspace_bytes(WS_LTI_BWD, Bsz, P, 0, L, 0)
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=x.device)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    a.stream = _stream()
    _check(lib().lrnnx_lti_diag_scan_bwd(ctypes.byref(a)))
    return dv, dlam, dx0


@_native_first
def lrnnx_diag_scan(a, b, x0=None, return_last_state=False, out=None, workspace=None, chain_status=None):
    """x [B,L,P] of x_k = a_k * x_{k-1} + b_k for float32 or complex64 a, b; see lrnnx_diag_scan_args."""
    if a.dtype not in (torch.float32, torch.complex64) or b.dtype != a.dtype:
        raise TypeError("a and b must both be float32 or both complex64")
    if not a.is_contiguous() or not b.is_contiguous() or a.shape != b.shape or b.dim() != 3:
        raise ValueError("a and b must be contiguous [B,L,P] tensors of one shape")
    Bsz, L, P = b.shape
    dt = C64 if a.dtype == torch.complex64 else F32
    g = DiagScanArgs()
    g.struct_size = ctypes.sizeof(DiagScanArgs)
    g.B, g.P, g.L, g.dtype = Bsz, P, L, dt
    g.a, g.b = a.data_ptr(), b.data_ptr()
    if x0 is not None:
        if x0.dtype != a.dtype or not x0.is_contiguous() or tuple(x0.shape) != (Bsz, P):
            raise ValueError("x0: expected a contiguous [B,P] tensor of the dtype of a")
        g.x0 = x0.data_ptr()
    if out is not None and (out.dtype != b.dtype or not out.is_contiguous() or out.shape != b.shape):
        raise ValueError("out: expected a contiguous tensor of the dtype and shape of b")
    x = out if out is not None else torch.empty_like(b)
    g.x = x.data_ptr()
    x_last = torch.empty((Bsz, P), dtype=a.dtype, device=b.device) if return_last_state else None
    g.x_last = _ptr(x_last)
    g.chain_status = _status_word(chain_status)
    if workspace is None:
        nbytes = lrnnx_workspace_bytes(WS_DIAG, Bsz, P, 0, L, dt)
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=b.device)
    g.workspace, g.workspace_bytes = workspace.data_ptr(), workspace.numel()
    g.stream = _stream()
    _check(lib().lrnnx_diag_scan(ctypes.byref(g)))
    return (x, x_last) if return_last_state else x


@_native_first
def lrnnx_diag_scan_bwd(a, x, gx, x0=None, want_dx0=True, workspace=None, chain_status=None):
    """(da, db [B,L,P], dx0 [B,P] or None) from the forward call's a, saved states x and the incoming gradient gx;
    see lrnnx_diag_scan_bwd_args."""
    for t, name in ((a, "a"), (x, "x"), (gx, "gx")):
        if t.dtype != a.dtype or not t.is_contiguous() or t.shape != a.shape:
            raise ValueError(f"{name}: expected a contiguous tensor of the dtype and shape of a")
    if a.dtype not in (torch.float32, torch.complex64) or a.dim() != 3:
        raise TypeError("a must be a float32 or complex64 [B,L,P] tensor")
    Bsz, L, P = a.shape
    dt = C64 if a.dtype == torch.complex64 else F32
    g = DiagScanBwdArgs()
    g.struct_size = ctypes.sizeof(DiagScanBwdArgs)
    g.B, g.P, g.L, g.dtype = Bsz, P, L, dt
    g.a, g.x, g.gx = a.data_ptr(), x.data_ptr(), gx.data_ptr()
    if x0 is not None:
        if x0.dtype != a.dtype or not x0.is_contiguous() or tuple(x0.shape) != (Bsz, P):
            raise ValueError("x0: expected a contiguous [B,P] tensor of the dtype of a")
        g.x0 = x0.data_ptr()
    da, db = torch.empty_like(a), torch.empty_like(a)
    dx0 = torch.empty((Bsz, P), dtype=a.dtype, device=a.device) if want_dx0 else None
    g.da, g.db, g.dx0 = da.data_ptr(), db.data_ptr(), _ptr(dx0)
    g.chain_status = _status_word(chain_status)
    if workspace is None:
        nbytes = lrnnx_workspace_bytes(WS_DIAG_BWD, Bsz, P, 0, L, dt)
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=a.device)
    g.workspace, g.workspace_bytes = workspace.data_ptr(), workspace.numel()
    g.stream = _stream()
    _check(lib().lrnnx_diag_scan_bwd(ctypes.byref(g)))
    return da, db, dx0


def _bd(t, name, io):
    """(ptr, stride_b, stride_d) of a [B,D] tensor (any strides)."""
    if t is None:
        return 0, 0, 0
    if t.dim() != 2 or t.dtype != io:
        raise ValueError(f"{name}: expected a [B,D] tensor of dtype {io}")
    return t.data_ptr(), *t.stride()


@_native_first
def lrnnx_selective_step(x, u, delta, A, Bm, Cm, Dskip=None, delta_bias=None, z=None,
                         disc="zoh_s6", delta_softplus=True, out=None):
    """One token: updates the state x [B,D,N] in place and returns y [B,D]; see lrnnx_ss_step_args."""
    io = u.dtype
    Bsz, D, N = x.shape
    px = _f32c(x, "x", (Bsz, D, N))
    io_code, disc = _io_dtype(u), _code(disc, DISC)
    pu, u_sb, u_sd = _bd(u, "u", io)
    pdelta, dl_sb, dl_sd = _bd(delta, "delta", io)
    pz, z_sb, z_sd = _bd(z, "z", io)
    pA = _f32c(A, "A", (D, N))
    groups, one = 1, (Bsz, N)
    if not (Bm.shape == one and Cm.shape == one and Bm.dtype == io and Cm.dtype == io and Bm.is_contiguous() and Cm.is_contiguous()):
        for name, t in (("Bm", Bm), ("Cm", Cm)):
            ok = t.dtype == io and t.is_contiguous() and t.shape == Bm.shape and (
                t.shape == one or (t.dim() == 3 and t.shape[0] == Bsz and t.shape[2] == N))
            if not ok:
                raise ValueError(f"{name}: expected contiguous [B,N] or [B,G,N] of dtype {io}")
        groups = Bm.shape[1] if Bm.dim() == 3 else 1
        if D % groups:
            raise ValueError("D must be a multiple of the number of Bm/Cm groups")
    pD, pbias = _f32c(Dskip, "Dskip", (D,)), _f32c(delta_bias, "delta_bias", (D,))
    y = out if out is not None else torch.empty((Bsz, D), dtype=io, device=u.device)
    py, y_sb, y_sd = _bd(y, "y", io)
    _check(_call("lrnnx_selective_step", _pack_step(
        _STEP_SIZE, Bsz, D, N, groups, io_code, disc, bool(delta_softplus), 0, px,
        pu, u_sb, u_sd, pdelta, dl_sb, dl_sd, pA, Bm.data_ptr(), Cm.data_ptr(), pD, pbias, pz, z_sb, z_sd,
        py, y_sb, y_sd, _stream())))
    return y


@_native_first
def lrnnx_selective_step_complex(x, u, delta, A, Bm, Cm, Dskip=None, delta_bias=None, z=None,
                                 disc="zoh_s6", delta_softplus=True, out=None):
    """One token of the complex-A scan: updates the state x [B,D,N] complex64 in place and returns y [B,D]; see
    lrnnx_ss_step_complex_args.  Bm, Cm [B,N]: complex64 (float32 I/O) or bfloat16 [B,N,2] (re, im) pairs."""
    io = u.dtype
    if x.dtype != torch.complex64 or x.dim() != 3 or not x.is_contiguous():
        raise ValueError("x: expected contiguous complex64 [B,D,N]")
    Bsz, D, N = x.shape
    if A.dtype != torch.complex64 or tuple(A.shape) != (D, N) or not A.is_contiguous():
        raise ValueError("A: expected contiguous complex64 [D,N]")
    G = None
    for name, t in (("Bm", Bm), ("Cm", Cm)):
        shape = tuple(t.shape)
        if io == torch.bfloat16:
            ok = t.dtype == torch.bfloat16 and shape[-1:] == (2,)
            shape = shape[:-1]
        else:
            ok = io == torch.float32 and t.dtype == torch.complex64
        ok = ok and t.is_contiguous() and (shape == (Bsz, N) or (len(shape) == 3 and shape[0] == Bsz and shape[2] == N))
        g = shape[1] if ok and len(shape) == 3 else 1
        if not ok or (G is not None and g != G):
            raise ValueError(f"{name}: expected contiguous complex64 [B,N] or [B,G,N] (float32 I/O), or bfloat16 with a "
                             "trailing (re, im) axis")
        G = g
    if D % G:
        raise ValueError("D must be a multiple of the number of Bm/Cm groups")
    a = StepComplexArgs()
    a.struct_size = ctypes.sizeof(StepComplexArgs)
    a.B, a.D, a.N = Bsz, D, N
    a.bc_groups = G
    a.io_dtype = _io_dtype(u)
    a.disc = DISC[disc] if isinstance(disc, str) else int(disc)
    a.delta_softplus = int(bool(delta_softplus))
    a.x = x.data_ptr()
    a.u, a.u_stride_b, a.u_stride_d = _bd(u, "u", io)
    a.delta, a.delta_stride_b, a.delta_stride_d = _bd(delta, "delta", io)
    a.z, a.z_stride_b, a.z_stride_d = _bd(z, "z", io)
    a.A, a.Bm, a.Cm = A.data_ptr(), Bm.data_ptr(), Cm.data_ptr()
    a.Dskip = _f32c(Dskip, "Dskip", (D,))
    a.delta_bias = _f32c(delta_bias, "delta_bias", (D,))
    y = out if out is not None else torch.empty((Bsz, D), dtype=io, device=u.device)
    a.y, a.y_stride_b, a.y_stride_d = _bd(y, "y", io)
    a.stream = _stream()
    _check(lib().lrnnx_selective_step_complex(ctypes.byref(a)))
    return y


@_device_checked
def lrnnx_lti_step(lam, x, v):
    """One token of the LTI recurrence: x [B,P] complex64 is updated in place and returned."""
    for name, t in (("lam", lam), ("x", x), ("v", v)):
        if t.dtype != torch.complex64 or not t.is_contiguous():
            raise TypeError(f"{name}: expected contiguous complex64")
    Bsz, P = x.shape
    a = LtiStepArgs()
    a.struct_size = ctypes.sizeof(LtiStepArgs)
    a.B, a.P = Bsz, P
    a.lambda_, a.x, a.v = lam.data_ptr(), x.data_ptr(), v.data_ptr()
    a.stream = _stream()
    _check(lib().lrnnx_lti_step(ctypes.byref(a)))
    return x


# ---------------------------------------------------------------- gated delta rule
_DELTA_FWD_SIZE, _DELTA_BWD_SIZE, _DELTA_STEP_SIZE = (ctypes.sizeof(c) for c in (DeltaFwdArgs, DeltaBwdArgs, DeltaStepArgs))
_NORM_FWD_SIZE, _NORM_BWD_SIZE = ctypes.sizeof(NormFwdArgs), ctypes.sizeof(NormBwdArgs)


def _rows(t, name, shape, dtype):
    """(ptr, strides) of a tensor with a contiguous last axis; `shape` with that axis."""
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    *st, last = t.stride()
    if last != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: expected a contiguous last axis")
    return (t.data_ptr(), *st)


def _gates(g, beta, shape, io):
    """(gate code, (ptr, strides) of g, of beta): float32, or the I/O type."""
    if g.dtype != beta.dtype or g.dtype not in (torch.float32, io):
        raise TypeError(f"g, beta: expected both float32 or both {io}, got {g.dtype} and {beta.dtype}")
    for t, name in ((g, "g"), (beta, "beta")):
        if t.shape != shape:
            raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return BF16 if g.dtype == torch.bfloat16 else F32, (g.data_ptr(), *g.stride()), (beta.data_ptr(), *beta.stride())


def _out_rows(t, name, shape, dtype):
    """(ptr, strides) of an output whose rows must not overlap."""
    r = _rows(t, name, shape, dtype)
    need = shape[-1]
    for stride, count in sorted(zip(r[1:], shape[:-1])):
        if count > 1:
            if stride < need:
                raise ValueError(f"{name}: output rows overlap")
            need += stride * (count - 1)
    return r


def _delta_head(q, k, v, cu_seqlens, scale):
    """What the calls over a sequence have in common; the packed form gets a batch axis of one."""
    if q.dim() != (4 if cu_seqlens is None else 3) or k.dim() != q.dim() or v.dim() != q.dim():
        raise ValueError("q, k, v: expected [B,L,H,d], or [L,H,d] with cu_seqlens")
    S = _check_cu(cu_seqlens) if cu_seqlens is not None else None
    if S is not None:
        q, k, v = q.unsqueeze(0), k.unsqueeze(0), v.unsqueeze(0)
    lead, (Hk, dk), (Hv, dv) = q.shape[:2], q.shape[2:], v.shape[2:]
    if scale is None:
        scale = dk ** -0.5
    return q, k, v, lead, S if S is not None else lead[0], Hk, Hv, dk, dv, float(scale)


def _delta_inputs(q, k, v, g, beta, s0, lead, B, Hk, Hv, dk, dv, io, packed):
    if packed:
        g, beta = g.unsqueeze(0), beta.unsqueeze(0)
    gate, g, beta = _gates(g, beta, (*lead, Hv), io)
    return gate, (*_rows(q, "q", (*lead, Hk, dk), io), *_rows(k, "k", (*lead, Hk, dk), io), *_rows(v, "v", (*lead, Hv, dv), io),
                  *g, *beta, _f32c(s0, "s0", (B, Hv, dk, dv)))


def _scratch(workspace, nbytes, device, name="workspace"):
    if workspace is None:
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous uint8 tensor")
    return workspace


@_native_first
def lrnnx_gated_delta_fwd(q, k, v, g, beta, scale=None, s0=None, cu_seqlens=None, return_last_state=False, return_saved=False,
                          out=None, workspace=None):
    """o [B,L,Hv,dv] of the gated delta rule, and optionally the last state [B,Hv,dk,dv] float32 and `saved`, the opaque
    buffer that lrnnx_gated_delta_bwd takes; see lrnnx_delta_fwd_args.

    q, k [B,L,Hk,dk], v [B,L,Hv,dv] float32 or bfloat16, any strides with a contiguous last axis; g (log decay), beta
    [B,L,Hv] float32 or the I/O type (`saved` is then float32, or with bfloat16 gates 16 bits); scale: dk ** -0.5 by default.  With `cu_seqlens` (int64 [S+1] on the device) the
    batch is packed: q, k, v, g, beta, o without the batch axis, s0 and the last state [S,Hv,dk,dv]; rows of o outside every
    sequence are not written (a new o holds anything there)."""
    packed, io = cu_seqlens is not None, v.dtype
    q, k, v, lead, B, Hk, Hv, dk, dv, scale = _delta_head(q, k, v, cu_seqlens, scale)
    code = _io_dtype(v)
    gate, inputs = _delta_inputs(q, k, v, g, beta, s0, lead, B, Hk, Hv, dk, dv, io, packed)
    o = torch.empty((*lead, Hv, dv), dtype=io, device=v.device) if out is None else out.unsqueeze(0) if packed else out
    po = _out_rows(o, "out", (*lead, Hv, dv), io)
    s_last = torch.empty((B, Hv, dk, dv), dtype=torch.float32, device=v.device) if return_last_state else None
    head = (_DELTA_FWD_SIZE, B, Hk, Hv, dk, dv, code, gate, scale, lead[1], cu_seqlens.data_ptr() if packed else 0, *inputs, *po,
            0 if s_last is None else s_last.data_ptr())
    saved, psaved, nsaved = None, 0, 0
    if _lib is None:
        lib()
    if return_saved:
        nsaved = _call("lrnnx_gated_delta_saved_bytes", _pack_delta_fwd(*head, 0, 0, 0, 0, 0))
        saved = torch.empty(max(nsaved, 16), dtype=torch.uint8, device=v.device)
        psaved = saved.data_ptr()
    workspace = _scratch(workspace, 0 if workspace is not None else
                         _call("lrnnx_gated_delta_fwd_workspace_bytes", _pack_delta_fwd(*head, psaved, nsaved, 0, 0, 0)), v.device)
    _check(_call("lrnnx_gated_delta_fwd", _pack_delta_fwd(*head, psaved, nsaved, workspace.data_ptr(), workspace.numel(), _stream())))
    res = (o[0] if packed else o,) + ((s_last,) if return_last_state else ()) + ((saved,) if return_saved else ())
    return res[0] if len(res) == 1 else res


@_native_first
def lrnnx_gated_delta_bwd(q, k, v, g, beta, do, saved, scale=None, s0=None, ds_last=None, want_ds0=False, cu_seqlens=None,
                          workspace=None):
    """Gradients of sum(do * o) (and sum(ds_last * s_last)) as a dict: dq, dk, dv in the I/O type, dg, dbeta in the gates'
    type, ds0 float32 if wanted; see lrnnx_delta_bwd_args.  Inputs, scale, s0 and cu_seqlens as in the forward call that
    returned `saved`.  Gradients of steps outside every sequence of a packed batch are zeros."""
    packed, io = cu_seqlens is not None, v.dtype
    gdt, device = g.dtype, v.device
    q, k, v, lead, B, Hk, Hv, dk, dv, scale = _delta_head(q, k, v, cu_seqlens, scale)
    code = _io_dtype(v)
    gate, inputs = _delta_inputs(q, k, v, g, beta, s0, lead, B, Hk, Hv, dk, dv, io, packed)
    pdo = _rows(do.unsqueeze(0) if packed else do, "do", (*lead, Hv, dv), io)
    if saved.dtype != torch.uint8 or not saved.is_contiguous():
        raise TypeError("saved: expected the buffer that the forward call returned")
    rows = lead[1:] if packed else lead
    dq, dkey = (torch.empty((*rows, Hk, dk), dtype=io, device=device) for _ in range(2))
    dval = torch.empty((*rows, Hv, dv), dtype=io, device=device)
    dg, dbeta = (torch.empty((*rows, Hv), dtype=gdt, device=device) for _ in range(2))
    ds0 = torch.empty((B, Hv, dk, dv), dtype=torch.float32, device=device) if want_ds0 else None
    head = (_DELTA_BWD_SIZE, B, Hk, Hv, dk, dv, code, gate, scale, lead[1], cu_seqlens.data_ptr() if packed else 0, *inputs, *pdo,
            _f32c(ds_last, "ds_last", (B, Hv, dk, dv)), saved.data_ptr(), saved.numel(), dq.data_ptr(), dkey.data_ptr(),
            dval.data_ptr(), dg.data_ptr(), dbeta.data_ptr(), 0 if ds0 is None else ds0.data_ptr())
    workspace = _scratch(workspace, 0 if workspace is not None else
                         _call("lrnnx_gated_delta_bwd_workspace_bytes", _pack_delta_bwd(*head, 0, 0, 0)), device)
    _check(_call("lrnnx_gated_delta_bwd", _pack_delta_bwd(*head, workspace.data_ptr(), workspace.numel(), _stream())))
    res = dict(dq=dq, dk=dkey, dv=dval, dg=dg, dbeta=dbeta)
    if want_ds0:
        res["ds0"] = ds0
    return res


@_native_first
def lrnnx_gated_delta_step(q, k, v, g, beta, state, scale=None, out=None):
    """One token: updates state [B,Hv,dk,dv] float32 in place and returns o [B,Hv,dv]; q, k [B,Hk,dk], v [B,Hv,dv], g, beta
    [B,Hv]; see lrnnx_delta_step_args."""
    io = v.dtype
    if q.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k, v: expected [B,H,d]")
    (B, Hk, dk), (_, Hv, dv) = q.shape, v.shape
    gate, pg, pbeta = _gates(g, beta, (B, Hv), io)
    o = torch.empty((B, Hv, dv), dtype=io, device=v.device) if out is None else out
    _check(_call("lrnnx_gated_delta_step", _pack_delta_step(
        _DELTA_STEP_SIZE, B, Hk, Hv, dk, dv, _io_dtype(v), gate, dk ** -0.5 if scale is None else float(scale),
        *_rows(q, "q", (B, Hk, dk), io), *_rows(k, "k", (B, Hk, dk), io), *_rows(v, "v", (B, Hv, dv), io), *pg, *pbeta,
        _f32c(state, "state", (B, Hv, dk, dv)), *_out_rows(o, "out", (B, Hv, dv), io), _stream())))
    return o


# ---------------------------------------------------------------- norms around a block
GATE_ACT = {"silu": 0, "sigmoid": 1}


def _matrix(t, name, shape, dtypes):
    """(ptr, row stride) of an optional tensor [..., D] as M rows."""
    if t is None:
        return 0, 0
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {' or '.join(str(d) for d in dtypes)}")
    if t.is_contiguous():
        return t.data_ptr(), shape[-1]
    if t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: expected a contiguous last axis")
    row, need = None, None
    for stride, count in zip(reversed(t.stride()[:-1]), reversed(shape[:-1])):       # one stride for all rows
        if count > 1:
            if row is None:
                row, need = stride, stride * count
            elif stride != need:
                raise ValueError(f"{name}: rows are not evenly spaced")
            else:
                need = stride * count
    return t.data_ptr(), shape[-1] if row is None else row


def _norm_head(x, post_weight, groups, gate, gate_act, residual, res_scale, pre_weight, eps, size, res_dtype):
    if x.dim() < 1:
        raise ValueError("x: expected [..., D]")
    io, shape, D = x.dtype, x.shape, x.shape[-1]
    code, groups = _io_dtype(x), int(groups)
    if res_dtype not in (torch.float32, io):
        raise TypeError(f"residual: dtype {res_dtype}, expected torch.float32 or {io}")
    if groups < 1 or D % groups:
        raise ValueError("D must be a multiple of groups")
    shared = post_weight is not None and groups > 1 and post_weight.shape == (D // groups,)
    return (size, x.numel() // max(D, 1), D, groups, int(shared), _code(gate_act, GATE_ACT), code, _io_dtype_of(res_dtype), float(eps), 0,
            *_matrix(x, "x", shape, (io,)), _f32c(post_weight, "post_weight", (D // groups,) if shared else (D,)),
            *_matrix(gate, "gate", shape, (io,)), *_matrix(residual, "residual", shape, (res_dtype,)),
            _f32c(res_scale, "res_scale", (D,)), _f32c(pre_weight, "pre_weight", (D,)))


def _io_dtype_of(dtype):
    return BF16 if dtype == torch.bfloat16 else F32


@_native_first
def lrnnx_block_norm_fwd(x, post_weight=None, groups=1, gate=None, gate_act="silu", residual=None, res_scale=None, pre_weight=None,
                         eps=1e-6, out=None):
    """(h, y): the norm, gate and residual sum after a block and the norm before the next; see lrnnx_norm_fwd_args.

    x, gate [..., D]; post_weight [D] or [D // groups] (one for all groups), res_scale, pre_weight [D] float32; residual
    [..., D] float32 or the I/O type, which is h's type too (x's without a residual).  y is None without pre_weight.  `out`
    takes h: contiguous, in the residual's type if there is one (it may be the residual)."""
    res_dtype = residual.dtype if residual is not None else out.dtype if out is not None else x.dtype
    head = _norm_head(x, post_weight, groups, gate, gate_act, residual, res_scale, pre_weight, eps, _NORM_FWD_SIZE, res_dtype)
    h = torch.empty(x.shape, dtype=res_dtype, device=x.device) if out is None else out
    if h.dtype != res_dtype:
        raise TypeError(f"out: dtype {h.dtype}, expected {res_dtype}")
    if h.shape != x.shape or not h.is_contiguous():
        raise ValueError(f"out: expected a contiguous tensor of shape {tuple(x.shape)}")
    y = None if pre_weight is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _check(_call("lrnnx_block_norm_fwd", _pack_norm_fwd(*head, h.data_ptr(), 0 if y is None else y.data_ptr(), _stream())))
    return h, y


@_native_first
def lrnnx_block_norm_bwd(x, dh=None, dy=None, post_weight=None, groups=1, gate=None, gate_act="silu", residual=None, res_scale=None,
                         pre_weight=None, eps=1e-6, workspace=None):
    """Gradients of sum(dh * h) + sum(dy * y) as a dict: dx, and dgate, dresidual, dpost_weight, dres_scale, dpre_weight for
    the inputs given; see lrnnx_norm_bwd_args.  Inputs as in the forward call; dh in h's type, dy in x's."""
    if dh is None and dy is None:
        raise ValueError("dh, dy: one of them is needed")
    res_dtype = residual.dtype if residual is not None else dh.dtype if dh is not None else x.dtype
    head = _norm_head(x, post_weight, groups, gate, gate_act, residual, res_scale, pre_weight, eps, _NORM_BWD_SIZE, res_dtype)
    D = x.shape[-1]
    grads = dict(dx=torch.empty(x.shape, dtype=x.dtype, device=x.device))
    if gate is not None:
        grads["dgate"] = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if residual is not None:
        grads["dresidual"] = torch.empty(x.shape, dtype=res_dtype, device=x.device)
    for name, w in (("dpost_weight", post_weight), ("dres_scale", res_scale), ("dpre_weight", pre_weight)):
        if w is not None:
            grads[name] = torch.empty_like(w)
    ptrs = [grads[n].data_ptr() if n in grads else 0 for n in ("dx", "dgate", "dresidual", "dpost_weight", "dres_scale", "dpre_weight")]
    workspace = _scratch(workspace, 0 if workspace is not None else lib().lrnnx_block_norm_bwd_workspace_bytes(head[1], D), x.device)
    _check(_call("lrnnx_block_norm_bwd", _pack_norm_bwd(
        *head, *_matrix(dh, "dh", x.shape, (res_dtype,)), *_matrix(dy, "dy", x.shape, (x.dtype,)), *ptrs,
        workspace.data_ptr(), workspace.numel(), _stream())))
    return grads


def _on_current(t, name):
    """Work is enqueued on the current device's stream: tensors of another GPU are refused."""
    if t.is_cuda and t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name}: on {t.device}, but the current device is cuda:{torch.cuda.current_device()}")


# ---------------------------------------------------------------- short causal convolution
CONV_ACT = {"silu": 0, "none": 1}
CONV_LAYOUT = {"bld": 0, "bdl": 1}
_CONV_FWD_SIZE, _CONV_BWD_SIZE, _CONV_STEP_SIZE = (ctypes.sizeof(c) for c in (ConvFwdArgs, ConvBwdArgs, ConvStepArgs))


def _conv_rows(t, name, shape, io, out=False):
    """(ptr, stride of a batch entry, of a row) of [B,L,D] or [B,D,L] with a contiguous last axis."""
    ptr, sb, ss = (_out_rows if out else _rows)(t, name, shape, io)
    return ptr, sb, ss


def _not_in_place(t, name, *inputs):
    """Steps of an input are read again where a neighbour's result may be written by then.  (The library refuses whatever else shares an element.)"""
    if t is not None and any(t.data_ptr() == x.data_ptr() for x in inputs):
        raise ValueError(f"{name}: must not be an input")


def _state(t, name, shape, io):
    """Pointer of optional carried inputs, contiguous in the I/O type."""
    if t is None:
        return 0
    if t.dtype != io or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous {io} tensor")
    if t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _conv_head(size, x, weight, bias, act, x0, cu_seqlens, layout):
    """What the calls over a sequence have in common; the packed form gets a batch axis of one.  x, shape, sequences, W - 1, head."""
    if x.dim() != (3 if cu_seqlens is None else 2):
        raise ValueError("x: expected three axes, or two with cu_seqlens")
    _on_current(x, "x")
    S = _check_cu(cu_seqlens) if cu_seqlens is not None else None
    if S is not None:
        x = x.unsqueeze(0)
    time_last, io = _code(layout, CONV_LAYOUT), x.dtype
    shape = x.shape
    L, D = (shape[2], shape[1]) if time_last else (shape[1], shape[2])
    B = S if S is not None else shape[0]
    if weight.dim() != 2:
        raise ValueError("weight: expected [D,W]")
    W = weight.shape[1]
    return x, shape, B, (B, max(W - 1, 0), D), (
        size, B, D, W, time_last, _code(act, CONV_ACT), _io_dtype(x), L, 0 if S is None else cu_seqlens.data_ptr(),
        *_conv_rows(x, "x", shape, io), _f32c(weight, "weight", (D, W)), _f32c(bias, "bias", (D,)), _state(x0, "x0", (B, max(W - 1, 0), D), io))


@_native_first
def lrnnx_short_conv_fwd(x, weight, bias=None, act="silu", x0=None, cu_seqlens=None, layout="bld", return_last_state=False, out=None):
    """y, and optionally the last W - 1 inputs [B,W-1,D], of the short causal convolution; see lrnnx_conv_fwd_args.

    x [B,L,D] (layout "bld", channels contiguous) or [B,D,L] ("bdl", time axis contiguous) float32 or bfloat16, views of wider tensors
    among them; weight [D,W] (W = 2 .. 4) and bias [D] float32; act "silu" or "none"; x0 [B,W-1,D] in x's type, the inputs before
    the first.  With `cu_seqlens` (int64 [S+1] on the device) the batch is packed: x and y without the batch axis, x0 and the last inputs
    [S,W-1,D]; steps of y outside every sequence are not written (a new y holds anything there).  An `out` that shares an element with an input is
    refused; other channels of the same wider tensor do not."""
    packed = cu_seqlens is not None
    io, device = x.dtype, x.device
    x, shape, B, state, head = _conv_head(_CONV_FWD_SIZE, x, weight, bias, act, x0, cu_seqlens, layout)
    _not_in_place(out, "out", x)
    y = torch.empty(shape, dtype=io, device=device) if out is None else out.unsqueeze(0) if packed else out
    last = torch.empty(state, dtype=io, device=device) if return_last_state else None
    _check(_call("lrnnx_short_conv_fwd", _pack_conv_fwd(*head, *_conv_rows(y, "out", shape, io, out=True), 0 if last is None else last.data_ptr(), _stream())))
    y = y[0] if packed else y
    return (y, last) if return_last_state else y


@_native_first
def lrnnx_short_conv_bwd(x, weight, dy, bias=None, act="silu", x0=None, dx_last=None, want_dx0=False, cu_seqlens=None, layout="bld",
                         out=None, workspace=None):
    """Gradients of sum(dy * y) (and sum(dx_last * x_last)) as a dict: dx in x's type (in `out`, if given), dweight and with a bias dbias
    float32, dx0 in x's type if wanted; see lrnnx_conv_bwd_args.  Inputs as in the forward call.  dx of steps outside every sequence of a
    packed batch is zero."""
    packed = cu_seqlens is not None
    io, device = x.dtype, x.device
    x, shape, B, state, head = _conv_head(_CONV_BWD_SIZE, x, weight, bias, act, x0, cu_seqlens, layout)
    _not_in_place(out, "out", x, dy)
    pdy = _conv_rows(dy.unsqueeze(0) if packed else dy, "dy", shape, io)
    dx = torch.empty(shape, dtype=io, device=device) if out is None else out.unsqueeze(0) if packed else out
    pdx = _conv_rows(dx, "out", shape, io, out=True)
    res = dict(dx=dx[0] if packed else dx, dweight=torch.empty_like(weight))
    if bias is not None:
        res["dbias"] = torch.empty_like(bias)
    if want_dx0:
        res["dx0"] = torch.empty(state, dtype=io, device=device)
    args = (*head, *pdy, _state(dx_last, "dx_last", state, io), *pdx, *(res[n].data_ptr() if n in res else 0 for n in ("dweight", "dbias", "dx0")))
    workspace = _scratch(workspace, 0 if workspace is not None else _call("lrnnx_short_conv_bwd_workspace_bytes", _pack_conv_bwd(*args, 0, 0, 0)), device)
    _check(_call("lrnnx_short_conv_bwd", _pack_conv_bwd(*args, workspace.data_ptr(), workspace.numel(), _stream())))
    return res


@_native_first
def lrnnx_short_conv_step(x, weight, state, bias=None, act="silu", out=None):
    """One token: moves the last inputs, state [B,W-1,D] in x's type, on by x in place and returns y [B,D]; see lrnnx_conv_step_args."""
    io = x.dtype
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x, weight: expected [B,D] and [D,W]")
    _on_current(x, "x")
    (B, D), W = x.shape, weight.shape[1]
    y = torch.empty((B, D), dtype=io, device=x.device) if out is None else out
    if y.shape != x.shape:
        raise ValueError(f"out: expected shape {(B, D)}, got {tuple(y.shape)}")
    if state is None:
        raise TypeError("state: expected a tensor")
    _check(_call("lrnnx_short_conv_step", _pack_conv_step(
        _CONV_STEP_SIZE, B, D, W, _code(act, CONV_ACT), _io_dtype(x), 0, *_bd(x, "x", io), _f32c(weight, "weight", (D, W)),
        _f32c(bias, "bias", (D,)), _state(state, "state", (B, max(W - 1, 0), D), io), *_bd(y, "out", io), _stream())))
    return y


# ---------------------------------------------------------------- loss over a vocabulary
_VOCAB_FWD_SIZE, _VOCAB_BWD_SIZE = ctypes.sizeof(VocabFwdArgs), ctypes.sizeof(VocabBwdArgs)


def _vocab_head(size, h, weight, target):
    if h.dim() < 1 or weight.dim() != 2 or weight.shape[1] != h.shape[-1]:
        raise ValueError("h, weight: expected [..., K] and [V,K]")
    _on_current(h, "h")
    if target.dtype != torch.int64 or not target.is_contiguous():
        raise TypeError("target: expected a contiguous int64 tensor")
    if target.shape != h.shape[:-1]:
        raise ValueError(f"target: expected shape {tuple(h.shape[:-1])}, got {tuple(target.shape)}")
    return (size, target.numel(), weight.shape[0], weight.shape[1], _io_dtype(h), *_matrix(h, "h", h.shape, (h.dtype,)),
            *_matrix(weight, "weight", weight.shape, (h.dtype,)), target.data_ptr())


def _vocab_scratch(name, pack, args, workspace, device):
    if workspace is None:
        return torch.empty(max(_call(name, pack(*args, 0, 0, 0)), 16), dtype=torch.uint8, device=device)
    return _scratch(workspace, 0, device)


@_native_first
def lrnnx_vocab_loss_fwd(h, weight, target, workspace=None):
    """(loss, lse): softmax cross entropy of h [..., K] over the words of weight [V,K] (logits h weight^T, which are not kept), and the
    logarithm of the sum that lrnnx_vocab_loss_bwd takes; see lrnnx_vocab_fwd_args.

    h, weight float32 or bfloat16 with evenly spaced rows; target [...] int64: rows whose target is negative have no loss (0), rows whose
    target is V or more NaN.  loss and lse [...] float32."""
    args = _vocab_head(_VOCAB_FWD_SIZE, h, weight, target)
    loss, lse = (torch.empty(target.shape, dtype=torch.float32, device=h.device) for _ in range(2))
    args = (*args, loss.data_ptr(), lse.data_ptr())
    workspace = _vocab_scratch("lrnnx_vocab_loss_fwd_workspace_bytes", _pack_vocab_fwd, args, workspace, h.device)
    _check(_call("lrnnx_vocab_loss_fwd", _pack_vocab_fwd(*args, workspace.data_ptr(), workspace.numel(), _stream())))
    return loss, lse


@_native_first
def lrnnx_vocab_loss_bwd(h, weight, target, lse, dloss, want_dh=True, want_dweight=True, workspace=None):
    """Gradients of sum(dloss * loss) as a dict: dh [..., K] and dweight [V,K] in the I/O type (each if wanted); see
    lrnnx_vocab_bwd_args.  h, weight and target as in the forward call, lse as it returned it; dloss [...] float32, contiguous or one
    number expanded.  dh of rows without a target is zero."""
    args = _vocab_head(_VOCAB_BWD_SIZE, h, weight, target)
    if dloss.dtype != torch.float32:
        raise TypeError("dloss: expected a float32 tensor")
    if dloss.shape != target.shape:
        raise ValueError(f"dloss: expected shape {tuple(target.shape)}, got {tuple(dloss.shape)}")
    if not any(dloss.stride()) and dloss.numel() > 0:
        step = 0
    elif dloss.is_contiguous():
        step = 1
    else:
        raise ValueError("dloss: expected a contiguous tensor, or one number expanded")
    if not want_dh and not want_dweight:
        raise ValueError("want_dh, want_dweight: one of them is needed")
    res = {}
    if want_dh:
        res["dh"] = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    if want_dweight:
        res["dweight"] = torch.empty(weight.shape, dtype=h.dtype, device=h.device)
    args = (*args, _f32c(lse, "lse", target.shape), dloss.data_ptr(), step, *(res[n].data_ptr() if n in res else 0 for n in ("dh", "dweight")))
    workspace = _vocab_scratch("lrnnx_vocab_loss_bwd_workspace_bytes", _pack_vocab_bwd, args, workspace, h.device)
    _check(_call("lrnnx_vocab_loss_bwd", _pack_vocab_bwd(*args, workspace.data_ptr(), workspace.numel(), _stream())))
    return res


# ---------------------------------------------------------------- norm and clipping of gradients
_GRAD_NORM_SIZE, _GRAD_CLIP_SIZE = ctypes.sizeof(GradNormArgs), ctypes.sizeof(GradClipArgs)


def _grad_list(grads, name, device=None):
    """The tensors as a list, with host arrays of their pointers, sizes and types."""
    grads = list(grads)
    if not grads:
        raise ValueError(f"{name}: expected one tensor at least")
    for t in grads:
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name}: expected tensors")
        if device is None:
            device = t.device
        if not t.is_cuda or t.device != device:
            raise TypeError(f"{name}: a tensor is on {t.device}; the library needs tensors of one GPU")
        if not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous tensors")
    _on_current(grads[0], name)
    n = len(grads)
    return grads, ((_vp * n)(*(t.data_ptr() for t in grads)), (_i64 * n)(*(t.numel() for t in grads)), (_i32 * n)(*(_io_dtype(t) for t in grads)))


def _apart(out, name, grads=()):
    """Tensors that are written must not overlap each other, nor what is read for another one (its own tensor is read before)."""
    def span(t, written):
        return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), written
    spans = [span(t, True) for t in out if t.numel()]
    spans += [span(g, False) for g, t in zip(grads, out) if g.numel() and span(g, True) != span(t, True)]
    any_end = written_end = 0
    for start, end, written in sorted(spans):
        if start < (any_end if written else written_end):
            raise ValueError(f"{name}: tensors overlap")
        any_end = max(any_end, end)
        if written:
            written_end = max(written_end, end)


@_native_first
def lrnnx_grad_norm(grads, workspace=None):
    """The 2-norm of all elements of a list of tensors together, a float32 tensor without axes; see lrnnx_grad_norm_args.
    Tensors contiguous, float32 or bfloat16, mixed as they are."""
    grads, arrays = _grad_list(grads, "grads")
    device = grads[0].device
    norm = torch.empty((), dtype=torch.float32, device=device)
    args = (_GRAD_NORM_SIZE, len(grads), *(ctypes.addressof(a) for a in arrays), norm.data_ptr())
    workspace = _scratch(workspace, 0 if workspace is not None else _call("lrnnx_grad_norm_workspace_bytes", _pack_grad_norm(*args, 0, 0, 0)), device)
    _check(_call("lrnnx_grad_norm", _pack_grad_norm(*args, workspace.data_ptr(), workspace.numel(), _stream())))
    return norm


@_native_first
def lrnnx_grad_clip(grads, norm, max_norm, eps=1e-6, out=None):
    """Scales all tensors by min(1, max_norm / (norm + eps)), in place or into the tensors `out` (float32, or each in its type), and returns
    them; see lrnnx_grad_clip_args.  norm: a float32 tensor of one element, what lrnnx_grad_norm returned or any other (a norm over
    several processes).  No tensor is waited for."""
    grads, arrays = _grad_list(grads, "grads")
    if norm.dtype != torch.float32 or norm.numel() != 1 or norm.device != grads[0].device:
        raise TypeError("norm: expected a float32 tensor of one element on the device of the gradients")
    outs, to = grads, (0, 0)
    if out is not None:
        outs, more = _grad_list(out, "out", grads[0].device)
        if len(outs) != len(grads):
            raise ValueError("out: expected as many tensors as grads")
        for g, o in zip(grads, outs):
            if o.shape != g.shape:
                raise ValueError(f"out: expected shape {tuple(g.shape)}, got {tuple(o.shape)}")
            if o.dtype not in (torch.float32, g.dtype):
                raise TypeError(f"out: dtype {o.dtype}, expected torch.float32 or {g.dtype}")
        to = (ctypes.addressof(more[0]), ctypes.addressof(more[2]))
    _apart(outs, "grads" if out is None else "out", () if out is None else grads)
    _check(_call("lrnnx_grad_clip", _pack_grad_clip(
        _GRAD_CLIP_SIZE, len(grads), *(ctypes.addressof(a) for a in arrays), *to, norm.data_ptr(), float(max_norm), float(eps), _stream())))
    return outs

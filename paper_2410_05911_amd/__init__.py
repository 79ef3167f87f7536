"""MI355X (gfx950) AECCT inference: Python binding of libaecct.so.

Argument marshalling only: every step of a decode runs in the library's HIP kernels.
PyTorch provides device memory and streams.  Importing this package loads the built
library and raises if it is missing; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libaecct.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_OUT_OF_MEMORY, ERR_DEVICE, ERR_WORKSPACE_TOO_SMALL = range(6)
PATH_AUTO, PATH_LAYERED, PATH_FUSED = 0, 1, 2
ATTN_HPSA, ATTN_CASA = 0, 1
LAYERED_ATTN_AUTO, LAYERED_ATTN_UNFUSED, LAYERED_ATTN_LDS_F32, LAYERED_ATTN_LDS_I16, LAYERED_ATTN_LDS_SPLIT = -1, 0, 1, 2, 3
ACT_SCALE_TOKEN, ACT_SCALE_WORD = 0, 1
F32, BF16, F16 = range(3)
CODE_NONE, CODE_I8, CODE_E4M3 = range(3)
LIN_Q, LIN_K, LIN_V, LIN_O, LIN_FF1, LIN_FF2 = range(6)

_vp = C.c_void_p
_i8p = C.POINTER(C.c_int8)
_f32p = C.POINTER(C.c_float)
_u8p = C.POINTER(C.c_uint8)


class Weights(C.Structure):
    _fields_ = [("embed", _f32p), ("pos", _f32p), ("w_q", _i8p), ("w_k", _i8p), ("w_v", _i8p), ("w_o", _i8p),
                ("w_ff1", _i8p), ("w_ff2", _i8p), ("scale", _f32p), ("b_q", _f32p), ("b_k", _f32p), ("b_v", _f32p),
                ("b_o", _f32p), ("b_ff1", _f32p), ("b_ff2", _f32p), ("ln1_g", _f32p), ("ln1_b", _f32p),
                ("ln2_g", _f32p), ("ln2_b", _f32p), ("head_w1", _f32p), ("head_b1", C.c_float),
                ("head_wo", _f32p), ("head_bo", _f32p)]


class Options(C.Structure):
    _fields_ = [("first_ring_heads", C.c_int32), ("d_ff", C.c_int32), ("ln_eps", C.c_float), ("path", C.c_int32),
                ("attention", C.c_int32), ("layered_attention", C.c_int32), ("act_scale_mode", C.c_int32)]


class ModelInfo(C.Structure):
    _fields_ = [("n", C.c_int32), ("m", C.c_int32), ("L", C.c_int32), ("d", C.c_int32), ("n_layers", C.c_int32),
                ("heads", C.c_int32), ("first_ring_heads", C.c_int32), ("d_ff", C.c_int32), ("path", C.c_int32),
                ("nnz_first_ring", C.c_int64), ("nnz_second_ring", C.c_int64), ("device_bytes", C.c_size_t),
                ("attention", C.c_int32), ("layered_attention", C.c_int32), ("act_scale_mode", C.c_int32),
                ("device", C.c_int32), ("compute_units", C.c_int32), ("lds_bytes", C.c_int64)]


class SpeParams(C.Structure):
    _fields_ = [("d_pe", C.c_int32), ("heads", C.c_int32), ("w_in", _f32p), ("b_in", _f32p),
                ("w_q", _f32p), ("w_k", _f32p), ("w_v", _f32p), ("w_o", _f32p),
                ("b_q", _f32p), ("b_k", _f32p), ("b_v", _f32p), ("b_o", _f32p),
                ("w_red", _f32p), ("b_red", C.c_float)]


_TRAIN_FIELDS = ["embed", "pos", "w_q", "w_k", "w_v", "w_o", "w_ff1", "w_ff2", "delta", "b_q", "b_k", "b_v", "b_o",
                 "b_ff1", "b_ff2", "ln1_g", "ln1_b", "ln2_g", "ln2_b", "head_w1", "head_b1", "head_wo", "head_bo"]


class TrainParams(C.Structure):
    _fields_ = [(f, _vp) for f in _TRAIN_FIELDS]


class TrainGrads(C.Structure):
    _fields_ = [(f, _vp) for f in _TRAIN_FIELDS if f != "pos"]


class RmsNormArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int64), ("type", C.c_int32), ("gain_type", C.c_int32), ("eps", C.c_float),
                ("code_type", C.c_int32), ("group", C.c_int32), ("x", _vp), ("ldx", C.c_int64), ("res", _vp),
                ("ldres", C.c_int64), ("gain", _vp), ("h", _vp), ("ldh", C.c_int64), ("y", _vp), ("ldy", C.c_int64),
                ("codes", _vp), ("ldcodes", C.c_int64), ("alpha", _vp)]


class RmsNormGradArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("d", C.c_int64), ("type", C.c_int32), ("gain_type", C.c_int32), ("eps", C.c_float),
                ("h", _vp), ("ldh", C.c_int64), ("dy", _vp), ("lddy", C.c_int64), ("dres", _vp), ("lddres", C.c_int64),
                ("gain", _vp), ("dh", _vp), ("lddh", C.c_int64), ("dgain", _vp)]


class Tensor(C.Structure):
    _fields_ = [("data", _vp), ("count", C.c_int64), ("type", C.c_int32)]


class AdamOptions(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("max_norm", C.c_double), ("lr_device", _vp)]


class AecctError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {lib().aecct_status_string(status).decode()} (status {status})")


_lib = None


def lib():
    """The loaded libaecct.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with paper_2410_05911_amd/build.py "
                              "(or __graft_entry__.build()); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        L.aecct_status_string.restype = C.c_char_p
        L.aecct_status_string.argtypes = [C.c_int]
        L.aecct_create.restype = C.c_int
        L.aecct_create.argtypes = [_u8p, C.c_int32, C.c_int32, C.POINTER(Weights), C.c_int32, C.c_int32, C.c_int32,
                                   C.POINTER(Options), C.POINTER(_vp)]
        L.aecct_destroy.restype = None
        L.aecct_destroy.argtypes = [_vp]
        L.aecct_get_info.restype = C.c_int
        L.aecct_get_info.argtypes = [_vp, C.POINTER(ModelInfo)]
        L.aecct_workspace_size.restype = C.c_int
        L.aecct_workspace_size.argtypes = [_vp, C.c_int64, C.POINTER(C.c_size_t)]
        L.aecct_decode.restype = C.c_int
        L.aecct_decode.argtypes = [_vp, _vp, C.c_int64, _vp, _vp, _vp, C.c_size_t, _vp]
        L.aecct_decode_static.restype = C.c_int
        L.aecct_decode_static.argtypes = [_vp, _vp, C.c_int64, _vp, _vp, _vp]
        L.aecct_stage_embed.restype = C.c_int
        L.aecct_stage_embed.argtypes = [_vp, _vp, C.c_int64, _vp, _vp, _vp, _vp]
        L.aecct_stage_qkv.restype = C.c_int
        L.aecct_stage_qkv.argtypes = [_vp, C.c_int32, _vp, _vp, C.c_int64, _vp, _vp]
        L.aecct_stage_attention.restype = C.c_int
        L.aecct_stage_attention.argtypes = [_vp, _vp, C.c_int64, _vp, _vp, _vp, _vp]
        L.aecct_stage_oproj_ln.restype = C.c_int
        L.aecct_stage_oproj_ln.argtypes = [_vp, C.c_int32, _vp, _vp, _vp, C.c_int64, _vp, _vp, _vp, _vp]
        L.aecct_stage_ffn1.restype = C.c_int
        L.aecct_stage_ffn1.argtypes = [_vp, C.c_int32, _vp, _vp, C.c_int64, _vp, _vp, _vp]
        L.aecct_stage_ffn2_ln.restype = C.c_int
        L.aecct_stage_ffn2_ln.argtypes = [_vp, C.c_int32, _vp, _vp, _vp, C.c_int64, _vp, _vp, _vp, _vp]
        L.aecct_stage_head.restype = C.c_int
        L.aecct_stage_head.argtypes = [_vp, _vp, _vp, C.c_int64, _vp, _vp, _vp]
        L.aecct_ternary_gemm.restype = C.c_int
        L.aecct_ternary_gemm.argtypes = [_vp, C.c_int32, C.c_int32, _vp, C.c_int64, _vp, _vp]
        L.aecct_aap_ternarize.restype = C.c_int
        L.aecct_aap_ternarize.argtypes = [_f32p, C.c_int64, C.c_float, C.c_float, C.c_float, _i8p, _f32p]
        _f64p = C.POINTER(C.c_double)
        L.aecct_tanner_spectrum.restype = C.c_int
        L.aecct_tanner_spectrum.argtypes = [_u8p, C.c_int32, C.c_int32, _f64p, _f64p]
        L.aecct_spe_table_from_spectrum.restype = C.c_int
        L.aecct_spe_table_from_spectrum.argtypes = [_f64p, _f64p, C.c_int32, C.POINTER(SpeParams), C.c_int32,
                                                    _f32p]
        L.aecct_spe_table.restype = C.c_int
        L.aecct_spe_table.argtypes = [_u8p, C.c_int32, C.c_int32, C.POINTER(SpeParams), C.c_int32, _f32p]
        L.aecct_train_create.restype = C.c_int
        L.aecct_train_create.argtypes = [_u8p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                         C.POINTER(Options), C.c_float, C.POINTER(_vp)]
        L.aecct_train_destroy.restype = None
        L.aecct_train_destroy.argtypes = [_vp]
        L.aecct_train_workspace_size.restype = C.c_int
        L.aecct_train_workspace_size.argtypes = [_vp, C.c_int64, C.POINTER(C.c_size_t)]
        L.aecct_train_grad.restype = C.c_int
        L.aecct_train_grad.argtypes = [_vp, C.POINTER(TrainParams), _vp, _vp, C.c_int64, C.POINTER(TrainGrads), _vp,
                                       _vp, C.c_size_t, _vp]
        L.aecct_rms_norm.restype = C.c_int
        L.aecct_rms_norm.argtypes = [C.POINTER(RmsNormArgs), _vp]
        L.aecct_rms_norm_grad_workspace_size.restype = C.c_int
        L.aecct_rms_norm_grad_workspace_size.argtypes = [C.c_int64, C.c_int64, C.POINTER(C.c_size_t)]
        L.aecct_rms_norm_grad.restype = C.c_int
        L.aecct_rms_norm_grad.argtypes = [C.POINTER(RmsNormGradArgs), _vp, C.c_size_t, _vp]
        _tp = C.POINTER(Tensor)
        L.aecct_update_workspace_size.restype = C.c_int
        L.aecct_update_workspace_size.argtypes = [C.c_int32, C.POINTER(C.c_size_t)]
        L.aecct_grad_norm.restype = C.c_int
        L.aecct_grad_norm.argtypes = [_tp, C.c_int32, _vp, _vp, C.c_size_t, _vp]
        L.aecct_grad_clip.restype = C.c_int
        L.aecct_grad_clip.argtypes = [_tp, _tp, C.c_int32, C.c_double, _vp, _vp, C.c_size_t, _vp]
        L.aecct_adam_step.restype = C.c_int
        L.aecct_adam_step.argtypes = [_tp, _tp, _tp, _tp, _tp, C.c_int32, C.POINTER(AdamOptions), _vp, _vp, _vp, C.c_size_t,
                                      _vp]
        _gp = C.POINTER(TrainGrads)
        L.aecct_train_update.restype = C.c_int
        L.aecct_train_update.argtypes = [_vp, _gp, _gp, _gp, _gp, C.POINTER(AdamOptions), _vp, _vp, _vp, C.c_size_t, _vp]
        L.aecct_check_device_arith.restype = C.c_int
        L.aecct_check_device_arith.argtypes = [C.POINTER(C.c_uint64)]
        _lib = L
    return _lib


def aap_ternarize(w, percentile: float = 0.5, delta: float = 1.0, eps: float = 1e-8):
    """AAP import of one trained fp32 weight matrix (Section 4.1, Eq. 1) by the library:
    returns (ternary int8 array of w's shape, weight scale gamma*delta as np.float32)."""
    w = np.ascontiguousarray(w, dtype=np.float32)
    t = np.zeros(w.shape, np.int8)
    sc = C.c_float(0.0)
    _check(lib().aecct_aap_ternarize(w.ctypes.data_as(_f32p), w.size, float(np.float32(percentile)),
                                     float(np.float32(delta)), float(np.float32(eps)), t.ctypes.data_as(_i8p),
                                     C.byref(sc)), "aecct_aap_ternarize")
    return t, np.float32(sc.value)


def tanner_spectrum(H):
    """Laplacian spectrum of the Tanner graph of H by the library (host, float64): returns
    (eigenvalues ascending [L], eigenvectors [L, L] with ROW i the canonical vector i)."""
    H = np.ascontiguousarray(H, dtype=np.uint8)
    m, n = H.shape
    lam = np.zeros(n + m, np.float64)
    vec = np.zeros((n + m, n + m), np.float64)
    _check(lib().aecct_tanner_spectrum(H.ctypes.data_as(_u8p), m, n, lam.ctypes.data_as(C.POINTER(C.c_double)),
                                       vec.ctypes.data_as(C.POINTER(C.c_double))), "aecct_tanner_spectrum")
    return lam, vec


def _spe_struct(p: dict, L: int):
    keep = {k: _host(p.get(k), np.float32) for k in ("w_in", "b_in", "w_q", "w_k", "w_v", "w_o", "b_q", "b_k",
                                                     "b_v", "b_o", "w_red")}
    if keep["w_red"] is not None and keep["w_red"].size != L:
        raise ValueError(f"w_red must have {L} entries")
    s = SpeParams(d_pe=int(p["d_pe"]), heads=int(p["heads"]), b_red=float(np.float32(p.get("b_red", 0.0))))
    for k, a in keep.items():
        setattr(s, k, _p32(a))
    return s, keep


def _p32(a):
    return a.ctypes.data_as(_f32p) if a is not None else None


def spe_table_from_spectrum(lam, vec_rows, p: dict, d: int):
    """Positional table [L, d] fp32 from a spectrum (ROW i of vec_rows = eigenvector i) and
    the SPE parameters (Section 4.3); the attention runs on the current GPU."""
    lam = np.ascontiguousarray(lam, dtype=np.float64)
    vec = np.ascontiguousarray(vec_rows, dtype=np.float64)
    L = lam.size
    s, keep = _spe_struct(p, L)
    out = np.zeros((L, d), np.float32)
    _check(lib().aecct_spe_table_from_spectrum(lam.ctypes.data_as(C.POINTER(C.c_double)),
                                               vec.ctypes.data_as(C.POINTER(C.c_double)), L, C.byref(s), d,
                                               out.ctypes.data_as(_f32p)), "aecct_spe_table_from_spectrum")
    return out


def spe_table(H, p: dict, d: int):
    """The whole SPE construction (spectrum, then attention) for H: positional table [L, d]."""
    H = np.ascontiguousarray(H, dtype=np.uint8)
    m, n = H.shape
    s, keep = _spe_struct(p, n + m)
    out = np.zeros((n + m, d), np.float32)
    _check(lib().aecct_spe_table(H.ctypes.data_as(_u8p), m, n, C.byref(s), d, out.ctypes.data_as(_f32p)),
           "aecct_spe_table")
    return out


def check_device_arith():
    """Counts of fp32 operands where the device's fract/floor split, softmax reciprocal and
    127/alpha differ from their IEEE definitions (all 0 on a conforming GPU)."""
    counts = (C.c_uint64 * 3)()
    _check(lib().aecct_check_device_arith(counts), "aecct_check_device_arith")
    return tuple(int(c) for c in counts)


def _check(status: int, what: str):
    if status != OK:
        raise AecctError(status, what)


def _host(a, dtype):
    return None if a is None else np.ascontiguousarray(a, dtype=dtype)


def _ptr(t):
    """Device address of a torch tensor (or None)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _stream_ptr(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _on_stream(stream):
    """Context in which torch's allocations and the library's launches belong to `stream`."""
    import torch
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


def _on_current_gpu(index: int):
    """Refuses tensors of another GPU than the current one, where the library launches (index: get_device())."""
    import torch
    current = torch.cuda.current_device() if index >= 0 else -1
    if index != current or index < 0:
        raise ValueError("tensors must be on the GPU" if index < 0 else
                         f"tensors are on cuda:{index}, the current device is cuda:{current}")


def _current_stream(index: int) -> int:
    """Handle of the current stream of a GPU, without a Stream object around it where torch hands it out."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream


_DTYPES: dict = {}


def _dtype_code(t):
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"unsupported type {t.dtype}: float32, bfloat16 or float16")
    return code


def _rows_of(t, shape, dtype, index: int, what):
    """(address, row stride) of a tensor of rows [..., d] of that shape, type and GPU."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype != dtype or t.get_device() != index:
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)} on cuda:{index}")
    d = shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), d
    if len(shape) != 2:
        raise ValueError(f"{what}: rows of other than two dimensions must be contiguous")
    ld, one = t.stride()
    if one != 1 and d > 1:
        raise ValueError(f"{what}: a row's values must be contiguous")
    return t.data_ptr(), ld if shape[0] > 1 else d


def _gain_of(gain, d: int, index: int):
    if gain is None:
        return None, F32
    if gain.dim() != 1 or gain.numel() != d or not gain.is_contiguous() or gain.get_device() != index:
        raise ValueError(f"gain must be {d} contiguous values on cuda:{index}")
    return gain.data_ptr(), _dtype_code(gain)


def rms_norm(x, gain=None, res=None, eps: float = 1e-5, *, y=None, h=None, codes=None, alpha=None, with_y: bool = True,
             code_type=None, group: int = 0, stream=None):
    """Root-mean-square norm of rows with the residual's addition: h = x + res, y = h / sqrt(mean(h^2) + eps) * gain, and
    y's 8-bit codes (Eq. 2) with their alphas, one for a row or for `group` (32, 64 or 128) columns.

    x, res: CUDA tensors [..., d] of one type (float32, bfloat16, float16), contiguous or of two dimensions with contiguous
    rows; gain [d] float32 or that type.  Autograd does not record the call: rms_norm_grad is its gradient.  code_type:
    None, torch.int8 (value = code * alpha / 127) or torch.float8_e4m3fn (value = code * alpha / 448).  y, h, codes,
    alpha: outputs to write to, else new tensors (h or y may be x or res itself).
    Returns (y, h, codes, alpha), None where there is no such output: y without with_y, h without res."""
    import torch
    if stream is not None:
        with _on_stream(stream):
            return rms_norm(x, gain, res, eps, y=y, h=h, codes=codes, alpha=alpha, with_y=with_y, code_type=code_type,
                            group=group)
    shape = x.shape
    if not shape or shape[-1] < 1:
        raise ValueError("x must be [..., d] with d >= 1")
    d, dtype = shape[-1], x.dtype
    kind = CODE_NONE if code_type is None else CODE_I8 if code_type == torch.int8 else \
        CODE_E4M3 if code_type == torch.float8_e4m3fn else -1
    if kind < 0:
        raise ValueError("code_type must be None, torch.int8 or torch.float8_e4m3fn")
    if kind == CODE_NONE and (codes is not None or alpha is not None or group):
        raise ValueError("codes, alpha and group need a code_type")
    if group not in (0, 32, 64, 128):
        raise ValueError("group must be 0, 32, 64 or 128")
    index = x.get_device()
    _on_current_gpu(index)
    px, ldx = _rows_of(x, shape, dtype, index, "x")
    pres, ldres = _rows_of(res, shape, dtype, index, "res")
    pgain, gain_type = _gain_of(gain, d, index)
    like = x if x.is_contiguous() else x.new_empty(shape)   # what new outputs are made like
    fresh_y = y is None and with_y
    if fresh_y:
        y = torch.empty_like(like)
    py, ldy = (y.data_ptr(), d) if fresh_y else _rows_of(y, shape, dtype, index, "y")
    fresh_h = h is None and res is not None
    if fresh_h:
        h = like if like is not x else torch.empty_like(x)
    ph, ldh = (h.data_ptr(), d) if fresh_h else _rows_of(h, shape, dtype, index, "h")
    pcodes, ldcodes, palpha = None, 0, None
    if kind != CODE_NONE:
        if codes is None:
            codes = torch.empty_like(like, dtype=code_type)
        pcodes, ldcodes = _rows_of(codes, shape, code_type, index, "codes")
        scales = shape[:-1] + ((d + group - 1) // group,) if group else shape[:-1]
        if alpha is None:
            alpha = torch.empty(scales, dtype=torch.float32, device=x.device)
        elif alpha.shape != scales or alpha.dtype != torch.float32 or not alpha.is_contiguous() or alpha.get_device() != index:
            raise ValueError(f"alpha must be contiguous float32 {tuple(scales)} on cuda:{index}")
        palpha = alpha.data_ptr()
    a = RmsNormArgs(x.numel() // d, d, _dtype_code(x), gain_type, eps, kind, group, px, ldx, pres, ldres, pgain, ph, ldh, py,
                    ldy, pcodes, ldcodes, palpha)
    _check(lib().aecct_rms_norm(C.byref(a), _current_stream(index)), "aecct_rms_norm")
    return y, h, codes, alpha


@functools.lru_cache(maxsize=256)
def _norm_grad_workspace(rows: int, d: int) -> int:
    size = C.c_size_t()
    _check(lib().aecct_rms_norm_grad_workspace_size(rows, d, C.byref(size)), "aecct_rms_norm_grad_workspace_size")
    return size.value


def rms_norm_grad(h, dy, gain=None, dres=None, eps: float = 1e-5, *, dh=None, dgain=None, with_dgain: bool = True, stream=None):
    """Gradient of rms_norm: h as the norm read it (x, or the h it returned), dy the gradient of y (or of the codes'
    values), dres the gradient that reaches h along the residual.  Returns (dh, dgain): dh is the gradient of x and
    of res, dgain float32 [d] (None without with_dgain)."""
    import torch
    if stream is not None:
        with _on_stream(stream):
            return rms_norm_grad(h, dy, gain, dres, eps, dh=dh, dgain=dgain, with_dgain=with_dgain)
    shape = h.shape
    if not shape or shape[-1] < 1:
        raise ValueError("h must be [..., d] with d >= 1")
    d, dtype = shape[-1], h.dtype
    rows = h.numel() // d
    index = h.get_device()
    _on_current_gpu(index)
    ph, ldh = _rows_of(h, shape, dtype, index, "h")
    pdy, lddy = _rows_of(dy, shape, dtype, index, "dy")
    pres, lddres = _rows_of(dres, shape, dtype, index, "dres")
    pgain, gain_type = _gain_of(gain, d, index)
    if dh is None:
        dh = torch.empty_like(h) if h.is_contiguous() else h.new_empty(shape)
    pdh, lddh = _rows_of(dh, shape, dtype, index, "dh")
    pdgain = pws = None
    need = 0
    if dgain is not None or with_dgain:
        if dgain is None:
            dgain = torch.empty(d, dtype=torch.float32, device=h.device)
        elif dgain.shape != (d,) or dgain.dtype != torch.float32 or not dgain.is_contiguous() or dgain.get_device() != index:
            raise ValueError(f"dgain must be {d} contiguous float32 values on cuda:{index}")
        pdgain = dgain.data_ptr()
        need = _norm_grad_workspace(rows, d)
        ws = torch.empty(need, dtype=torch.uint8, device=h.device)
        pws = ws.data_ptr()
    a = RmsNormGradArgs(rows, d, _dtype_code(h), gain_type, eps, ph, ldh, pdy, lddy, pres, lddres, pgain, pdh, lddh, pdgain)
    _check(lib().aecct_rms_norm_grad(C.byref(a), pws, need, _current_stream(index)), "aecct_rms_norm_grad")
    return dh, dgain


class TensorList:
    """A list of contiguous CUDA tensors (float32, bfloat16, float16; one device) as the library takes it.  A program that
    uses the same tensors again and again keeps the list; the calls below take any sequence of tensors too.  The list
    stands for the memory that the tensors have when it is made, and keeps that memory: a tensor that is given other
    memory later (`t.data = ...`, `module.to(...)`, `set_`) needs a new list, and `resize_` must not move it.  (Adam
    looks after its own lists.)"""

    def __init__(self, tensors, *, _keep: bool = True):
        self.tensors = list(tensors)
        self._keep = _keep
        self._read()
        size = C.c_size_t()
        _check(lib().aecct_update_workspace_size(len(self), C.byref(size)), "aecct_update_workspace_size")
        self.workspace_bytes = size.value

    def _read(self):
        """Takes the tensors' addresses, and (not for the list of a single call) holds on to the memory there: the tensor
        objects alone do not, their storage can be exchanged."""
        n = len(self.tensors)
        array = (Tensor * n)()
        device = self.tensors[0].get_device() if n else None
        for i, t in enumerate(self.tensors):
            if not t.is_contiguous():
                raise ValueError(f"tensor {i} must be contiguous")
            if t.get_device() != device or device < 0:
                raise ValueError("the tensors must be on one GPU")
            array[i] = Tensor(t.data_ptr(), t.numel(), _dtype_code(t))
        self.array, self.device = array, device
        if self._keep:
            self._addresses = self._places()
            self._memory = [t.untyped_storage() for t in self.tensors]

    def _places(self):
        import torch
        return list(map(torch.Tensor.data_ptr, self.tensors))

    def _follow(self):
        """Takes the addresses anew if a tensor has moved since."""
        if self._places() != self._addresses:
            self._read()

    def __len__(self):
        return len(self.tensors)


def _list(tensors):   # for one call
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors, _keep=False)


def _kept_list(tensors):
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors)


def _one_gpu(*lists):
    """The GPU of the lists, which must be the current one."""
    import torch
    index = None
    for t in lists:
        if t is not None and t.device is not None:
            if index is not None and t.device != index:
                raise ValueError("the lists must be on one GPU")
            index = t.device
    if index is None:
        return torch.cuda.current_device()
    _on_current_gpu(index)
    return index


def grad_norm(grads, stream=None):
    """The norm over every value of a list of tensors (a TensorList or any sequence): one-element float32 tensor."""
    import torch
    if stream is not None:
        with _on_stream(stream):
            return grad_norm(grads)
    g = _list(grads)
    device = _one_gpu(g)
    norm = torch.empty(1, dtype=torch.float32, device=device)
    ws = torch.empty(g.workspace_bytes, dtype=torch.uint8, device=device)
    _check(lib().aecct_grad_norm(g.array, len(g), norm.data_ptr(), ws.data_ptr(), g.workspace_bytes, _current_stream(device)),
           "aecct_grad_norm")
    return norm


def grad_clip(grads, max_norm: float, out=None, stream=None):
    """Scales every gradient by min(1, max_norm / norm), in place or into the tensors of `out`; returns the norm before
    clipping.  Where any value is not finite, none is scaled.  A max_norm of 0 makes every value 0.  Autograd does not see
    the write (no version counter moves)."""
    import torch
    if stream is not None:
        with _on_stream(stream):
            return grad_clip(grads, max_norm, out)
    g = _list(grads)
    o = None if out is None else _list(out)
    if o is not None and len(o) != len(g):
        raise ValueError(f"out must hold {len(g)} tensors")
    device = _one_gpu(g, o)
    norm = torch.empty(1, dtype=torch.float32, device=device)
    ws = torch.empty(g.workspace_bytes, dtype=torch.uint8, device=device)
    _check(lib().aecct_grad_clip(g.array, None if o is None else o.array, len(g), max_norm, norm.data_ptr(), ws.data_ptr(),
                                 g.workspace_bytes, _current_stream(device)), "aecct_grad_clip")
    return norm


def _adam_options(lr, betas, eps, weight_decay, max_norm):
    lr_device = None
    if hasattr(lr, "data_ptr"):
        import torch
        if lr.dtype != torch.float32 or lr.numel() != 1 or lr.get_device() != torch.cuda.current_device():
            raise ValueError("lr must be a number or one float32 value on the current GPU")
        lr_device, lr = lr.data_ptr(), 0.0
    return AdamOptions(lr, betas[0], betas[1], eps, weight_decay, 0.0 if max_norm is None else max_norm, lr_device)


def _step_tensor(step, device: int):
    import torch
    if step is None:
        return torch.zeros(1, dtype=torch.int64, device=device)
    if step.dtype != torch.int64 or step.numel() != 1 or step.get_device() != device:
        raise ValueError(f"step must be one int64 value on cuda:{device}")
    return step


class Adam:
    """Adam over a list of float32 tensors (Section 6), updated in place: moments m and v (zeros, or the given float32
    tensors), the number of updates made in `step` (one int64 value on the GPU), decoupled weight decay, gradients
    clipped to max_norm over the whole list (None: not; 0: not, but measured), and optional 16-bit `copies` of the parameters.
    lr: a number, or one float32 value on the GPU that captured graphs read at each replay.  Parameters and copies that have
    been given other memory since (`p.data = ...`, `module.to(...)`) are updated where they are; the moments stay.  Autograd
    does not see the update (no version counter moves): finish a backward pass before the step that follows it."""

    def __init__(self, params, lr=1e-4, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0, max_norm=None,
                 m=None, v=None, step=None, copies=None):
        import torch
        self.params = _kept_list(params)
        self.m = _kept_list(m if m is not None else [torch.zeros_like(p) for p in self.params.tensors])
        self.v = _kept_list(v if v is not None else [torch.zeros_like(p) for p in self.params.tensors])
        self.copies = None if copies is None else _kept_list(copies)
        for what, t in (("m", self.m), ("v", self.v), ("copies", self.copies)):
            if t is not None and len(t) != len(self.params):
                raise ValueError(f"{what} must hold {len(self.params)} tensors")
        self.device = _one_gpu(self.params, self.m, self.v, self.copies)
        self.lr, self.betas, self.eps, self.weight_decay, self.max_norm = lr, betas, eps, weight_decay, max_norm
        self.step_count = _step_tensor(step, self.device)

    def step(self, grads, lr=None, stream=None):
        """One update from the gradients (a TensorList or any sequence, any of the types).  Returns the norm before
        clipping (None without max_norm); where any gradient then is not finite nothing is updated."""
        import torch
        if stream is not None:
            with _on_stream(stream):
                return self.step(grads, lr)
        g = _list(grads)
        if len(g) != len(self.params):
            raise ValueError(f"grads must hold {len(self.params)} tensors")
        self.params._follow()
        if self.copies is not None:
            self.copies._follow()
        device = _one_gpu(self.params, self.m, self.v, self.copies, g) if len(g) else self.device
        opt = _adam_options(self.lr if lr is None else lr, self.betas, self.eps, self.weight_decay, self.max_norm)
        norm = None if self.max_norm is None else torch.empty(1, dtype=torch.float32, device=device)
        ws = torch.empty(g.workspace_bytes, dtype=torch.uint8, device=device)
        _check(lib().aecct_adam_step(self.params.array, self.m.array, self.v.array, g.array,
                                     None if self.copies is None else self.copies.array, len(g), C.byref(opt),
                                     self.step_count.data_ptr(), None if norm is None else norm.data_ptr(), ws.data_ptr(),
                                     g.workspace_bytes, _current_stream(device)), "aecct_adam_step")
        return norm


class Decoder:
    """An AECCT model on the current GPU.

    `H` is the (n-k) x n parity-check matrix (0/1) and `w` carries the model parameters
    with the attribute names of `workloads.ModelWeights` (embed, pos, w[kind], b[kind], scale,
    ln1_g, ..., head_wo, head_bo, and optionally attention = "hpsa" | "casa" and
    act_scale = "token" | "word").  `path` and `layered_attention` choose the kernels
    (aecct_path, aecct_layered_attention; -1 = automatic).
    """

    def __init__(self, H, w, path: int = PATH_AUTO, layered_attention: int = LAYERED_ATTN_AUTO):
        H = _host(H, np.uint8)
        m, n = H.shape
        self._keep = [H]

        def f32(a):
            a = _host(a, np.float32)
            self._keep.append(a)
            return None if a is None else a.ctypes.data_as(_f32p)

        def i8(a):
            a = _host(a, np.int8)
            self._keep.append(a)
            return a.ctypes.data_as(_i8p)

        st = Weights()
        st.embed, st.pos = f32(w.embed), f32(w.pos)
        st.w_q, st.w_k, st.w_v, st.w_o = (i8(w.w[k]) for k in ("q", "k", "v", "o"))
        st.w_ff1, st.w_ff2 = i8(w.w["ff1"]), i8(w.w["ff2"])
        st.scale = f32(w.scale)
        st.b_q, st.b_k, st.b_v, st.b_o = (f32(w.b[k]) for k in ("q", "k", "v", "o"))
        st.b_ff1, st.b_ff2 = f32(w.b["ff1"]), f32(w.b["ff2"])
        st.ln1_g, st.ln1_b, st.ln2_g, st.ln2_b = f32(w.ln1_g), f32(w.ln1_b), f32(w.ln2_g), f32(w.ln2_b)
        st.head_w1, st.head_b1 = f32(w.head_w1), float(np.float32(w.head_b1))
        st.head_wo, st.head_bo = f32(w.head_wo), f32(w.head_bo)
        attention = {"hpsa": ATTN_HPSA, "casa": ATTN_CASA}[getattr(w, "attention", "hpsa")]
        act = {"token": ACT_SCALE_TOKEN, "word": ACT_SCALE_WORD}[getattr(w, "act_scale", "token")]
        opt = Options(int(w.first_ring_heads), int(w.d_ff), float(w.ln_eps), int(path), attention,
                      int(layered_attention), act)
        h = _vp()
        _check(lib().aecct_create(H.ctypes.data_as(_u8p), m, n, C.byref(st), int(w.d), int(w.n_layers),
                                  int(w.heads), C.byref(opt), C.byref(h)), "aecct_create")
        self._h = h
        self._keep = None
        info = ModelInfo()
        _check(lib().aecct_get_info(h, C.byref(info)), "aecct_get_info")
        self.info = info
        self.n, self.m, self.L, self.d = info.n, info.m, info.L, info.d
        self.n_layers, self.d_ff, self.path = info.n_layers, info.d_ff, info.path
        self._ws = None

    def close(self):
        if getattr(self, "_h", None):
            lib().aecct_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ------------------------------------------------------------------ decode
    def workspace_size(self, batch: int) -> int:
        sz = C.c_size_t()
        _check(lib().aecct_workspace_size(self._h, int(batch), C.byref(sz)), "aecct_workspace_size")
        return sz.value

    def workspace(self, batch: int, device=None):
        """A cached uint8 device tensor large enough for `batch` words."""
        import torch
        need = self.workspace_size(batch)
        if need == 0:
            return None
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=device or "cuda")
        return self._ws

    def decode(self, y, bits=None, logits=None, workspace=None, stream=None, with_logits: bool = True):
        """y: fp32 CUDA tensor [B, n].  Returns (bits uint8 [B, n], logits fp32 [B, n] or None)."""
        import torch
        B = y.shape[0]
        if bits is None:
            bits = torch.empty((B, self.n), dtype=torch.uint8, device=y.device)
        if logits is None and with_logits:
            logits = torch.empty((B, self.n), dtype=torch.float32, device=y.device)
        ws = workspace if workspace is not None else self.workspace(B, y.device)
        _check(lib().aecct_decode(self._h, _ptr(y), B, _ptr(bits), _ptr(logits), _ptr(ws),
                                  0 if ws is None else ws.numel(), _stream_ptr(stream)), "aecct_decode")
        return bits, logits

    def decode_static(self, y, bits=None, logits=None, stream=None, with_logits: bool = True):
        """aecct_decode_static: the same decode with the library's static device scratch (no
        workspace, no allocation by the library)."""
        import torch
        B = y.shape[0]
        if bits is None:
            bits = torch.empty((B, self.n), dtype=torch.uint8, device=y.device)
        if logits is None and with_logits:
            logits = torch.empty((B, self.n), dtype=torch.float32, device=y.device)
        _check(lib().aecct_decode_static(self._h, _ptr(y), B, _ptr(bits), _ptr(logits), _stream_ptr(stream)),
               "aecct_decode_static")
        return bits, logits

    # ------------------------------------------------------------------ stages
    def stage_embed(self, y, stream=None):
        import torch
        W = y.shape[0]
        R = W * self.L
        x = torch.empty((R, self.d), dtype=torch.float32, device=y.device)
        xq = torch.empty((R, self.d), dtype=torch.int8, device=y.device)
        ax = torch.empty((R,), dtype=torch.float32, device=y.device)
        _check(lib().aecct_stage_embed(self._h, _ptr(y), W, _ptr(x), _ptr(xq), _ptr(ax), _stream_ptr(stream)),
               "aecct_stage_embed")
        return x, xq, ax

    def stage_qkv(self, layer, xq, ax, stream=None):
        import torch
        W = xq.shape[0] // self.L
        qkv = torch.empty((xq.shape[0], 3 * self.d), dtype=torch.float32, device=xq.device)
        _check(lib().aecct_stage_qkv(self._h, layer, _ptr(xq), _ptr(ax), W, _ptr(qkv), _stream_ptr(stream)),
               "aecct_stage_qkv")
        return qkv

    def stage_attention(self, qkv, with_o: bool = True, stream=None):
        import torch
        R = qkv.shape[0]
        W = R // self.L
        o = torch.empty((R, self.d), dtype=torch.float32, device=qkv.device) if with_o else None
        oq = torch.empty((R, self.d), dtype=torch.int8, device=qkv.device)
        ao = torch.empty((R,), dtype=torch.float32, device=qkv.device)
        _check(lib().aecct_stage_attention(self._h, _ptr(qkv), W, _ptr(o), _ptr(oq), _ptr(ao), _stream_ptr(stream)),
               "aecct_stage_attention")
        return o, oq, ao

    def stage_oproj_ln(self, layer, oq, ao, x, stream=None):
        import torch
        R = oq.shape[0]
        x1 = torch.empty((R, self.d), dtype=torch.float32, device=oq.device)
        x1q = torch.empty((R, self.d), dtype=torch.int8, device=oq.device)
        a1 = torch.empty((R,), dtype=torch.float32, device=oq.device)
        _check(lib().aecct_stage_oproj_ln(self._h, layer, _ptr(oq), _ptr(ao), _ptr(x), R // self.L, _ptr(x1),
                                          _ptr(x1q), _ptr(a1), _stream_ptr(stream)), "aecct_stage_oproj_ln")
        return x1, x1q, a1

    def stage_ffn1(self, layer, x1q, a1, stream=None):
        import torch
        R = x1q.shape[0]
        gq = torch.empty((R, self.d_ff), dtype=torch.int8, device=x1q.device)
        ag = torch.empty((R,), dtype=torch.float32, device=x1q.device)
        _check(lib().aecct_stage_ffn1(self._h, layer, _ptr(x1q), _ptr(a1), R // self.L, _ptr(gq), _ptr(ag),
                                      _stream_ptr(stream)), "aecct_stage_ffn1")
        return gq, ag

    def stage_ffn2_ln(self, layer, gq, ag, x1, stream=None):
        import torch
        R = gq.shape[0]
        x = torch.empty((R, self.d), dtype=torch.float32, device=gq.device)
        xq = torch.empty((R, self.d), dtype=torch.int8, device=gq.device)
        ax = torch.empty((R,), dtype=torch.float32, device=gq.device)
        _check(lib().aecct_stage_ffn2_ln(self._h, layer, _ptr(gq), _ptr(ag), _ptr(x1), R // self.L, _ptr(x),
                                         _ptr(xq), _ptr(ax), _stream_ptr(stream)), "aecct_stage_ffn2_ln")
        return x, xq, ax

    def stage_head(self, x, y, stream=None):
        import torch
        W = y.shape[0]
        bits = torch.empty((W, self.n), dtype=torch.uint8, device=y.device)
        logits = torch.empty((W, self.n), dtype=torch.float32, device=y.device)
        _check(lib().aecct_stage_head(self._h, _ptr(x), _ptr(y), W, _ptr(bits), _ptr(logits), _stream_ptr(stream)),
               "aecct_stage_head")
        return bits, logits

    def ternary_gemm(self, layer, kind, a, stream=None):
        import torch
        rows = a.shape[0]
        n_out = self.d_ff if kind == LIN_FF1 else self.d
        acc = torch.empty((rows, n_out), dtype=torch.int32, device=a.device)
        _check(lib().aecct_ternary_gemm(self._h, layer, kind, _ptr(a), rows, _ptr(acc), _stream_ptr(stream)),
               "aecct_ternary_gemm")
        return acc


_TRAIN_KINDS = ("q", "k", "v", "o", "ff1", "ff2")


class Trainer:
    """The quantisation-aware training step (Section 6, second phase) on the current GPU for the
    code of H: forward with Eq. 1 / Eq. 2 straight-through quantisation, the loss of the
    multiplicative noise and every parameter's gradient, in the library's kernels.

    Parameters and gradients are dicts of contiguous fp32 CUDA tensors with the keys of
    `workloads.random_qat_params` (w and b are dicts by map kind; head_b1 a one-element tensor).
    """

    def __init__(self, H, d: int, n_layers: int, heads: int = 8, first_ring_heads: int = -1,
                 attention: str = "hpsa", ln_eps: float = 1e-5, aap_eps: float = 1e-8):
        H = _host(H, np.uint8)
        m, n = H.shape
        self.n, self.m, self.L, self.d, self.n_layers = n, m, n + m, d, n_layers
        opt = Options(int(first_ring_heads), -1, float(ln_eps), PATH_AUTO,
                      {"hpsa": ATTN_HPSA, "casa": ATTN_CASA}[attention], LAYERED_ATTN_AUTO, ACT_SCALE_TOKEN)
        h = _vp()
        _check(lib().aecct_train_create(H.ctypes.data_as(_u8p), m, n, int(d), int(n_layers), int(heads), C.byref(opt),
                                        float(np.float32(aap_eps)), C.byref(h)), "aecct_train_create")
        self._h = h
        self._ws = None

    def close(self):
        if getattr(self, "_h", None):
            lib().aecct_train_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_size(self, batch: int) -> int:
        sz = C.c_size_t()
        _check(lib().aecct_train_workspace_size(self._h, int(batch), C.byref(sz)), "aecct_train_workspace_size")
        return sz.value

    @staticmethod
    def _flat(d: dict):
        out = {}
        for k, v in d.items():
            if k in ("w", "b"):
                for kind in _TRAIN_KINDS:
                    out[f"{k}_{kind}"] = v[kind]
            else:
                out[k] = v
        return out

    def _counts(self) -> list:
        """Values of each tensor that the library updates, in the order of TrainGrads: they follow from the model, and the
        library reads and writes that many."""
        L, N, d, n = self.L, self.n_layers, self.d, self.n
        return [L * d] + [N * d * d] * 4 + [4 * N * d * d] * 2 + [6 * N] + [N * d] * 4 + [4 * N * d] + [N * d] * 5 + [d, 1, L * n, n]

    def grad(self, params: dict, y, xs=None, stream=None):
        """One step on the words y [B, n] (xs: transmitted +-1 words, None = all-zero codeword).
        Returns (loss one-element tensor, gradients dict shaped like params, without pos)."""
        import torch
        B = y.shape[0]
        flat = self._flat(params)
        tp = TrainParams(**{f: _ptr(flat.get(f)) for f in _TRAIN_FIELDS})
        grads = {k: (torch.empty_like(v) if k not in ("w", "b") else {kk: torch.empty_like(vv) for kk, vv in v.items()})
                 for k, v in params.items() if k != "pos" and v is not None}
        gflat = self._flat(grads)
        tg = TrainGrads(**{f: _ptr(gflat[f]) for f, _ in TrainGrads._fields_})
        need = self.workspace_size(B)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=y.device)
        loss = torch.empty(1, dtype=torch.float32, device=y.device)
        _check(lib().aecct_train_grad(self._h, C.byref(tp), _ptr(y), _ptr(xs), B, C.byref(tg), _ptr(loss),
                                      _ptr(self._ws), self._ws.numel(), _stream_ptr(stream)), "aecct_train_grad")
        return loss, grads

    def update_state(self, params: dict):
        """A fresh Adam state for `update`: dict with the moments m and v (shaped like params, zeros) and the step."""
        import torch
        zeros = lambda: {k: (torch.zeros_like(t) if k not in ("w", "b") else {kk: torch.zeros_like(tt) for kk, tt in t.items()})  # noqa: E731
                         for k, t in params.items() if k != "pos" and t is not None}
        return {"m": zeros(), "v": zeros(), "step": _step_tensor(None, params["embed"].get_device())}

    def update(self, params: dict, grads: dict, state: dict, lr, betas=(0.9, 0.999), eps: float = 1e-8,
               weight_decay: float = 0.0, max_norm=None, stream=None):
        """One Adam update of every parameter from `grad`'s gradients (aecct_train_update), in place.  Returns the norm
        of the gradients before clipping (None without max_norm); where any gradient then is not finite nothing is
        updated."""
        import torch
        if stream is not None:
            with _on_stream(stream):
                return self.update(params, grads, state, lr, betas, eps, weight_decay, max_norm)
        opt = _adam_options(lr, betas, eps, weight_decay, max_norm)
        fields = [f for f, _ in TrainGrads._fields_]
        lists = []
        flat = [self._flat(d) for d in (params, state["m"], state["v"], grads)]
        device = params["embed"].get_device()
        _on_current_gpu(device)
        counts = self._counts()
        for d in flat:
            for f, count in zip(fields, counts):
                if d[f].dtype != torch.float32 or d[f].numel() != count or d[f].get_device() != device:
                    raise ValueError(f"{f} must be float32, {count} values on cuda:{device}")
            lists.append(TrainGrads(*[_ptr(d[f]) for f in fields]))
        step = _step_tensor(state["step"], device)
        norm = None if max_norm is None else torch.empty(1, dtype=torch.float32, device=device)
        size = C.c_size_t()
        _check(lib().aecct_update_workspace_size(len(fields), C.byref(size)), "aecct_update_workspace_size")
        ws = torch.empty(size.value, dtype=torch.uint8, device=device)
        _check(lib().aecct_train_update(self._h, *[C.byref(t) for t in lists], C.byref(opt), step.data_ptr(),
                                        None if norm is None else norm.data_ptr(), ws.data_ptr(), size.value,
                                        _current_stream(device)), "aecct_train_update")
        return norm

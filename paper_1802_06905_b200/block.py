"""Operators of a gated feed-forward sub-block (``include/cconv_block.h``) on torch CUDA tensors.

    ffn_forward / ffn_backward                        y = (act(x Wg^T) * (x Wu^T)) Wd^T
    residual_norm_forward / residual_norm_backward    r' = scale r + gate norm(y) w_post, x = norm(r') w_pre
    residual_norm_quantize                            the same with x in 8 bits and scales
    fp8_product                                       8-bit operands with a scale for each block of 128
    quantize_blocks                                   the 8-bit values and the scales
    int4_product                                      4-bit weights with a scale for each group of a row
    quantize_groups                                   those weights, scales and zero points
    moe_forward                                       a mixture-of-experts layer for a few tokens
    gradient_norm, clip_gradients                     the norm over a list of gradients, and their clipping

Argument marshalling only: every step runs in ``libcconv.so``.  Results go to tensors that the caller
gives.  Calls are asynchronous on ``stream`` (default: the current stream of the operands' device).
``workspace`` is a CUDA tensor of at least the bytes that the matching ``*_workspace`` function gives; a
program that keeps one passes it, otherwise it is taken from torch's allocator for the call.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import binding
from .binding import OK, CconvError, EINVAL  # noqa: F401

TYPE_BF16, TYPE_FP16, TYPE_FP32 = 0, 1, 2
ACT_SILU, ACT_GELU, ACT_GELU_TANH, ACT_RELU = 0, 1, 2, 3
ACTS = {"silu": ACT_SILU, "gelu": ACT_GELU, "gelu_tanh": ACT_GELU_TANH, "relu": ACT_RELU}
_TYPES = {torch.bfloat16: TYPE_BF16, torch.float16: TYPE_FP16, torch.float32: TYPE_FP32}

EXPORTS = (
    "cconv_ffn_forward_workspace", "cconv_ffn_backward_workspace", "cconv_ffn_forward", "cconv_ffn_backward",
    "cconv_residual_norm_backward_workspace", "cconv_residual_norm_forward", "cconv_residual_norm_backward",
    "cconv_residual_norm_quantize",
    "cconv_fp8_product_workspace", "cconv_fp8_product", "cconv_quantize_blocks", "cconv_int4_product_workspace",
    "cconv_int4_product", "cconv_quantize_groups", "cconv_moe_workspace",
    "cconv_moe_forward", "cconv_clip_workspace",
    "cconv_gradient_norm", "cconv_clip_gradients", "cconv_block_status",
)

# The argument structures of the C ABI, field for field (P: address, q: 64-bit, i: 32-bit, f: float), without
# the workspace's address and size that end all but the last.
_MAT = "Pqq"
_FFN = struct.Struct("qqqii" + _MAT * 12)
_NORM = struct.Struct("qqiffxxxxq" + _MAT * 3 + "PP" + _MAT * 7 + "PP")
_FP8 = struct.Struct("qqqii" + _MAT * 5)
_QUANT = struct.Struct("qqii" + _MAT * 3)
_INT4 = struct.Struct("qqqiiii" + _MAT * 5)
_GROUPS = struct.Struct("qqiiii" + _MAT * 4)
_MOE = struct.Struct("qqqqiiii" + _MAT * 5 + "qqq" + _MAT * 3)
_TENSOR = struct.Struct("Pqqqqii")
_CLIP = struct.Struct("qPPffiiP")
_TWO = struct.Struct(_MAT * 2)  # behind the norm's, in the call with 8-bit results
_SPACE = struct.Struct("PQ")
_NO_SPACE = _SPACE.pack(0, 0)
_NONE = (0, 0, 0)

_fn = {}
_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _f(name):
    """The library's function ``name``; the library is loaded on the first call."""
    f = _fn.get(name)
    if f is None:
        f = getattr(binding.load_library(), name)
        if name.endswith("_workspace"):
            f.restype, f.argtypes = ctypes.c_int64, [ctypes.c_char_p]
        elif name == "cconv_block_status":
            f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int)]
        else:
            f.restype, f.argtypes = ctypes.c_int, [ctypes.c_char_p, ctypes.c_void_p]
        _fn[name] = f
    return f


def _mat(t, shape, dtype, dev, name):
    """(address, row stride, column stride) of a matrix operand, checked; dev: the device's index."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on cuda:{dev}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    rows, cols = t.stride()
    return t.data_ptr(), rows, cols


def _row(t, shape, dtype, dev, name):
    """As _mat, of a matrix whose rows are contiguous."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
        _mat(t, shape, dtype, dev, name)  # says what is wrong
    rows, cols = t.stride()
    if cols != 1 and shape[1] > 1:
        raise ValueError(f"{name} must have contiguous rows, got strides {t.stride()}")
    return t.data_ptr(), rows, cols


def _vec(t, n, dtype, dev, name):
    """Address of a vector operand (0: absent), checked."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != dev or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {(n,)} on cuda:{dev}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _type(t, name, allowed=_TYPES):
    """(type code, device index) of a matrix that gives a call its type and device."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    ty = allowed.get(t.dtype)
    if ty is None:
        raise ValueError(f"{name} has type {t.dtype}; supported: {', '.join(str(d) for d in allowed)}")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix, got shape {tuple(t.shape)}")
    return ty, dev


_HALF_TYPES = {torch.bfloat16: TYPE_BF16, torch.float16: TYPE_FP16}


def _need(name, args, dev):
    """Bytes of workspace of the call with these arguments."""
    f = _fn.get(name) or _f(name)
    if _current_device() == dev:
        n = f(args + _NO_SPACE)
    else:
        with torch.cuda.device(dev):
            n = f(args + _NO_SPACE)
    if n < 0:
        raise CconvError(n, name)
    return n


def _call(name, args, dev, stream):
    """Runs the entry point on ``stream``, with the operands' device current."""
    f = _fn.get(name) or _f(name)
    raw = _current_stream(dev) if stream is None else stream.cuda_stream
    if _current_device() == dev:
        rc = f(args, raw)
    else:
        with torch.cuda.device(dev):
            rc = f(args, raw)
    if rc != OK:
        raise CconvError(rc, name)


def _call_with_space(name, need, args, dev, workspace, stream):
    """_call with a workspace: the caller's, or one from torch's allocator (which reuses the memory in the
    order of the stream that it was taken on)."""
    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on cuda:{dev}")
        _call(name, args + _SPACE.pack(workspace.data_ptr(), workspace.numel() * workspace.element_size()), dev, stream)
        return
    n = _need(need, args, dev)
    if n == 0:
        _call(name, args + _NO_SPACE, dev, stream)
        return
    if stream is None:
        w = torch.empty(n, dtype=torch.uint8, device=dev)
    else:
        with torch.cuda.stream(stream):
            w = torch.empty(n, dtype=torch.uint8, device=dev)
    _call(name, args + _SPACE.pack(w.data_ptr(), n), dev, stream)


# ---- gated feed-forward block ---------------------------------------------------------------------

def _ffn_common(x, w_gate, w_up, w_down):
    dtype, dev = _type(x, "x", _HALF_TYPES)
    T, D = x.shape
    if w_gate.dim() != 2:
        raise ValueError(f"w_gate must be a matrix, got shape {tuple(w_gate.shape)}")
    F, dt = w_gate.shape[0], x.dtype
    mats = (x.data_ptr(), *x.stride(), *_mat(w_gate, (F, D), dt, dev, "w_gate"), *_mat(w_up, (F, D), dt, dev, "w_up"),
            *_mat(w_down, (D, F), dt, dev, "w_down"))
    return T, D, F, dtype, dt, dev, mats


def _ffn_forward_args(x, w_gate, w_up, w_down, out, act, gate_pre, up_pre):
    T, D, F, dtype, dt, dev, mats = _ffn_common(x, w_gate, w_up, w_down)
    if (gate_pre is None) != (up_pre is None):
        raise ValueError("gate_pre and up_pre are given together or not at all")
    pre = _NONE + _NONE
    if gate_pre is not None:
        pre = _mat(gate_pre, (T, F), dt, dev, "gate_pre") + _mat(up_pre, (T, F), dt, dev, "up_pre")
    return _FFN.pack(T, D, F, dtype, act, *mats, *pre, *_mat(out, (T, D), dt, dev, "out"), *(_NONE * 5)), dev


def ffn_forward_workspace(x, w_gate, w_up, w_down, out, act=ACT_SILU, gate_pre=None, up_pre=None):
    """cconv_ffn_forward_workspace: bytes of workspace of the call with these tensors."""
    args, dev = _ffn_forward_args(x, w_gate, w_up, w_down, out, act, gate_pre, up_pre)
    return _need("cconv_ffn_forward_workspace", args, dev)


def ffn_forward(x, w_gate, w_up, w_down, out, act=ACT_SILU, gate_pre=None, up_pre=None, workspace=None, stream=None):
    """cconv_ffn_forward: out = (act(x w_gate^T) * (x w_up^T)) w_down^T.

    x, out [T, D]; w_gate, w_up [F, D]; w_down [D, F]; bf16 or fp16, any strides.  Given ``gate_pre`` and
    ``up_pre`` [T, F], the pre-activations are written there for ffn_backward."""
    args, dev = _ffn_forward_args(x, w_gate, w_up, w_down, out, act, gate_pre, up_pre)
    _call_with_space("cconv_ffn_forward", "cconv_ffn_forward_workspace", args, dev, workspace, stream)
    return out


def _ffn_backward_args(dout, x, w_gate, w_up, w_down, gate_pre, up_pre, dx, dw_gate, dw_up, dw_down, act):
    T, D, F, dtype, dt, dev, mats = _ffn_common(x, w_gate, w_up, w_down)
    return _FFN.pack(T, D, F, dtype, act, *mats, *_mat(gate_pre, (T, F), dt, dev, "gate_pre"),
            *_mat(up_pre, (T, F), dt, dev, "up_pre"), *_NONE, *_mat(dout, (T, D), dt, dev, "dout"),
            *_mat(dx, (T, D), dt, dev, "dx"), *_mat(dw_gate, (F, D), dt, dev, "dw_gate"),
            *_mat(dw_up, (F, D), dt, dev, "dw_up"), *_mat(dw_down, (D, F), dt, dev, "dw_down")), dev


def ffn_backward_workspace(dout, x, w_gate, w_up, w_down, gate_pre, up_pre, dx, dw_gate, dw_up, dw_down, act=ACT_SILU):
    """cconv_ffn_backward_workspace: bytes of workspace of the call with these tensors."""
    args, dev = _ffn_backward_args(dout, x, w_gate, w_up, w_down, gate_pre, up_pre, dx, dw_gate, dw_up, dw_down, act)
    return _need("cconv_ffn_backward_workspace", args, dev)


def ffn_backward(dout, x, w_gate, w_up, w_down, gate_pre, up_pre, dx, dw_gate, dw_up, dw_down, act=ACT_SILU,
                 workspace=None, stream=None):
    """cconv_ffn_backward: the gradients dx, dw_gate, dw_up, dw_down (all written) for dout = dL/dy and
    the pre-activations that ffn_forward saved."""
    args, dev = _ffn_backward_args(dout, x, w_gate, w_up, w_down, gate_pre, up_pre, dx, dw_gate, dw_up, dw_down, act)
    _call_with_space("cconv_ffn_backward", "cconv_ffn_backward_workspace", args, dev, workspace, stream)
    return dx, dw_gate, dw_up, dw_down


# ---- norms before and after a block, with its gate and residual scale -------------------------------

def _gate(gate, T, D, rows_per_gate, dt, dev, name):
    if gate is None:
        return _NONE
    groups = -(-T // rows_per_gate) if rows_per_gate else 1
    return _row(gate, (groups, D), dt, dev, name)


def _norm_forward_args(resid, resid_out, norm_out, block, w_post, gate, w_pre, rows_per_gate, scale, eps):
    dtype, dev = _type(resid, "resid")
    shape = T, D = resid.shape
    dt = resid.dtype
    return _NORM.pack(
        T, D, dtype, scale, eps, rows_per_gate, *_row(resid, shape, dt, dev, "resid"),
        *(_NONE if block is None else _row(block, shape, dt, dev, "block")),
        *_gate(gate, T, D, rows_per_gate, dt, dev, "gate"), _vec(w_post, D, dt, dev, "w_post"),
        _vec(w_pre, D, dt, dev, "w_pre"), *_row(resid_out, shape, dt, dev, "resid_out"),
        *(_NONE if norm_out is None else _row(norm_out, shape, dt, dev, "norm_out")),
        0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) + _NO_SPACE, dev


def residual_norm_forward(resid, resid_out, norm_out=None, block=None, w_post=None, gate=None, w_pre=None,
                          rows_per_gate=0, scale=1.0, eps=1e-6, stream=None):
    """cconv_residual_norm_forward: resid_out = scale resid + gate norm(block) w_post and
    norm_out = norm(resid_out before its rounding) w_pre.

    Matrices [T, D] with contiguous rows, vectors [D]; bf16, fp16 or fp32.  Without ``block`` only the
    residual is scaled; without ``w_post`` the block is not normed; without ``gate`` it counts in full;
    without ``norm_out`` there is no second norm.  ``gate`` [ceil(T / rows_per_gate), D] has a row for
    each ``rows_per_gate`` tokens (0: one row for all).  ``resid_out`` may be ``resid``."""
    args, dev = _norm_forward_args(resid, resid_out, norm_out, block, w_post, gate, w_pre, rows_per_gate, scale, eps)
    _call("cconv_residual_norm_forward", args, dev, stream)
    return resid_out, norm_out


def residual_norm_quantize(resid, resid_out, q, q_scale, norm_out=None, block=None, w_post=None, gate=None, w_pre=None,
                           rows_per_gate=0, scale=1.0, eps=1e-6, stream=None):
    """cconv_residual_norm_quantize: residual_norm_forward whose x = norm(resid_out before its rounding) w_pre is
    written as float8_e4m3fn values ``q`` [T, D] (contiguous rows) and fp32 scales ``q_scale`` [T, ceil(D/128)].

    q = x / q_scale and q_scale = max|x| / 448 as quantize_blocks gives them, for x before its rounding to the
    type.  ``norm_out``, if given, gets x rounded to the type.  Everything else as residual_norm_forward."""
    args, dev = _norm_forward_args(resid, resid_out, norm_out, block, w_post, gate, w_pre, rows_per_gate, scale, eps)
    T, D = resid.shape
    args += _TWO.pack(*_row(q, (T, D), torch.float8_e4m3fn, dev, "q"),
                      *_mat(q_scale, (T, (D + 127) // 128), torch.float32, dev, "q_scale"))
    _call("cconv_residual_norm_quantize", args, dev, stream)
    return resid_out, q, q_scale


def _norm_backward_args(dresid_out, dnorm_out, resid_out, dresid, block, dblock, w_post, dw_post, gate, dgate, w_pre,
                        dw_pre, rows_per_gate, scale, eps):
    dtype, dev = _type(dresid, "dresid")
    shape = T, D = dresid.shape
    dt = dresid.dtype

    def opt(t, name):
        return _NONE if t is None else _row(t, shape, dt, dev, name)
    return _NORM.pack(T, D, dtype, scale, eps, rows_per_gate, *_NONE, *opt(block, "block"),
            *_gate(gate, T, D, rows_per_gate, dt, dev, "gate"), _vec(w_post, D, dt, dev, "w_post"),
            _vec(w_pre, D, dt, dev, "w_pre"), *opt(resid_out, "resid_out"), *_NONE, *opt(dresid_out, "dresid_out"),
            *opt(dnorm_out, "dnorm_out"), *_row(dresid, shape, dt, dev, "dresid"), *opt(dblock, "dblock"),
            *_gate(dgate, T, D, rows_per_gate, dt, dev, "dgate"), _vec(dw_post, D, dt, dev, "dw_post"),
            _vec(dw_pre, D, dt, dev, "dw_pre")), dev


def residual_norm_backward_workspace(dresid_out, dnorm_out, resid_out, dresid, block=None, dblock=None, w_post=None,
                                     dw_post=None, gate=None, dgate=None, w_pre=None, dw_pre=None, rows_per_gate=0,
                                     scale=1.0, eps=1e-6):
    """cconv_residual_norm_backward_workspace: bytes of workspace of the call with these tensors."""
    args, dev = _norm_backward_args(dresid_out, dnorm_out, resid_out, dresid, block, dblock, w_post, dw_post, gate,
                                    dgate, w_pre, dw_pre, rows_per_gate, scale, eps)
    return _need("cconv_residual_norm_backward_workspace", args, dev)


def residual_norm_backward(dresid_out, dnorm_out, resid_out, dresid, block=None, dblock=None, w_post=None, dw_post=None,
                           gate=None, dgate=None, w_pre=None, dw_pre=None, rows_per_gate=0, scale=1.0, eps=1e-6,
                           workspace=None, stream=None):
    """cconv_residual_norm_backward: dresid, dblock, dw_post, dgate and dw_pre, each given exactly when
    its operand is (all written).

    ``dresid_out`` is the gradient of resid_out by its direct uses, ``dnorm_out`` that of norm_out; one
    of them may be None.  ``resid_out`` is the forward result (not read without ``dnorm_out``).
    ``dresid`` may be ``dresid_out``."""
    args, dev = _norm_backward_args(dresid_out, dnorm_out, resid_out, dresid, block, dblock, w_post, dw_post, gate,
                                    dgate, w_pre, dw_pre, rows_per_gate, scale, eps)
    _call_with_space("cconv_residual_norm_backward", "cconv_residual_norm_backward_workspace", args, dev, workspace, stream)
    return dresid, dblock, dw_post, dgate, dw_pre


# ---- 8-bit product and quantisation -----------------------------------------------------------------

def _fp8_args(a, a_scale, b, b_scale, out):
    dtype, dev = _type(out, "out")
    M, N = out.shape
    if a.dim() != 2:
        raise ValueError(f"a must be a matrix, got shape {tuple(a.shape)}")
    K, e4m3, f32 = a.shape[1], torch.float8_e4m3fn, torch.float32
    kb = (K + 127) // 128
    return _FP8.pack(M, N, K, dtype, 0, *_mat(a, (M, K), e4m3, dev, "a"), *_mat(b, (N, K), e4m3, dev, "b"),
            *_mat(a_scale, (M, kb), f32, dev, "a_scale"), *_mat(b_scale, ((N + 127) // 128, kb), f32, dev, "b_scale"),
            out.data_ptr(), *out.stride()), dev


def fp8_product_workspace(a, a_scale, b, b_scale, out):
    """cconv_fp8_product_workspace: bytes of workspace of the call with these tensors."""
    args, dev = _fp8_args(a, a_scale, b, b_scale, out)
    return _need("cconv_fp8_product_workspace", args, dev)


def fp8_product(a, a_scale, b, b_scale, out, workspace=None, stream=None):
    """cconv_fp8_product: out[m,n] = sum_kb a_scale[m,kb] b_scale[n/128,kb] sum_{k in kb} a[m,k] b[n,k].

    a [M, K], b [N, K] float8_e4m3fn; a_scale [M, ceil(K/128)], b_scale [ceil(N/128), ceil(K/128)] fp32;
    out [M, N] bf16, fp16 or fp32; any strides."""
    args, dev = _fp8_args(a, a_scale, b, b_scale, out)
    _call_with_space("cconv_fp8_product", "cconv_fp8_product_workspace", args, dev, workspace, stream)
    return out


def quantize_blocks(x, q, scale, block_rows=1, stream=None):
    """cconv_quantize_blocks: q = x / scale in float8_e4m3fn, scale = max|x| / 448 of each block of
    ``block_rows`` (1 or 128) x 128 elements, fp32 [ceil(T/block_rows), ceil(D/128)]."""
    dtype, dev = _type(x, "x")
    T, D = x.shape
    if block_rows not in (1, 128):
        raise ValueError(f"block_rows must be 1 or 128, got {block_rows}")
    args = _QUANT.pack(T, D, dtype, block_rows, x.data_ptr(), *x.stride(), *_mat(q, (T, D), torch.float8_e4m3fn, dev, "q"),
                       *_mat(scale, (-(-T // block_rows), -(-D // 128)), torch.float32, dev, "scale"))
    _call("cconv_quantize_blocks", args, dev, stream)
    return q, scale


# ---- 4-bit weights -----------------------------------------------------------------------------------

def _scale_type(scale):
    ty = _TYPES.get(scale.dtype)
    if ty is None:
        raise ValueError(f"scale has type {scale.dtype}; supported: {', '.join(str(d) for d in _TYPES)}")
    return ty


def _group(group):
    if group not in (32, 64, 128):
        raise ValueError(f"group must be 32, 64 or 128, got {group}")


def _int4_args(x, q, scale, out, zero, group):
    dtype, dev = _type(x, "x", _HALF_TYPES)
    M, K = x.shape
    _group(group)
    if q.dim() != 2:
        raise ValueError(f"q must be a matrix, got shape {tuple(q.shape)}")
    N, groups, u8 = q.shape[0], (K + group - 1) // group, torch.uint8
    return _INT4.pack(M, N, K, dtype, _scale_type(scale), group, 0, x.data_ptr(), *x.stride(),
                      *_mat(q, (N, (K + 1) // 2), u8, dev, "q"), *_mat(scale, (N, groups), scale.dtype, dev, "scale"),
                      *(_NONE if zero is None else _mat(zero, (N, groups), u8, dev, "zero")),
                      *_mat(out, (M, N), x.dtype, dev, "out")), dev


def int4_product_workspace(x, q, scale, out, zero=None, group=128):
    """cconv_int4_product_workspace: bytes of workspace of the call with these tensors."""
    args, dev = _int4_args(x, q, scale, out, zero, group)
    return _need("cconv_int4_product_workspace", args, dev)


def int4_product(x, q, scale, out, zero=None, group=128, workspace=None, stream=None):
    """cconv_int4_product: out[m,n] = sum_g scale[n,g] sum_{k in group g} (q[n,k] - zero[n,g]) x[m,k].

    x [M, K], out [M, N] bf16 or fp16; q [N, ceil(K/2)] uint8, element 2j of a row in the low half of byte j; scale
    [N, ceil(K/group)] bf16, fp16 or fp32; zero of the same shape, uint8 of 0 to 15 (None: 8 throughout); group 32, 64 or
    128; any strides.  With more than 64 tokens the weights scale (q - zero) are rounded to the precision of x's type."""
    args, dev = _int4_args(x, q, scale, out, zero, group)
    _call_with_space("cconv_int4_product", "cconv_int4_product_workspace", args, dev, workspace, stream)
    return out


def quantize_groups(w, q, scale, zero=None, group=128, stream=None):
    """cconv_quantize_groups: the 4-bit values q [N, ceil(K/2)] (uint8, two a byte) and scales [N, ceil(K/group)]
    of w [N, K], bf16, fp16 or fp32 each; with ``zero`` (uint8, as scale) a group's range need not be symmetric."""
    dtype, dev = _type(w, "w")
    N, K = w.shape
    _group(group)
    groups, u8 = (K + group - 1) // group, torch.uint8
    args = _GROUPS.pack(N, K, dtype, _scale_type(scale), group, 0, w.data_ptr(), *w.stride(),
                        *_mat(q, (N, (K + 1) // 2), u8, dev, "q"), *_mat(scale, (N, groups), scale.dtype, dev, "scale"),
                        *(_NONE if zero is None else _mat(zero, (N, groups), u8, dev, "zero")))
    _call("cconv_quantize_groups", args, dev, stream)
    return q, scale, zero


# ---- mixture of experts ------------------------------------------------------------------------------

def _experts(t, shape, dtype, dev, name):
    """((address, row stride, column stride) of expert 0's matrix, elements to the next one's), checked."""
    if t.dtype is not dtype or t.get_device() != dev or t.shape != shape:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on cuda:{dev}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    expert, rows, cols = t.stride()
    return (t.data_ptr(), rows, cols), expert


def _moe_args(x, w_router, w_gate, w_up, w_down, out, ids, weights, act, normalize):
    dtype, dev = _type(x, "x", _HALF_TYPES)
    T, D = x.shape
    if w_gate.dim() != 3:
        raise ValueError(f"w_gate must have the dimensions experts, hidden channels, channels, got shape {tuple(w_gate.shape)}")
    E, F, dt = w_gate.shape[0], w_gate.shape[1], x.dtype
    if ids.dim() != 2 or ids.shape[1] < 1:
        raise ValueError(f"ids must be a matrix with a column for each choice, got shape {tuple(ids.shape)}")
    top_k = ids.shape[1]
    gate, gate_stride = _experts(w_gate, (E, F, D), dt, dev, "w_gate")
    up, up_stride = _experts(w_up, (E, F, D), dt, dev, "w_up")
    down, down_stride = _experts(w_down, (E, D, F), dt, dev, "w_down")
    return _MOE.pack(T, D, F, E, dtype, act, top_k, int(normalize), x.data_ptr(), *x.stride(),
                     *(_NONE if w_router is None else _mat(w_router, (E, D), dt, dev, "w_router")), *gate, *up, *down,
                     gate_stride, up_stride, down_stride, *_mat(ids, (T, top_k), torch.int32, dev, "ids"),
                     *_mat(weights, (T, top_k), torch.float32, dev, "weights"), *_mat(out, (T, D), dt, dev, "out")), dev


def moe_workspace(x, w_router, w_gate, w_up, w_down, out, ids, weights, act=ACT_SILU, normalize=True):
    """cconv_moe_workspace: bytes of workspace of the call with these tensors."""
    args, dev = _moe_args(x, w_router, w_gate, w_up, w_down, out, ids, weights, act, normalize)
    return _need("cconv_moe_workspace", args, dev)


def moe_forward(x, w_router, w_gate, w_up, w_down, out, ids, weights, act=ACT_SILU, normalize=True, workspace=None,
                stream=None):
    """cconv_moe_forward: out[t] = sum_j weights[t,j] (act(x Wg_e^T) * (x Wu_e^T)) Wd_e^T,  e = ids[t,j].

    x, out [T, D]; w_gate, w_up [E, F, D]; w_down [E, D, F]; bf16 or fp16, any strides.  With ``w_router`` [E, D], ids
    (int32 [T, k]) and weights (fp32 [T, k]) are written: the k experts of the largest x w_router^T in falling order
    (of equal ones the lower number first) and the softmax over them (``normalize``) or over all experts.  Without
    (None) they are read: numbers outside 0 .. E - 1 add nothing.  Made for a few tokens: 64 at a time."""
    args, dev = _moe_args(x, w_router, w_gate, w_up, w_down, out, ids, weights, act, normalize)
    _call_with_space("cconv_moe_forward", "cconv_moe_workspace", args, dev, workspace, stream)
    return out, ids, weights


# ---- the norm of a list of gradients, and clipping ----------------------------------------------------

def _as_rows(t, name):
    """(rows, cols, row stride, col stride) of a tensor's elements, taken in the order of its strides."""
    if t.is_contiguous():
        return 1, t.numel(), t.numel(), 1
    dims = []  # (size, stride), outer ones first, neighbours that follow one another merged
    for size, stride in sorted(((n, st) for n, st in zip(t.shape, t.stride()) if n > 1), key=lambda d: -d[1]):
        if dims and dims[-1][1] == size * stride:
            dims[-1] = (dims[-1][0] * size, stride)
        else:
            dims.append((size, stride))
    if len(dims) > 2:
        raise ValueError(f"{name}: a tensor of shape {tuple(t.shape)} and strides {t.stride()} is no list of rows")
    dims = [(1, t.numel())] * (2 - len(dims)) + dims
    return dims[0][0], dims[1][0], dims[0][1], dims[1][1]


class TensorList:
    """A list of tensors of one device as the library takes it, for lists that several calls share: gradients that
    a program keeps from step to step.  It holds the tensors; their storage, shapes and strides must not change."""

    def __init__(self, tensors, name="tensors"):
        self.tensors = list(tensors)
        if not self.tensors:
            raise ValueError(f"{name} must hold at least one tensor")
        self.device = self.tensors[0].get_device()
        packed = []
        for i, t in enumerate(self.tensors):
            ty = _TYPES.get(t.dtype)
            if ty is None or t.get_device() != self.device or self.device < 0:
                raise ValueError(f"{name}[{i}] must be a bf16, fp16 or fp32 tensor on one CUDA device, got {t.dtype} on {t.device}")
            packed.append(_TENSOR.pack(t.data_ptr(), *_as_rows(t, f"{name}[{i}]"), ty, 0))
        # of tensors of the same layout the elements correspond in the order above
        self.layout = repr([(str(t.dtype), tuple(t.shape), t.is_contiguous() or t.stride()) for t in self.tensors])
        self._array = ctypes.create_string_buffer(b"".join(packed))
        self.address, self.count = ctypes.addressof(self._array), len(packed)

    def __len__(self):
        return self.count


def _tensor_list(tensors, name):
    return tensors if isinstance(tensors, TensorList) else TensorList(tensors, name)


def _clip_args(grads, outs, max_norm, eps, norm_given, norm):
    if outs is not None and (outs.device != grads.device or outs.layout != grads.layout):
        raise ValueError("outs must have the types, shapes, strides and device of grads")
    return _CLIP.pack(grads.count, grads.address, 0 if outs is None else outs.address, max_norm, eps, norm_given, 0,
                      _vec(norm, 1, torch.float32, grads.device, "norm"))


def clip_workspace(grads):
    """cconv_clip_workspace: bytes of workspace of gradient_norm and clip_gradients with these tensors."""
    grads = _tensor_list(grads, "grads")
    return _need("cconv_clip_workspace", _CLIP.pack(grads.count, grads.address, 0, 1.0, 0.0, 0, 0, 0), grads.device)


def gradient_norm(grads, norm, workspace=None, stream=None):
    """cconv_gradient_norm: norm[0] = sqrt of the sum of squares over all elements of ``grads``.

    ``grads``: a list of bf16, fp16 and fp32 tensors of one device, or a TensorList; ``norm``: fp32 [1]."""
    grads = _tensor_list(grads, "grads")
    args = _clip_args(grads, None, 1.0, 0.0, 0, norm)
    _call_with_space("cconv_gradient_norm", "cconv_clip_workspace", args, grads.device, workspace, stream)
    return norm


def clip_gradients(grads, max_norm, norm, outs=None, eps=1e-6, norm_given=False, workspace=None, stream=None):
    """cconv_clip_gradients: every gradient times min(1, max_norm / (norm + eps)), in place or to ``outs``.

    ``grads``, ``outs``: lists of tensors, or TensorLists; ``norm`` (fp32 [1]) gets the norm over all of them, or,
    with ``norm_given``, holds it: that of other ranks' gradients too, say.  Nothing waits for the host.  A list is described
    anew in each call (1.5 to 2 us a tensor on the host); a program that keeps its gradients makes a TensorList of them."""
    grads = _tensor_list(grads, "grads")
    outs = None if outs is None else _tensor_list(outs, "outs")
    args = _clip_args(grads, outs, max_norm, eps, int(norm_given), norm)
    if norm_given:
        _call("cconv_clip_gradients", args + _NO_SPACE, grads.device, stream)
    else:
        _call_with_space("cconv_clip_gradients", "cconv_clip_workspace", args, grads.device, workspace, stream)
    return norm


def status(stream=None):
    """cconv_block_status: synchronises and returns (code, detail bit mask) of the product kernels that
    ran on the current device since the last call, and clears it."""
    detail = ctypes.c_int(0)
    raw = torch.cuda.current_stream().cuda_stream if stream is None else stream.cuda_stream
    return _f("cconv_block_status")(raw, ctypes.byref(detail)), detail.value

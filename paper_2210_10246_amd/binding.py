"""Thin binding of libtempo.so: same names as the C ABI, argument marshalling only.

The calls go through _native.so (csrc/binding.cpp), which makes the checks below in native code and
calls the C ABI on the current stream.  Whatever it does not take (an explicit stream, an argument
that one of the checks refuses or that is no plain tensor) goes through the ctypes path here, which
raises; so does every call if _native.so cannot be loaded, at 8-10 us of Python each.

Tensors are torch CUDA tensors (PyTorch supplies device memory and the stream; every step
of the layers runs in the HIP kernels).  Outputs are written into tensors the caller passes.
There is no CPU fallback: if the shared library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtempo.so")

TEMPO_OK = 0
TEMPO_F32, TEMPO_BF16 = 0, 1
TEMPO_GELU_ERF, TEMPO_GELU_TANH = 0, 1
_DT = {torch.float32: TEMPO_F32, torch.bfloat16: TEMPO_BF16}
_KIND = {"erf": TEMPO_GELU_ERF, "tanh": TEMPO_GELU_TANH}
_LAYOUT = {"half": 0, "interleaved": 1}
_GLU_KIND = {"silu": 0, "gelu_erf": 1, "gelu_tanh": 2}

_vp, _i64, _u64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_uint64
_int, _f32, _sz = ctypes.c_int, ctypes.c_float, ctypes.c_size_t


class _RotaryHeads(ctypes.Structure):
    _fields_ = [("x", _vp), ("y", _vp), ("heads", _i64), ("x_strides", _i64 * 3), ("y_strides", _i64 * 3)]


class _RotaryPositions(ctypes.Structure):
    _fields_ = [("positions", _vp), ("bits", _int), ("strides", _i64 * 2), ("start", _i64)]


_rotary_args = [ctypes.POINTER(_RotaryHeads), ctypes.POINTER(_RotaryHeads), _vp, ctypes.POINTER(_RotaryPositions), _i64, _i64,
                _i64, _i64, _int, _f32, _int, _vp]

_SIGNATURES = {
    "tempo_status_string": (ctypes.c_char_p, [_int]),
    "tempo_version": (_int, []),
    "tempo_set_launch_param": (_int, [_int, _int]),
    "tempo_get_launch_param": (_int, [_int]),
    "tempo_copy": (_int, [_vp, _vp, _i64, _int, _vp]),
    "tempo_copy_streams": (_int, [_vp, _int, _vp, _int, _i64, _vp]),
    "tempo_gelu_fwd": (_int, [_vp, _vp, _vp, _i64, _int, _int, _vp]),
    "tempo_gelu_bwd": (_int, [_vp, _vp, _vp, _vp, _i64, _int, _int, _vp]),
    "tempo_silu_fwd": (_int, [_vp, _vp, _vp, _i64, _int, _vp]),
    "tempo_silu_bwd": (_int, [_vp, _vp, _vp, _vp, _i64, _int, _vp]),
    "tempo_layernorm_fwd": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _f32, _int, _vp]),
    "tempo_layernorm_bwd_workspace_bytes": (_sz, [_i64, _i64]),
    "tempo_layernorm_bwd": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _i64, _i64,
                                   _int, _vp]),
    "tempo_layernorm_bwd_static": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _i64, _int,
                                          _vp]),
    "tempo_attn_softmax_dropout_fwd": (_int, [_vp, _vp, _int, _vp, _vp, _vp, _i64, _i64, _i64,
                                              _i64, _f32, _u64, _u64, _int, _vp]),
    "tempo_attn_softmax_dropout_bwd": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64,
                                              _f32, _int, _vp]),
    "tempo_attn_softmax_dropout_bwd_bytemask": (_int, [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64,
                                                       _i64, _f32, _int, _vp]),
    "tempo_attn_softmax_dropout_bwd_regen": (_int, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _i64,
                                                    _f32, _u64, _u64, _int, _vp]),
    "tempo_rotary_fwd": (_int, _rotary_args),
    "tempo_rotary_bwd": (_int, _rotary_args),
    "tempo_glu_fwd_workspace_bytes": (_sz, [_i64, _i64, _i64, _int]),
    "tempo_glu_bwd_workspace_bytes": (_sz, [_i64, _i64, _i64, _int]),
    "tempo_glu_fwd": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _sz, _i64, _i64, _i64, _int, _int, _vp]),
    "tempo_glu_bwd": (_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _i64, _i64, _i64, _int, _int, _vp]),
    "tempo_mask_bits_to_bytes": (_int, [_vp, _vp, _i64, _vp]),
    "tempo_mask_bytes_to_bits": (_int, [_vp, _vp, _i64, _vp]),
}

_lib = None
_native = None  # the module _native.so, once load() has run and found it


class TempoError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def load() -> ctypes.CDLL:
    """Load libtempo.so (built in-tree by build.py), raising if it is missing, and _native.so."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} not found: build it with `python -m paper_2210_10246_amd.build` "
                "(there is no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        try:
            from . import _native as native
            _native = native
        except ImportError as e:  # not built, or for another torch
            warnings.warn(f"_native.so: {e}; calls go through ctypes, which is slower: build it with "
                          "`python -m paper_2210_10246_amd.build`", RuntimeWarning)
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().tempo_status_string(status).decode()


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous CUDA tensors")
    return t.data_ptr()


def _want(name: str, t: Optional[torch.Tensor], dtype, numel: Optional[int] = None,
          at_least: Optional[int] = None):
    """The C ABI reads raw bytes: a tensor of another dtype or size would be misread, or read
    out of bounds, on the device.  None is let through (optional arguments)."""
    if t is None:
        return
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements, got {t.numel()}")
    if at_least is not None and t.numel() < at_least:
        raise ValueError(f"{name} must have at least {at_least} elements, got {t.numel()}")


def _act_dtype(name: str, t: torch.Tensor) -> int:
    if t.dtype not in _DT:
        raise ValueError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    return _DT[t.dtype]


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _check(status: int, where: str):
    if status != TEMPO_OK:
        raise TempoError(status, where)


def mask_words(n: int) -> int:
    return (n + 31) // 32


def tempo_set_launch_param(key: int, value: int):
    _check(load().tempo_set_launch_param(key, value), "tempo_set_launch_param")


def tempo_get_launch_param(key: int) -> int:
    return load().tempo_get_launch_param(key)


def tempo_copy(src, dst, blocks_per_cu=16, stream=None):
    """Plain streaming copy of src into dst (same byte size, multiple of 16)."""
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    _check(load().tempo_copy(_ptr(src), _ptr(dst), nbytes, blocks_per_cu, _stream(stream)),
           "tempo_copy")


def tempo_copy_streams(reads, writes, stream=None):
    """Plain streaming kernel over len(reads) input and len(writes) output tensors of one size."""
    nbytes = reads[0].numel() * reads[0].element_size()
    for t in list(reads) + list(writes):
        if t.numel() * t.element_size() != nbytes:
            raise ValueError("all tensors must have the same size in bytes")
    r = (ctypes.c_void_p * len(reads))(*[_ptr(t) for t in reads])
    w = (ctypes.c_void_p * len(writes))(*[_ptr(t) for t in writes])
    _check(load().tempo_copy_streams(r, len(reads), w, len(writes), nbytes, _stream(stream)),
           "tempo_copy_streams")


def tempo_gelu_fwd(x, y, mask, kind="erf", stream=None):
    """(y, mask) = GELU*(x); y may be x."""
    if stream is None and _native is not None:
        status = _native.tempo_gelu_fwd(x, y, mask, kind)
        if status is not None:
            return _check(status, "tempo_gelu_fwd")
    n = x.numel()
    dt = _act_dtype("x", x)
    _want("y", y, x.dtype, n)
    _want("mask", mask, torch.int32, at_least=mask_words(n))
    _check(load().tempo_gelu_fwd(_ptr(x), _ptr(y), _ptr(mask), n, dt,
                                 _KIND[kind], _stream(stream)), "tempo_gelu_fwd")


def tempo_gelu_bwd(dy, y, mask, dx, kind="erf", stream=None):
    """dx = dy * GELU'(GELU*^-1(y, mask)); dx may be dy."""
    if stream is None and _native is not None:
        status = _native.tempo_gelu_bwd(dy, y, mask, dx, kind)
        if status is not None:
            return _check(status, "tempo_gelu_bwd")
    n = y.numel()
    dt = _act_dtype("y", y)
    _want("dy", dy, y.dtype, n)
    _want("dx", dx, y.dtype, n)
    _want("mask", mask, torch.int32, at_least=mask_words(n))
    _check(load().tempo_gelu_bwd(_ptr(dy), _ptr(y), _ptr(mask), _ptr(dx), n, dt,
                                 _KIND[kind], _stream(stream)), "tempo_gelu_bwd")


def tempo_silu_fwd(x, y, mask, stream=None):
    """(y, mask) = SiLU*(x); y may be x."""
    if stream is None and _native is not None:
        status = _native.tempo_silu_fwd(x, y, mask)
        if status is not None:
            return _check(status, "tempo_silu_fwd")
    n = x.numel()
    dt = _act_dtype("x", x)
    _want("y", y, x.dtype, n)
    _want("mask", mask, torch.int32, at_least=mask_words(n))
    _check(load().tempo_silu_fwd(_ptr(x), _ptr(y), _ptr(mask), n, dt,
                                 _stream(stream)), "tempo_silu_fwd")


def tempo_silu_bwd(dy, y, mask, dx, stream=None):
    """dx = dy * SiLU'(SiLU*^-1(y, mask)); dx may be dy."""
    if stream is None and _native is not None:
        status = _native.tempo_silu_bwd(dy, y, mask, dx)
        if status is not None:
            return _check(status, "tempo_silu_bwd")
    n = y.numel()
    dt = _act_dtype("y", y)
    _want("dy", dy, y.dtype, n)
    _want("dx", dx, y.dtype, n)
    _want("mask", mask, torch.int32, at_least=mask_words(n))
    _check(load().tempo_silu_bwd(_ptr(dy), _ptr(y), _ptr(mask), _ptr(dx), n, dt,
                                 _stream(stream)), "tempo_silu_bwd")


def tempo_layernorm_fwd(x, gamma, beta, y, rstd, mean=None, eps=1e-5, stream=None):
    if stream is None and _native is not None:
        status = _native.tempo_layernorm_fwd(x, gamma, beta, y, rstd, mean, eps)
        if status is not None:
            return _check(status, "tempo_layernorm_fwd")
    M = x.shape[-1]
    N = x.numel() // M if M else 0
    dt = _act_dtype("x", x)
    _want("y", y, x.dtype, x.numel())
    _want("gamma", gamma, torch.float32, M)
    _want("beta", beta, torch.float32, M)
    _want("rstd", rstd, torch.float32, N)
    _want("mean", mean, torch.float32, N)
    _check(load().tempo_layernorm_fwd(_ptr(x), _ptr(gamma), _ptr(beta), _ptr(y), _ptr(rstd),
                                      _ptr(mean), N, M, eps, dt, _stream(stream)),
           "tempo_layernorm_fwd")


def tempo_layernorm_bwd_workspace_bytes(N: int, M: int) -> int:
    return load().tempo_layernorm_bwd_workspace_bytes(N, M)


def tempo_layernorm_bwd(dy, y, gamma, beta, rstd, dx, dgamma, dbeta, workspace, stream=None):
    if stream is None and _native is not None:
        status = _native.tempo_layernorm_bwd(dy, y, gamma, beta, rstd, dx, dgamma, dbeta, workspace)
        if status is not None:
            return _check(status, "tempo_layernorm_bwd")
    M = y.shape[-1]
    N = y.numel() // M if M else 0
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    dt = _act_dtype("y", y)
    _want("dy", dy, y.dtype, y.numel())
    _want("dx", dx, y.dtype, y.numel())
    _want("gamma", gamma, torch.float32, M)
    _want("beta", beta, torch.float32, M)
    _want("rstd", rstd, torch.float32, N)
    _want("dgamma", dgamma, torch.float32, M)
    _want("dbeta", dbeta, torch.float32, M)
    _check(load().tempo_layernorm_bwd(_ptr(dy), _ptr(y), _ptr(gamma), _ptr(beta), _ptr(rstd),
                                      _ptr(dx), _ptr(dgamma), _ptr(dbeta), _ptr(workspace),
                                      ws_bytes, N, M, dt, _stream(stream)),
           "tempo_layernorm_bwd")


def tempo_layernorm_bwd_static(dy, y, gamma, beta, rstd, dx, dgamma, dbeta, stream=None):
    """tempo_layernorm_bwd with the library's static scratch array as workspace."""
    if stream is None and _native is not None:
        status = _native.tempo_layernorm_bwd_static(dy, y, gamma, beta, rstd, dx, dgamma, dbeta)
        if status is not None:
            return _check(status, "tempo_layernorm_bwd_static")
    M = y.shape[-1]
    N = y.numel() // M if M else 0
    dt = _act_dtype("y", y)
    _want("dy", dy, y.dtype, y.numel())
    _want("dx", dx, y.dtype, y.numel())
    _want("gamma", gamma, torch.float32, M)
    _want("beta", beta, torch.float32, M)
    _want("rstd", rstd, torch.float32, N)
    _want("dgamma", dgamma, torch.float32, M)
    _want("dbeta", dbeta, torch.float32, M)
    _check(load().tempo_layernorm_bwd_static(_ptr(dy), _ptr(y), _ptr(gamma), _ptr(beta), _ptr(rstd),
                                             _ptr(dx), _ptr(dgamma), _ptr(dbeta), N, M, dt,
                                             _stream(stream)), "tempo_layernorm_bwd_static")


def tempo_attn_softmax_dropout_fwd(scores, key_len, causal, probs, out, keep_bits, p, seed, offset,
                                   stream=None):
    if stream is None and _native is not None:
        status = _native.tempo_attn_softmax_dropout_fwd(scores, key_len, causal, probs, out,
                                                        keep_bits, p, seed, offset)
        if status is not None:
            return _check(status, "tempo_attn_softmax_dropout_fwd")
    B, A, Sq, Sk = scores.shape
    n = scores.numel()
    dt = _act_dtype("scores", scores)
    _want("key_len", key_len, torch.int32, B)
    _want("probs", probs, scores.dtype, n)
    _want("out", out, scores.dtype, n)
    _want("keep_bits", keep_bits, torch.int32, at_least=mask_words(n))
    _check(load().tempo_attn_softmax_dropout_fwd(
        _ptr(scores), _ptr(key_len), int(bool(causal)), _ptr(probs), _ptr(out), _ptr(keep_bits),
        B, A, Sq, Sk, p, seed, offset, dt, _stream(stream)),
        "tempo_attn_softmax_dropout_fwd")


def tempo_attn_softmax_dropout_bwd(dout, probs, keep_bits, dscores, out_recomputed, p, stream=None):
    if stream is None and _native is not None:
        status = _native.tempo_attn_softmax_dropout_bwd(dout, probs, keep_bits, dscores,
                                                        out_recomputed, p)
        if status is not None:
            return _check(status, "tempo_attn_softmax_dropout_bwd")
    B, A, Sq, Sk = probs.shape
    n = probs.numel()
    dt = _act_dtype("probs", probs)
    _want("dout", dout, probs.dtype, n)
    _want("dscores", dscores, probs.dtype, n)
    _want("out_recomputed", out_recomputed, probs.dtype, n)
    _want("keep_bits", keep_bits, torch.int32, at_least=mask_words(n))
    _check(load().tempo_attn_softmax_dropout_bwd(
        _ptr(dout), _ptr(probs), _ptr(keep_bits), _ptr(dscores), _ptr(out_recomputed),
        B, A, Sq, Sk, p, dt, _stream(stream)),
        "tempo_attn_softmax_dropout_bwd")


def tempo_attn_softmax_dropout_bwd_bytemask(dout, probs, keep_bytes, dscores, out_recomputed, p,
                                            stream=None):
    """Backward reading a mask of one byte per element (uint8 or bool tensor; non-zero = kept)."""
    if stream is None and _native is not None:
        status = _native.tempo_attn_softmax_dropout_bwd_bytemask(dout, probs, keep_bytes, dscores,
                                                                 out_recomputed, p)
        if status is not None:
            return _check(status, "tempo_attn_softmax_dropout_bwd_bytemask")
    B, A, Sq, Sk = probs.shape
    n = probs.numel()
    dt = _act_dtype("probs", probs)
    _want("dout", dout, probs.dtype, n)
    _want("dscores", dscores, probs.dtype, n)
    _want("out_recomputed", out_recomputed, probs.dtype, n)
    if keep_bytes.dtype not in (torch.uint8, torch.bool) or keep_bytes.numel() != n:
        raise ValueError(f"keep_bytes must be uint8 or bool with {n} elements, got "
                         f"{keep_bytes.dtype} with {keep_bytes.numel()}")
    _check(load().tempo_attn_softmax_dropout_bwd_bytemask(
        _ptr(dout), _ptr(probs), _ptr(keep_bytes), _ptr(dscores), _ptr(out_recomputed),
        B, A, Sq, Sk, p, dt, _stream(stream)), "tempo_attn_softmax_dropout_bwd_bytemask")


def tempo_attn_softmax_dropout_bwd_regen(dout, probs, dscores, out_recomputed, p, seed, offset,
                                         stream=None):
    if stream is None and _native is not None:
        status = _native.tempo_attn_softmax_dropout_bwd_regen(dout, probs, dscores, out_recomputed,
                                                              p, seed, offset)
        if status is not None:
            return _check(status, "tempo_attn_softmax_dropout_bwd_regen")
    B, A, Sq, Sk = probs.shape
    n = probs.numel()
    dt = _act_dtype("probs", probs)
    _want("dout", dout, probs.dtype, n)
    _want("dscores", dscores, probs.dtype, n)
    _want("out_recomputed", out_recomputed, probs.dtype, n)
    _check(load().tempo_attn_softmax_dropout_bwd_regen(
        _ptr(dout), _ptr(probs), _ptr(dscores), _ptr(out_recomputed), B, A, Sq, Sk, p, seed,
        offset, dt, _stream(stream)), "tempo_attn_softmax_dropout_bwd_regen")


def _same_device(*tensors):
    """All on the current device: the call goes to its stream."""
    if not all(t.is_cuda for t in tensors if t is not None):
        raise ValueError("tensors must be CUDA tensors")
    current = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.device.index != current:
            raise ValueError(f"tensors must be on the current device, cuda:{current}, got {t.device}")


def _rotary_heads(name, x, y, like=None):
    if x is None and y is None:
        return None, None
    if x is None or y is None:
        raise ValueError(f"{name} and {name}_out go together")
    for n, t in ((name, x), (name + "_out", y)):
        if t.dim() != 4 or t.shape[-1] < 2 or t.stride(-1) != 1:
            raise ValueError(f"{n} must be [batch, tokens, heads, elements] with adjacent elements")
    if y.shape != x.shape:
        raise ValueError(f"{name}_out must have shape {tuple(x.shape)}, got {tuple(y.shape)}")
    _want(name + "_out", y, x.dtype)
    if like is not None:
        _want(name, x, like.dtype)
        if x.shape[:2] != like.shape[:2] or x.shape[3] != like.shape[3]:
            raise ValueError(f"{name} must have the batch, tokens and elements of q, {tuple(like.shape)}, got {tuple(x.shape)}")
    s = _RotaryHeads(x.data_ptr(), y.data_ptr(), x.shape[2], (_i64 * 3)(*x.stride()[:3]), (_i64 * 3)(*y.stride()[:3]))
    return s, ctypes.byref(s)


def _rotary(where, q, k, freqs, positions, q_out, k_out, layout, scale, start, stream):
    if stream is None and _native is not None:
        status = getattr(_native, where)(q, k, freqs, positions, q_out, k_out, layout, scale, start)
        if status is not None:
            return _check(status, where)
    dt = _act_dtype("q", q)
    _want("freqs", freqs, torch.float64)
    if layout not in _LAYOUT:
        raise ValueError(f"layout must be one of {sorted(_LAYOUT)}, got {layout!r}")
    qs, q_ref = _rotary_heads("q", q, q_out)
    ks, k_ref = _rotary_heads("k", k, k_out, q)
    B, S, _, D = q.shape
    if not 1 <= freqs.numel() <= D // 2:
        raise ValueError(f"freqs must have 1 to {D // 2} elements, got {freqs.numel()}")
    if abs(start) > 2 ** 53:
        raise ValueError(f"start must lie within 2^53, got {start}")
    at = _RotaryPositions(None, 64, (_i64 * 2)(0, 0), start)
    if positions is not None:
        if positions.dtype not in (torch.int32, torch.int64):
            raise ValueError(f"positions must be int32 or int64, got {positions.dtype}")
        if positions.shape not in ((S,), (1, S), (B, S)):
            raise ValueError(f"positions must be [{S}] or [{B}, {S}], got {tuple(positions.shape)}")
        shared = positions.dim() == 1 or positions.shape[0] == 1
        at = _RotaryPositions(positions.data_ptr(), 8 * positions.element_size(),
                              (_i64 * 2)(0 if shared else positions.stride(0), positions.stride(-1)), start)
    _same_device(q, k, freqs, positions, q_out, k_out)
    f = _ptr(freqs)
    _check(getattr(load(), where)(q_ref, k_ref, f, ctypes.byref(at), B, S, D, 2 * freqs.numel(), _LAYOUT[layout], scale, dt,
                                  _stream(stream)), where)


def tempo_rotary_fwd(q, k, freqs, positions, q_out, k_out, layout="half", scale=1.0, start=0, stream=None):
    """Rotary positions of q and k [batch, tokens, heads, elements], any strides over the first three dimensions; k and k_out
    may be None, q_out may be q and k_out k.  freqs: float64, for the first 2 freqs.numel() elements of a head.  positions:
    [tokens] or [batch, tokens], int32 or int64, or None for 0, 1, ...; start is added to them."""
    _rotary("tempo_rotary_fwd", q, k, freqs, positions, q_out, k_out, layout, scale, start, stream)


def tempo_rotary_bwd(dq, dk, freqs, positions, dq_out, dk_out, layout="half", scale=1.0, start=0, stream=None):
    """The gradients of tempo_rotary_fwd's q and k from those of its outputs; arguments as there."""
    _rotary("tempo_rotary_bwd", dq, dk, freqs, positions, dq_out, dk_out, layout, scale, start, stream)


def tempo_glu_fwd_workspace_bytes(T: int, H: int, F: int, dtype) -> int:
    return load().tempo_glu_fwd_workspace_bytes(T, H, F, _DT[dtype])


def tempo_glu_bwd_workspace_bytes(T: int, H: int, F: int, dtype) -> int:
    return load().tempo_glu_bwd_workspace_bytes(T, H, F, _DT[dtype])


def _glu_sizes(x, w):
    if w.dim() != 2 or w.shape[0] % 2 != 0:
        raise ValueError(f"w must be [2 F, H], got {tuple(w.shape)}")
    F, H = w.shape[0] // 2, w.shape[1]
    if x.dim() < 1 or x.shape[-1] != H:
        raise ValueError(f"x must be [..., {H}], got {tuple(x.shape)}")
    return x.shape[:-1].numel(), H, F


def _workspace(workspace, nbytes, device, stream):
    """The caller's, or memory for the call that is given back to the stream it runs on."""
    if workspace is not None:
        return workspace
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _glu_kind(kind):
    if kind not in _GLU_KIND:
        raise ValueError(f"kind must be one of {sorted(_GLU_KIND)}, got {kind!r}")
    return _GLU_KIND[kind]


def tempo_glu_fwd(x, w, bias, gu, h, kind="silu", workspace=None, stream=None):
    """[g | u] = x w^T + bias into gu (None: not kept), act(g) u into h; w [2F, H]: the rows of the gate first.  kind: "silu",
    "gelu_erf" or "gelu_tanh".  workspace: tempo_glu_fwd_workspace_bytes() bytes, or None: allocated for the call."""
    if stream is None and _native is not None:
        status = _native.tempo_glu_fwd(x, w, bias, gu, h, kind, workspace)
        if status is not None:
            return _check(status, "tempo_glu_fwd")
    dt, act = _act_dtype("x", x), _glu_kind(kind)
    T, H, F = _glu_sizes(x, w)
    _want("w", w, x.dtype)
    _want("bias", bias, x.dtype, 2 * F)
    _want("gu", gu, x.dtype, T * 2 * F)
    _want("h", h, x.dtype, T * F)
    pointers = [_ptr(t) for t in (x, w, bias, gu, h)]
    _same_device(x, w, bias, gu, h, workspace)
    ws = _workspace(workspace, tempo_glu_fwd_workspace_bytes(T, H, F, x.dtype), x.device, stream)
    _check(load().tempo_glu_fwd(*pointers, _ptr(ws), ws.numel() * ws.element_size(), T, H, F, act, dt, _stream(stream)),
           "tempo_glu_fwd")


def tempo_glu_bwd(dh, gu, x, w, dgu, h, dx, dw, dbias, kind="silu", workspace=None, stream=None):
    """From the gradient of h and the kept gu: the gradients of x, w and the bias, and h once more, each of which may be None;
    dgu, a buffer like gu or gu itself, holds the gradient of gu afterwards."""
    if stream is None and _native is not None:
        status = _native.tempo_glu_bwd(dh, gu, x, w, dgu, h, dx, dw, dbias, kind, workspace)
        if status is not None:
            return _check(status, "tempo_glu_bwd")
    dt, act = _act_dtype("gu", gu), _glu_kind(kind)
    T, H, F = _glu_sizes(x, w)
    _want("x", x, gu.dtype)
    _want("w", w, gu.dtype)
    for name, t, n in (("gu", gu, T * 2 * F), ("dh", dh, T * F), ("dgu", dgu, T * 2 * F), ("h", h, T * F), ("dx", dx, T * H),
                       ("dw", dw, 2 * F * H), ("dbias", dbias, 2 * F)):
        _want(name, t, gu.dtype, n)
    pointers = [_ptr(t) for t in (dh, gu, x, w, dgu, h, dx, dw, dbias)]
    _same_device(dh, gu, x, w, dgu, h, dx, dw, dbias, workspace)
    ws = _workspace(workspace, tempo_glu_bwd_workspace_bytes(T, H, F, gu.dtype), gu.device, stream)
    _check(load().tempo_glu_bwd(*pointers, _ptr(ws), ws.numel() * ws.element_size(), T, H, F, act, dt, _stream(stream)),
           "tempo_glu_bwd")


def tempo_mask_bits_to_bytes(bits, bytes_, n, stream=None):
    _want("bits", bits, torch.int32, at_least=mask_words(n))
    _want("bytes", bytes_, torch.uint8, at_least=n)
    _check(load().tempo_mask_bits_to_bytes(_ptr(bits), _ptr(bytes_), n, _stream(stream)),
           "tempo_mask_bits_to_bytes")


def tempo_mask_bytes_to_bits(bytes_, bits, n, stream=None):
    _want("bits", bits, torch.int32, at_least=mask_words(n))
    _want("bytes", bytes_, torch.uint8, at_least=n)
    _check(load().tempo_mask_bytes_to_bits(_ptr(bytes_), _ptr(bits), n, _stream(stream)),
           "tempo_mask_bytes_to_bits")


def encoder_fwd(*args):
    """One native call for the forward of modules.TempoEncoderLayer (csrc/binding.cpp names the arguments): the offset it
    drew from and what its backward needs, or None if the call was not made."""
    r = _native.tempo_encoder_fwd(*args)
    if r is None:
        return None
    _check(r[0], "encoder_fwd")
    return r[1:]


def encoder_bwd(*args):
    """The same for the backward: the gradients of x and the parameters, or None if the call was not made."""
    r = _native.tempo_encoder_bwd(*args)
    if r is None:
        return None
    _check(r[0], "encoder_bwd")
    return r[1:]

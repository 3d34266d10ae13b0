"""Binding of include/pbsa_layer.h: what a layer runs around its block-sparse attention.  Same names, same library and the same
manner as pbsa.py: a description made once (make_rotary, make_cross), tensors passed through, no fallback.

Tensors are [n, heads, tokens, d] views with a contiguous last dimension, of any memory order.  Positions (int64), frequencies
(float64), norm weights and their gradients (float32), lengths (int32), masks (bytes) and lse (float32) are refused (ValueError) where
they are of another type, too small or not laid out as the description says.  rotary_frequencies makes the frequencies that the
rotation takes, scaled for long contexts or not.

The calls write into tensors that they are given, and autograd records none of them: what is to have a gradient goes through a
torch.autograd.Function whose backward makes the _bwd call (pbsa_rotate with inverse=True).
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import pbsa
from .pbsa import PbsaError  # noqa: F401  (what the calls raise)

PBSA_BF16, PBSA_FP16, PBSA_FP32 = 0, 1, 2
PBSA_ROTARY_MAX_D, PBSA_ROTARY_MAX_AXES, PBSA_LAYER_MAX_HEADS, PBSA_CROSS_MAX_NK = 256, 3, 4096, 1 << 24
_DTYPES = {torch.bfloat16: PBSA_BF16, torch.float16: PBSA_FP16, torch.float32: PBSA_FP32}
_Strides = ctypes.c_int64 * 3


class pbsa_rotary(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("n", ctypes.c_int32), ("T", ctypes.c_int32),
                ("Hq", ctypes.c_int32), ("Hk", ctypes.c_int32), ("d", ctypes.c_int32), ("rot", ctypes.c_int32),
                ("half", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("pairs", ctypes.c_int32 * PBSA_ROTARY_MAX_AXES),
                ("mscale", ctypes.c_float), ("eps", ctypes.c_float), ("pos_stride_b", ctypes.c_int64),
                ("q", _Strides), ("k", _Strides), ("qo", _Strides), ("ko", _Strides), ("dq", _Strides), ("dk", _Strides)]


class pbsa_cross(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("n", ctypes.c_int32), ("T", ctypes.c_int32),
                ("Nk", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hk", ctypes.c_int32), ("d", ctypes.c_int32),
                ("scale", ctypes.c_float), ("mask_stride_b", ctypes.c_int64),
                ("q", _Strides), ("k", _Strides), ("v", _Strides), ("o", _Strides),
                ("dO", _Strides), ("dq", _Strides), ("dk", _Strides), ("dv", _Strides)]


def _view(name, x, like=None):
    """Element strides {sequence, head, token} of a tensor; its shape and type are those of `like`."""
    if x.dim() != 4 or (x.shape[3] > 1 and x.stride(3) != 1):
        raise ValueError(f"{name}: [n, heads, tokens, d] with a contiguous last dimension, not {tuple(x.shape)} by {x.stride()}")
    if like is not None and (x.shape != like.shape or x.dtype != like.dtype or x.device != like.device):
        raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device}, {tuple(like.shape)} {like.dtype} on {like.device} wanted")
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name}: {x.dtype} is not a type that the library takes")
    return _Strides(*x.stride()[:3])


def make_rotary(q, k, qo, ko, sections=None, half=False, mscale=1.0, eps=1e-6, pos_stride_b=None, dq=None, dk=None) -> pbsa_rotary:
    """The description of a rotation, with or without the norm.  q, k: the inputs (k = ko = None: one tensor); qo, ko: what is
    written, or in a backward pass the gradients that come in; dq, dk: the gradients that go out.  sections: pairs of each axis
    (None: one axis, the whole head).  pos_stride_b: None where each sequence has positions of its own, 0 where they share them."""
    n, Hq, T, d = q.shape
    sections = (d // 2,) if sections is None else tuple(int(m) for m in sections)
    if not 1 <= len(sections) <= PBSA_ROTARY_MAX_AXES:
        raise ValueError(f"sections: 1 to {PBSA_ROTARY_MAX_AXES} axes, not {len(sections)}")
    if k is not None and (k.shape[0] != n or k.shape[2:] != q.shape[2:] or k.dtype != q.dtype):
        raise ValueError(f"k: {tuple(k.shape)} {k.dtype} beside q: {tuple(q.shape)} {q.dtype}")
    none = _Strides()
    view = lambda name, x, like: none if x is None else _view(name, x, like)  # noqa: E731
    qs = _view("q", q)
    return pbsa_rotary(ctypes.sizeof(pbsa_rotary), _DTYPES[q.dtype], n, T, Hq, 0 if k is None else k.shape[1], d, 2 * sum(sections),
                       int(half), len(sections), (ctypes.c_int32 * PBSA_ROTARY_MAX_AXES)(*sections), mscale, eps,
                       T * len(sections) if pos_stride_b is None else pos_stride_b, qs, view("k", k, None), view("qo", qo, q),
                       view("ko", ko, k), view("dq", dq, q), view("dk", dk, k))


def make_cross(q, k, v, o, scale=None, mask_stride_b=None, do=None, dq=None, dk=None, dv=None) -> pbsa_cross:
    """The description of a cross attention.  mask_stride_b: None where each sequence has a mask of its own, 0 for one mask."""
    n, Hq, T, d = q.shape
    Hk, Nk = k.shape[1], k.shape[2]
    if k.shape[0] != n or k.shape[3] != d or k.dtype != q.dtype:
        raise ValueError(f"k: {tuple(k.shape)} {k.dtype} beside q: {tuple(q.shape)} {q.dtype}")
    view = lambda name, x, like: _Strides() if x is None else _view(name, x, like)  # noqa: E731
    return pbsa_cross(ctypes.sizeof(pbsa_cross), _DTYPES[q.dtype] if q.dtype in _DTYPES else -1, n, T, Nk, Hq, Hk, d,
                      d ** -0.5 if scale is None else scale, Nk if mask_stride_b is None else mask_stride_b, _view("q", q), _view("k", k),
                      _view("v", v, k), _view("o", o, q), view("do", do, q), view("dq", dq, q), view("dk", dk, k), view("dv", dv, k))


def rotary_frequencies(sections, theta=1e4, scaling=None, factor=1.0, trained=None, slow=1.0, fast=32.0, device=None):
    """(freq, mscale): binary64 radians per step of every pair, axis after axis, and what the rotation multiplies by.

    Pair i of an axis of m pairs turns by theta^(-i / m) a step.  For contexts `factor` times as long as the `trained` ones:
      None      as trained
      linear    positions are squeezed: every frequency over the factor
      base      theta grows so that the slowest pair is squeezed by the factor and the fastest hardly at all
      parts     pairs of at least `fast` turns over the trained length stay, those of at most `slow` are squeezed, in between
                the two mix; the logits grow by 1 + 0.1 log factor for each of Q and K, as mscale
    """
    if scaling not in (None, "linear", "base", "parts"):
        raise ValueError(f"scaling: {scaling!r} is none of None, 'linear', 'base', 'parts'")
    if not factor >= 1:
        raise ValueError(f"factor: {factor} is less than 1")
    if scaling == "parts" and not (trained and fast > slow > 0):
        raise ValueError("scaling 'parts' goes by the trained length, and fast > slow > 0")
    out, mscale = [], 1.0
    for m in sections:
        i = torch.arange(m, dtype=torch.float64, device=device)
        base = theta * factor ** (m / (m - 1)) if scaling == "base" and m > 1 else theta
        f = base ** (-i / max(m, 1))
        if scaling == "linear":
            f = f / factor
        elif scaling == "parts":
            turns = trained * f / (2 * math.pi)
            keep = ((turns - slow) / (fast - slow)).clamp(0, 1)
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    if scaling == "parts":
        mscale = 1.0 + 0.1 * math.log(factor)
    return torch.cat(out), mscale


# Kinds of arguments as in pbsa.py; the description goes as the address of its bytes.
_SIGNATURES = {
    "pbsa_rotate": "wttttttiw",
    "pbsa_norm_rotate_fwd": "wttttttttw",
    "pbsa_norm_rotate_workspace_bytes": "wo",
    "pbsa_norm_rotate_bwd": "w" + 12 * "t" + "wzw",
    "pbsa_cross_workspace_bytes": "wo",
    "pbsa_cross_attention_fwd": "w" + 7 * "t" + "wzw",
    "pbsa_cross_bwd_workspace_bytes": "wo",
    "pbsa_cross_attention_bwd": "w" + 11 * "t" + "wzw",
}
EXPORTS = tuple(_SIGNATURES)


class _Functions(dict):
    """Address and argument kinds of each function, looked up (and the library loaded) on first use."""

    def __missing__(self, name):
        fn = _typed(name)
        self[name] = f = (ctypes.cast(fn, ctypes.c_void_p).value, _SIGNATURES[name].encode())
        return f


def _typed(name):
    types = dict(t=ctypes.c_void_p, w=ctypes.c_void_p, i=ctypes.c_int32, z=ctypes.c_size_t, o=ctypes.POINTER(ctypes.c_size_t))
    fn = getattr(pbsa.lib(), name)
    fn.restype, fn.argtypes = ctypes.c_int, [types[k] for k in _SIGNATURES[name]]
    return fn


_F = _Functions()


def _described(p, kind):
    if type(p) is not kind:
        raise TypeError(f"pbsa: a {kind.__name__} is wanted, not a {type(p).__name__}")
    return ctypes.addressof(p)


def _native():
    """The binding's native half takes the place of the two functions below."""
    global _rotary, _cross
    try:
        from . import _pbsa_host
    except ImportError as e:
        raise ImportError("the binding's native half is missing: build it with `python -m paper_2604_21221_amd.build`") from e
    _pbsa_host.setup_layer(pbsa_rotary, pbsa_cross)
    _rotary, _cross = _pbsa_host.rotary, _pbsa_host.cross


def _rotary(*args):
    """_rotary(description, pos, freq, wq, wk, dwq, dwk): the address of the description, with the arguments that it does not describe
    checked against it (csrc/pbsa_host.cpp)"""
    _native()
    return _rotary(*args)


def _cross(*args):
    """_cross(description, k_len, k_mask, lse), likewise"""
    _native()
    return _cross(*args)


def _call(name, *args):
    rc = pbsa._invoke(*_F[name], *args)
    if rc is NotImplemented:                 # anything but plain tensors and integers: ctypes and _ptr take it or refuse it
        rc = _typed(name)(*[pbsa._ptr(a) if k == "t" else a for k, a in zip(_SIGNATURES[name], args)])
    pbsa._check(rc)


def _size(name, p, kind):
    out = ctypes.c_size_t(0)
    pbsa._check(_typed(name)(_described(p, kind), ctypes.byref(out)))
    return out.value


def pbsa_rotate(p, Q, K, pos, freq, Qo, Ko, inverse=False, stream=None):
    _call("pbsa_rotate", _rotary(p, pos, freq, None, None, None, None), Q, K, pos, freq, Qo, Ko, int(inverse), pbsa._stream(stream))


def pbsa_norm_rotate_fwd(p, Q, K, wq, wk, pos, freq, Qo, Ko, stream=None):
    _call("pbsa_norm_rotate_fwd", _rotary(p, pos, freq, wq, wk, None, None), Q, K, wq, wk, pos, freq, Qo, Ko, pbsa._stream(stream))


def pbsa_norm_rotate_workspace_bytes(p: pbsa_rotary) -> int:
    return _size("pbsa_norm_rotate_workspace_bytes", p, pbsa_rotary)


def pbsa_norm_rotate_bwd(p, Q, K, wq, wk, pos, freq, dQo, dKo, dQ, dK, dwq, dwk, ws, stream=None):
    w, wb = pbsa._ws(ws)
    _call("pbsa_norm_rotate_bwd", _rotary(p, pos, freq, wq, wk, dwq, dwk), Q, K, wq, wk, pos, freq, dQo, dKo, dQ, dK, dwq, dwk, w, wb,
          pbsa._stream(stream))


def pbsa_cross_workspace_bytes(p: pbsa_cross) -> int:
    return _size("pbsa_cross_workspace_bytes", p, pbsa_cross)


def pbsa_cross_attention_fwd(p, Q, K, V, k_len, k_mask, O, lse=None, ws=None, stream=None):
    w, wb = pbsa._ws(ws)
    _call("pbsa_cross_attention_fwd", _cross(p, k_len, k_mask, lse), Q, K, V, k_len, k_mask, O, lse, w, wb, pbsa._stream(stream))


def pbsa_cross_bwd_workspace_bytes(p: pbsa_cross) -> int:
    return _size("pbsa_cross_bwd_workspace_bytes", p, pbsa_cross)


def pbsa_cross_attention_bwd(p, Q, K, V, k_len, k_mask, O, dO, lse, dQ, dK, dV, ws, stream=None):
    w, wb = pbsa._ws(ws)
    _call("pbsa_cross_attention_bwd", _cross(p, k_len, k_mask, lse), Q, K, V, k_len, k_mask, O, dO, lse, dQ, dK, dV, w, wb,
          pbsa._stream(stream))

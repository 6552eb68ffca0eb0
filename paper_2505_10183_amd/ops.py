"""Binding of the operators of kt_ops.h: shapes and strides of torch tensors to the sizes and addresses that the C calls take.

All results go into tensors that the caller gives.  The calls are asynchronous on `stream` (None: torch's current one; a torch
stream or a raw handle).  Plain tensors go to the library through _kt_marshal.so, everything else, and
everything where that is missing, through ctypes.  A `workspace` is a tensor of at least as many bytes as the library asks for, on the GPU; None takes one from torch's
allocator for the call, tied to that stream.  There is no fallback: tensors that are not on the current GPU are refused.

The calls stand outside autograd, as those of binding.py do: inputs that require a gradient are taken as they are, outputs carry no
graph, and version counters do not move; the backward pass is the caller's own sequence of calls.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import binding
from .binding import KT_BF16, KT_F32, _check, _stream

_TYPES = {torch.float32: KT_F32, torch.bfloat16: KT_BF16}
_lib = None         # the library that the prototypes below were given to

ACT8_GROUP = 32


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class _Attention(ctypes.Structure):
    _fields_ = [("dt", ctypes.c_int), ("batch", ctypes.c_int64), ("nq", ctypes.c_int64), ("nk", ctypes.c_int64),
                ("heads", ctypes.c_int64), ("kv_heads", ctypes.c_int64), ("dim", ctypes.c_int64), ("scale", ctypes.c_float),
                ("causal", ctypes.c_int), ("k_lens", ctypes.c_void_p)]


def _library() -> ctypes.CDLL:
    global _lib
    L = binding.lib()
    if L is not _lib:
        i32, i64, vp, f32 = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
        L.kt_layernorm_fwd.argtypes = [i32, i32, i64, i64, vp, i64, vp, vp, f32, vp, i64, vp, vp, vp, vp, vp]
        L.kt_layernorm_bwd_workspace.argtypes = [i64, i64]
        L.kt_layernorm_bwd_workspace.restype = i64
        L.kt_layernorm_bwd.argtypes = [i32, i32, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, i64, vp]
        L.kt_act8_save.argtypes = [i32, i64, i64, vp, i64, vp, vp, vp]
        L.kt_act8_restore.argtypes = [i32, i64, i64, vp, vp, vp, i64, vp]
        L.kt_act8_weight_grad_workspace.argtypes = [i32, i64, i64, i64]
        L.kt_act8_weight_grad_workspace.restype = i64
        L.kt_act8_weight_grad.argtypes = [i32, i32, i64, i64, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp]
        hp, ap = ctypes.POINTER(_Heads), ctypes.POINTER(_Attention)
        L.kt_attention_fwd.argtypes = [ap, hp, hp, hp, hp, vp, vp]
        L.kt_attention_bwd_workspace.argtypes = [ap]
        L.kt_attention_bwd_workspace.restype = i64
        L.kt_attention_bwd.argtypes = [ap, hp, hp, hp, hp, hp, vp, hp, hp, hp, vp, i64, vp]
        for n in ("kt_layernorm_fwd", "kt_layernorm_bwd", "kt_act8_save", "kt_act8_restore", "kt_act8_weight_grad",
                  "kt_attention_fwd", "kt_attention_bwd"):
            getattr(L, n).restype = i32
        _lib = L
    return L


_plain_of = {}      # the native calls of each loaded library
_ENTRIES = ("kt_layernorm_fwd", "kt_layernorm_bwd_workspace", "kt_layernorm_bwd", "kt_act8_save", "kt_act8_restore",
            "kt_act8_weight_grad_workspace", "kt_act8_weight_grad", "kt_attention_fwd", "kt_attention_bwd_workspace", "kt_attention_bwd")


def _plainly(name: str, *args) -> bool:
    """Make the call natively; False where an argument is of a form that is left to the code below."""
    L = _library()
    calls = _plain_of.get(L)
    if calls is None:
        m = binding._marshal_module()
        calls = _plain_of[L] = m.Ops(*[ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in _ENTRIES]) if m else False
    if not calls:
        return False
    status = getattr(calls, name)(*args)
    if status:
        _check(status, L)
    return status is not None


def _type(x, what: str) -> int:
    t = _TYPES.get(x.dtype)
    if t is None:
        raise ValueError("%s: float32 or bfloat16 is needed, got %s" % (what, x.dtype))
    return t


def _on_gpu(x, what: str):
    if not x.is_cuda or x.get_device() != torch.cuda.current_device():
        raise ValueError("%s: a tensor on the current GPU is needed, got one on %s" % (what, x.device))


def _matrix(x, what: str) -> Tuple[int, int, int, int]:
    """(address, rows, cols, ld) of a tensor whose last dimension is that of the columns."""
    _on_gpu(x, what)
    if x.dim() == 2:
        rows, cols = x.shape
        ld, one = x.stride()
        if cols > 1 and one != 1:
            raise ValueError("%s: adjacent columns are needed, got stride %d" % (what, one))
        return x.data_ptr(), rows, cols, ld if rows > 1 else cols
    if x.dim() < 1:
        raise ValueError("%s: a matrix is needed" % what)
    try:
        return _matrix(x.view(-1, x.shape[-1]), what)
    except RuntimeError as e:
        raise ValueError("%s: its leading dimensions cannot be taken as one (%s)" % (what, e)) from None


def _vector(x, n: int, dtype, what: str) -> int:
    """Address of n adjacent elements; 0 for None."""
    if x is None:
        return 0
    _on_gpu(x, what)
    if x.dtype != dtype or x.numel() != n or not x.is_contiguous():
        raise ValueError("%s: %d adjacent elements of %s are needed, got %s %s" % (what, n, dtype, tuple(x.shape), x.dtype))
    return x.data_ptr()


def _like(x, rows: int, cols: int, dtype, what: str) -> Tuple[int, int]:
    """(address, ld) of a matrix of this shape and type."""
    p, r, c, ld = _matrix(x, what)
    if (r, c) != (rows, cols) or x.dtype != dtype:
        raise ValueError("%s: [%d, %d] of %s is needed, got %s %s" % (what, rows, cols, dtype, tuple(x.shape), x.dtype))
    return p, ld


def kt_act8_shapes(rows: int, cols: int) -> Tuple[Tuple[int, int], Tuple[int, int]]:
    """Shapes of the two parts of a checkpoint of [rows, cols]: q (int8) and e (uint8)."""
    groups = (cols + ACT8_GROUP - 1) // ACT8_GROUP
    return (rows, groups * ACT8_GROUP), (rows, groups)


def _act8(q, e, rows: int, cols: int, what: str) -> Tuple[int, int]:
    qs, es = kt_act8_shapes(rows, cols)
    return _vector(q, qs[0] * qs[1], torch.int8, what + " (q)"), _vector(e, es[0] * es[1], torch.uint8, what + " (e)")


def _workspace(given, need: int, stream, device) -> Tuple[int, int, Optional[torch.Tensor]]:
    """(address, bytes, tensor to hold until the call is made)."""
    if given is not None:
        _on_gpu(given, "workspace")
        if not given.is_contiguous():
            raise ValueError("workspace: adjacent elements are needed")
        return given.data_ptr(), given.numel() * given.element_size(), given
    if need == 0:
        return 0, 0, None
    if stream is None:
        t = torch.empty(need, dtype=torch.uint8, device=device)
    else:           # memory that torch gives to later work of that stream only
        s = torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream
        with torch.cuda.stream(s):
            t = torch.empty(need, dtype=torch.uint8, device=device)
    return t.data_ptr(), need, t


def kt_layernorm_fwd(x, gamma, beta, eps: float, y, mean=None, rstd=None, y8=None, stream=None):
    """y = (x - mean) * rstd * gamma + beta over the last dimension; beta, and mean with rstd (float32, a value a row), may be
    None.  y8 = (q, e): the 8-bit checkpoint of y, written in the same pass.  y may be x itself."""
    if _plainly("layernorm_fwd", x, gamma, beta, eps, y, mean, rstd, y8, stream):
        return
    L = _library()
    p, rows, cols, ld = _matrix(x, "x")
    py, ldy = _like(y, rows, cols, x.dtype, "y")
    q, e = (0, 0) if y8 is None else _act8(y8[0], y8[1], rows, cols, "y8")
    status = L.kt_layernorm_fwd(_type(x, "x"), _type(gamma, "gamma"), rows, cols, p, ld, _vector(gamma, cols, gamma.dtype, "gamma"),
                                _vector(beta, cols, gamma.dtype, "beta"), eps, py, ldy, _vector(mean, rows, torch.float32, "mean"),
                                _vector(rstd, rows, torch.float32, "rstd"), q, e, _stream(stream))
    if status:
        _check(status, L)


def kt_layernorm_bwd_workspace(rows: int, cols: int) -> int:
    return _library().kt_layernorm_bwd_workspace(rows, cols)


def kt_layernorm_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta=None, workspace=None, stream=None):
    """Gradients of input, weight and bias.  x: the input, or (q, e) of its 8-bit checkpoint.  dgamma and dbeta have gamma's type and
    may lie in a bucket; dx may be dy or x itself."""
    if _plainly("layernorm_bwd", dy, x, gamma, mean, rstd, dx, dgamma, dbeta, workspace, stream):
        return
    L = _library()
    p, rows, cols, ld = _matrix(dy, "dy")
    px = ldx = q = e = 0
    if isinstance(x, (tuple, list)):
        q, e = _act8(x[0], x[1], rows, cols, "x")
    else:
        px, ldx = _like(x, rows, cols, dy.dtype, "x")
    pdx, lddx = _like(dx, rows, cols, dy.dtype, "dx")
    need = L.kt_layernorm_bwd_workspace(rows, cols)
    ws, size, held = _workspace(workspace, need, stream, dy.device)
    status = L.kt_layernorm_bwd(_type(dy, "dy"), _type(gamma, "gamma"), rows, cols, p, ld, px, ldx, q, e,
                                _vector(gamma, cols, gamma.dtype, "gamma"), _vector(mean, rows, torch.float32, "mean"),
                                _vector(rstd, rows, torch.float32, "rstd"), pdx, lddx,
                                _vector(dgamma, cols, gamma.dtype, "dgamma"), _vector(dbeta, cols, gamma.dtype, "dbeta"), ws, size,
                                _stream(stream))
    if status:
        _check(status, L)


def kt_act8_save(x, q, e, stream=None):
    """The 8-bit checkpoint (q, e) of x; shapes as kt_act8_shapes says, over the last dimension."""
    if _plainly("act8_save", x, q, e, stream):
        return
    L = _library()
    p, rows, cols, ld = _matrix(x, "x")
    pq, pe = _act8(q, e, rows, cols, "checkpoint")
    status = L.kt_act8_save(_type(x, "x"), rows, cols, p, ld, pq, pe, _stream(stream))
    if status:
        _check(status, L)


def kt_act8_restore(q, e, y, stream=None):
    """What the checkpoint (q, e) stands for, into y."""
    if _plainly("act8_restore", q, e, y, stream):
        return
    L = _library()
    p, rows, cols, ld = _matrix(y, "y")
    pq, pe = _act8(q, e, rows, cols, "checkpoint")
    status = L.kt_act8_restore(_type(y, "y"), rows, cols, pq, pe, p, ld, _stream(stream))
    if status:
        _check(status, L)


def kt_act8_weight_grad_workspace(dtype, tokens: int, out: int, inn: int) -> int:
    return _library().kt_act8_weight_grad_workspace(_TYPES[dtype], tokens, out, inn)


def kt_act8_weight_grad(dy, q, e, dw, workspace=None, stream=None):
    """dw [out, in] = dy^T x8: the weight gradient of a linear layer from dy [tokens, out] and the 8-bit checkpoint of its
    input [tokens, in].  dw may be float32 or bfloat16 whatever dy is, and may lie in a bucket."""
    if _plainly("act8_weight_grad", dy, q, e, dw, workspace, stream):
        return
    L = _library()
    p, tokens, out, ld = _matrix(dy, "dy")
    pw, rows, inn, ldw = _matrix(dw, "dw")
    if rows != out:
        raise ValueError("dw: %d rows are needed, got %d" % (out, rows))
    t = _type(dy, "dy")
    pq, pe = _act8(q, e, tokens, inn, "checkpoint")
    ws, size, held = _workspace(workspace, L.kt_act8_weight_grad_workspace(t, tokens, out, inn), stream, dy.device)
    status = L.kt_act8_weight_grad(t, _type(dw, "dw"), tokens, out, inn, p, ld, pq, pe, pw, ldw, ws, size, _stream(stream))
    if status:
        _check(status, L)


def _heads(x, shape, dtype, what: str) -> _Heads:
    _on_gpu(x, what)
    if x.dtype != dtype or x.shape != shape:
        raise ValueError("%s: %s of %s is needed, got %s of %s" % (what, list(shape), dtype, list(x.shape), x.dtype))
    b, t, h, d = x.stride()
    if d != 1 and shape[3] > 1:
        raise ValueError("%s: adjacent elements of a head are needed, got stride %d" % (what, d))
    return _Heads(x.data_ptr(), b, t, h)


def _attention(q, k, causal, scale, k_lens) -> Tuple[_Attention, tuple, tuple]:
    """The sizes, and the shapes of the query and the key side."""
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k: [batch, tokens, heads, dim] is needed")
    batch, nq, heads, dim = q.shape
    qs, ks = q.shape, torch.Size((batch, k.shape[1], k.shape[2], dim))
    lens = _vector(k_lens, batch, torch.int32, "k_lens")
    return _Attention(_type(q, "q"), batch, nq, k.shape[1], heads, k.shape[2], dim, dim ** -0.5 if scale is None else scale,
                      1 if causal else 0, lens), qs, ks


def kt_attention_fwd(q, k, v, o, lse=None, causal: bool = False, scale: Optional[float] = None, k_lens=None, stream=None):
    """o = softmax(scale q k^T) v; all tensors [batch, tokens, heads, dim] with adjacent elements of a head and any strides else,
    k and v with a divisor of q's heads.  lse [batch, heads, queries] (float32): what the backward pass needs.  scale: None =
    1 / sqrt(dim).  causal: the last query sees the last key.  k_lens [batch] (int32): keys of each sequence, on the GPU."""
    if _plainly("attention_fwd", q, k, v, o, lse, causal, scale, k_lens, stream):
        return
    L = _library()
    a, qs, ks = _attention(q, k, causal, scale, k_lens)
    t = q.dtype
    status = L.kt_attention_fwd(a, _heads(q, qs, t, "q"), _heads(k, ks, t, "k"), _heads(v, ks, t, "v"), _heads(o, qs, t, "o"),
                                _vector(lse, qs[0] * qs[1] * qs[2], torch.float32, "lse"), _stream(stream))
    if status:
        _check(status, L)


def kt_attention_bwd_workspace(q, k) -> int:
    a, _, _ = _attention(q, k, False, None, None)
    return _library().kt_attention_bwd_workspace(a)


def kt_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, causal: bool = False, scale: Optional[float] = None, k_lens=None,
                     workspace=None, stream=None):
    """Gradients of q, k and v from that of o; o and lse are what kt_attention_fwd left for the same arguments.  dq, dk and dv may
    be views of one buffer, as q, k and v may."""
    if _plainly("attention_bwd", do, q, k, v, o, lse, dq, dk, dv, causal, scale, k_lens, workspace, stream):
        return
    L = _library()
    a, qs, ks = _attention(q, k, causal, scale, k_lens)
    t = q.dtype
    ws, size, held = _workspace(workspace, L.kt_attention_bwd_workspace(a), stream, q.device)
    status = L.kt_attention_bwd(a, _heads(do, qs, t, "do"), _heads(q, qs, t, "q"), _heads(k, ks, t, "k"), _heads(v, ks, t, "v"),
                                _heads(o, qs, t, "o"), _vector(lse, qs[0] * qs[1] * qs[2], torch.float32, "lse"),
                                _heads(dq, qs, t, "dq"), _heads(dk, ks, t, "dk"), _heads(dv, ks, t, "dv"), ws, size, _stream(stream))
    if status:
        _check(status, L)

"""ctypes binding of include/daf_attention.h: the operators of a transformer block's attention half.  Same names as the C ABI; Python checks and
marshals arguments only.  Heads are tensors [tokens, heads, head_dim] whose last dimension is contiguous: views of a projection's result go as
they are."""
import ctypes
import math
from typing import Optional

import torch

from .binding import _DTYPE_ID, _ELEM_DTYPES, DafError, _fast, _fast_calls, _stream_handle, load_library
from .block import _GATED_DTYPES, _Checks, _pointer

_declared = None
_EINVAL = -1                            # DAF_EINVAL


class _Heads(ctypes.Structure):
    _fields_ = [("at", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _HeadRotation(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("positions", ctypes.c_int64), ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("pairing", ctypes.c_int32),
                ("norm", ctypes.c_int32), ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("cos", ctypes.c_void_p),
                ("sin", ctypes.c_void_p), ("position", ctypes.c_void_p)]


class _WindowAttention(ctypes.Structure):
    _fields_ = [("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64), ("sequences", ctypes.c_int64), ("window", ctypes.c_int64), ("sinks", ctypes.c_int64),
                ("q_heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
                ("q_starts", ctypes.c_void_p), ("k_starts", ctypes.c_void_p), ("k_lengths", ctypes.c_void_p)]


def _library():
    """libdaf.so with the argument types of these calls."""
    global _declared
    if _declared is not None:
        return _declared
    L, c = load_library(), ctypes
    vp, i64, i32 = c.c_void_p, c.c_int64, c.c_int32
    for name, result, arguments in (
            ("daf_head_rotation", c.c_int, [vp] * 8 + [i64, vp]),
            ("daf_head_rotation_backward_workspace_bytes", i64, [i64, i32, i32, i32]),
            ("daf_head_rotation_backward", c.c_int, [vp] * 11),
            ("daf_window_attention", c.c_int, [vp] * 7),
            ("daf_window_attention_backward_workspace_bytes", i64, [i64, i32, i32, i32, i64, i64, i64]),
            ("daf_window_attention_backward", c.c_int, [vp] * 12),
            ("daf_window_attention_step_workspace_bytes", i64, [i64, i32, i32, i32, i64, i64, i64]),
            ("daf_window_attention_step", c.c_int, [vp] * 7)):
        getattr(L, name).restype = result
        getattr(L, name).argtypes = arguments
    if _fast_calls is not None:
        names = ("daf_head_rotation", "daf_head_rotation_backward", "daf_head_rotation_backward_workspace_bytes", "daf_window_attention",
                 "daf_window_attention_backward", "daf_window_attention_backward_workspace_bytes", "daf_window_attention_step",
                 "daf_window_attention_step_workspace_bytes")
        _fast_calls.bind_attention({name: c.cast(getattr(L, name), vp).value for name in names})
    _declared = L
    return L


class _HeadChecks(_Checks):
    """The tensors of one call; heads need not be contiguous.  All are on the current device, on which the call works."""

    def heads(self, name: str, t, dtype, rows=None, heads=None, dim=None) -> None:
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name}: expected a torch.Tensor, got {type(t).__name__}")
        if t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
            raise ValueError(f"{name}: dtype {t.dtype}, expected {dtype}")
        if t.dim() != 3 or (t.shape[0], t.shape[1], t.shape[2]) != (t.shape[0] if rows is None else rows, t.shape[1] if heads is None else heads,
                                                                   t.shape[2] if dim is None else dim):
            wanted = ", ".join("any" if n is None else str(n) for n in (rows, heads, dim))
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected ({wanted})")
        if t.shape[1] < 1 or t.shape[2] < 1:
            raise ValueError(f"{name}: no heads, or heads of no elements")
        step = 16 // t.element_size()
        for n, stride in ((t.shape[0], t.stride(0)), (t.shape[1], t.stride(1))):
            if t.shape[0] > 0 and n > 1 and (stride % step != 0 or stride < t.shape[2]):
                raise ValueError(f"{name}: strides {t.stride()}; those of tokens and heads must be multiples of {step} and at least {t.shape[2]}")
        if t.shape[0] > 0 and t.stride(2) != 1:
            raise ValueError(f"{name}: strides {t.stride()}; the last dimension must be contiguous")
        self.seen.append((name, t))

    def on_device(self) -> None:
        super().on_device()
        if self.seen[0][1].get_device() != torch.cuda.current_device():
            raise ValueError(f"{self.seen[0][0]}: on {self.seen[0][1].device}, the current device is cuda:{torch.cuda.current_device()}")


def _heads(t):
    return None if t is None else _Heads(t.data_ptr(), t.stride(0), t.stride(1))


def _int32(n: int) -> int:
    return min(n, 0x7FFFFFFF)                                             # (more is refused)


def _at(struct):
    return None if struct is None else ctypes.addressof(struct)


# ---- norms of heads and rotation by position ----
PAIRINGS = {"halves": 0, "pairs": 1}


def _rotation_parameters(chk, q, k, position, cos, sin, q_weight, k_weight, norm, eps, pairing):
    """Queries and keys (or their gradients, of the same sizes) and what goes with them, checked, and the struct."""
    if pairing not in PAIRINGS:
        raise ValueError(f"pairing: {pairing!r} not in {tuple(PAIRINGS)}")
    chk.heads("q", q, _ELEM_DTYPES)
    tokens, heads, dim = q.shape
    chk.heads("k", k, q.dtype, rows=tokens, dim=dim)
    chk.like("position", position, torch.int32, (tokens,))
    chk.tensor("cos", cos, torch.float32, 0)
    if cos.dim() != 2:
        raise ValueError(f"cos: shape {tuple(cos.shape)}, expected (positions, rotary_dim / 2)")
    chk.like("sin", sin, torch.float32, cos.shape)
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        chk.optional(name, w, q.dtype, (dim,))
        if w is not None and not norm:
            raise ValueError(f"{name}: belongs to norm=True")
    return _HeadRotation(tokens, cos.shape[0], _int32(heads), _int32(k.shape[1]), _int32(dim), _int32(2 * cos.shape[1]), _DTYPE_ID[q.dtype], PAIRINGS[pairing], int(bool(norm)), eps,
                         _pointer(q_weight), _pointer(k_weight), cos.data_ptr(), sin.data_ptr(), position.data_ptr())


def daf_head_rotation(q: torch.Tensor, k: torch.Tensor, position: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor, out_q: torch.Tensor,
                      out_k: torch.Tensor, *, q_weight=None, k_weight=None, norm: bool = True, eps: float = 1e-6, pairing: str = "halves",
                      v: Optional[torch.Tensor] = None, out_v: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None, stream=None) -> None:
    """Every head of q and k [tokens, heads, head_dim] normalized (norm) and rotated by its token's row of cos and sin [positions, rotary_dim / 2].  With
    `rows` (int32, one for each token) keys go to those rows of out_k [rows of a cache, heads, head_dim], and v's heads to those of out_v."""
    rc = _fast.head_rotation(q, k, position, cos, sin, out_q, out_k, q_weight, k_weight, norm, eps, PAIRINGS.get(pairing), v, out_v, rows, stream)
    if rc is None:
        rc = _general_head_rotation(q, k, position, cos, sin, out_q, out_k, q_weight, k_weight, norm, eps, pairing, v, out_v, rows, stream)
    if rc != 0:
        raise DafError(rc, "daf_head_rotation")


def _general_head_rotation(q, k, position, cos, sin, out_q, out_k, q_weight, k_weight, norm, eps, pairing, v, out_v, rows, stream):
    chk = _HeadChecks()
    p = _rotation_parameters(chk, q, k, position, cos, sin, q_weight, k_weight, norm, eps, pairing)
    tokens, dim = q.shape[0], q.shape[2]
    chk.heads("out_q", out_q, q.dtype, *q.shape)
    chk.optional("rows", rows, torch.int32, (tokens,))
    chk.heads("out_k", out_k, q.dtype, rows=tokens if rows is None else None, heads=k.shape[1], dim=dim)
    if (v is None) != (out_v is None):
        raise ValueError("v and out_v: both or neither")
    if v is not None:
        chk.heads("v", v, q.dtype, *k.shape)
        chk.heads("out_v", out_v, q.dtype, *out_k.shape)
    chk.on_device()
    given = [_heads(t) for t in (q, k, v, out_q, out_k, out_v)]
    return _library().daf_head_rotation(_at(p), *(_at(h) for h in given), _pointer(rows), out_k.shape[0], _stream_handle(stream))


def daf_head_rotation_backward_workspace_bytes(tokens: int, q_heads: int, kv_heads: int, head_dim: int) -> int:
    return int(_library().daf_head_rotation_backward_workspace_bytes(tokens, q_heads, kv_heads, head_dim))


def daf_head_rotation_backward(q: Optional[torch.Tensor], k: Optional[torch.Tensor], position: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor,
                               grad_q: torch.Tensor, grad_k: torch.Tensor, out_grad_q: torch.Tensor, out_grad_k: torch.Tensor,
                               workspace: Optional[torch.Tensor] = None, *, q_weight=None, k_weight=None, norm: bool = True, eps: float = 1e-6,
                               pairing: str = "halves", out_grad_q_weight=None, out_grad_k_weight=None, stream=None) -> None:
    """Backward of daf_head_rotation, from the gradients of its out_q and out_k.  The weights' gradients are float32; those that are None are not
    computed.  Without `norm`, q and k are not read and may be None."""
    rc = _fast.head_rotation_backward(q, k, position, cos, sin, grad_q, grad_k, out_grad_q, out_grad_k, workspace, q_weight, k_weight, norm, eps,
                                      PAIRINGS.get(pairing), out_grad_q_weight, out_grad_k_weight, stream)
    if rc is None:
        rc = _general_head_rotation_backward(q, k, position, cos, sin, grad_q, grad_k, out_grad_q, out_grad_k, workspace, q_weight, k_weight, norm, eps,
                                             pairing, out_grad_q_weight, out_grad_k_weight, stream)
    if rc != 0:
        raise DafError(rc, "daf_head_rotation_backward")


def _general_head_rotation_backward(q, k, position, cos, sin, grad_q, grad_k, out_grad_q, out_grad_k, workspace, q_weight, k_weight, norm, eps, pairing,
                                    out_grad_q_weight, out_grad_k_weight, stream):
    chk = _HeadChecks()
    p = _rotation_parameters(chk, grad_q, grad_k, position, cos, sin, q_weight, k_weight, norm, eps, pairing)
    if norm:
        chk.heads("q", q, grad_q.dtype, *grad_q.shape)
        chk.heads("k", k, grad_q.dtype, *grad_k.shape)
    else:
        q = k = None
    chk.heads("out_grad_q", out_grad_q, grad_q.dtype, *grad_q.shape)
    chk.heads("out_grad_k", out_grad_k, grad_q.dtype, *grad_k.shape)
    for name, t in (("out_grad_q_weight", out_grad_q_weight), ("out_grad_k_weight", out_grad_k_weight)):
        chk.optional(name, t, torch.float32, (grad_q.shape[2],))
        if t is not None and not norm:
            raise ValueError(f"{name}: belongs to norm=True")
    if out_grad_q_weight is not None or out_grad_k_weight is not None:
        chk.workspace(workspace, daf_head_rotation_backward_workspace_bytes(p.tokens, p.q_heads, p.kv_heads, p.head_dim))
    chk.on_device()
    given = [_heads(t) for t in (q, k, grad_q, grad_k, out_grad_q, out_grad_k)]
    return _library().daf_head_rotation_backward(_at(p), *(_at(h) for h in given), _pointer(out_grad_q_weight), _pointer(out_grad_k_weight),
                                                 _pointer(workspace), _stream_handle(stream))


# ---- attention with a window and sinks ----
def _attention_parameters(chk, q, k, v, window, sinks, scale, q_starts, k_starts, k_lengths, sequences):
    chk.heads("q", q, _GATED_DTYPES)
    chk.heads("k", k, q.dtype, dim=q.shape[2])
    chk.heads("v", v, q.dtype, *k.shape)
    if q.shape[1] % k.shape[1] != 0:
        raise ValueError(f"{q.shape[1]} heads of queries for {k.shape[1]} of keys")
    if q_starts is not None:
        chk.tensor("q_starts", q_starts, torch.int32, 2)
        if q_starts.dim() != 1:
            raise ValueError(f"q_starts: shape {tuple(q_starts.shape)}, expected (sequences + 1,)")
        sequences = q_starts.numel() - 1
    for name, n in (("window", window), ("sinks", sinks)):
        if not isinstance(n, int) or abs(n) >= 1 << 63:
            raise ValueError(f"{name}: {n!r}, expected an int below 2^63")
    if (k_starts is None) != (k_lengths is None):
        raise ValueError("k_starts and k_lengths: both or neither")
    chk.optional("k_starts", k_starts, torch.int32, (sequences,))
    chk.optional("k_lengths", k_lengths, torch.int32, (sequences,))
    if k_starts is None and k.shape[0] != q.shape[0]:
        raise ValueError(f"k: {k.shape[0]} rows for {q.shape[0]} queries, without k_starts and k_lengths")
    return _WindowAttention(q.shape[0], k.shape[0], sequences, window, sinks, _int32(q.shape[1]), _int32(k.shape[1]), _int32(q.shape[2]),
                            _DTYPE_ID[q.dtype], 1 / math.sqrt(q.shape[2]) if scale is None else scale, _pointer(q_starts), _pointer(k_starts), _pointer(k_lengths))


def daf_window_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, out_lse: Optional[torch.Tensor] = None, *, window: int = 0,
                         sinks: int = 0, scale: Optional[float] = None, q_starts: Optional[torch.Tensor] = None,
                         k_starts: Optional[torch.Tensor] = None, k_lengths: Optional[torch.Tensor] = None, stream=None) -> None:
    """Causal attention of q [rows, heads, head_dim] within each sequence: a query sees the `window` last keys up to its own (0: all) and the first `sinks`.
    q_starts (int32, sequences + 1): where sequences begin and the last one ends; None: one sequence.  k_starts, k_lengths (int32): the rows of k and v that are
    each sequence's keys, the last of them its last query's; None: the queries' rows.  out_lse: float32 [heads, rows], for the backward pass."""
    rc = _fast.window_attention(q, k, v, out, out_lse, window, sinks, scale, q_starts, k_starts, k_lengths, stream)
    if rc is None:
        rc = _general_window_attention(q, k, v, out, out_lse, window, sinks, scale, q_starts, k_starts, k_lengths, stream)
    if rc != 0:
        raise DafError(rc, "daf_window_attention")


def _general_window_attention(q, k, v, out, out_lse, window, sinks, scale, q_starts, k_starts, k_lengths, stream):
    chk = _HeadChecks()
    p = _attention_parameters(chk, q, k, v, window, sinks, scale, q_starts, k_starts, k_lengths, 1)
    chk.heads("out", out, q.dtype, *q.shape)
    chk.optional("out_lse", out_lse, torch.float32, (q.shape[1], q.shape[0]))
    chk.on_device()
    given = [_heads(t) for t in (q, k, v, out)]
    return _library().daf_window_attention(_at(p), *(_at(h) for h in given), _pointer(out_lse), _stream_handle(stream))


def daf_window_attention_backward_workspace_bytes(rows: int, q_heads: int, kv_heads: int, head_dim: int, sequences: int = 1, window: int = 0,
                                                  sinks: int = 0) -> int:
    """Enough for fewer rows and sequences too."""
    return int(_library().daf_window_attention_backward_workspace_bytes(rows, q_heads, kv_heads, head_dim, sequences, window, sinks))


def daf_window_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, grad_out: torch.Tensor,
                                  out_grad_q: torch.Tensor, out_grad_k: torch.Tensor, out_grad_v: torch.Tensor, workspace: torch.Tensor, *, window: int = 0,
                                  sinks: int = 0, scale: Optional[float] = None, q_starts: Optional[torch.Tensor] = None, stream=None) -> None:
    """Backward of daf_window_attention where the keys are the queries' rows: `out` and `lse` are its out and out_lse."""
    rc = _fast.window_attention_backward(q, k, v, out, lse, grad_out, out_grad_q, out_grad_k, out_grad_v, workspace, window, sinks, scale, q_starts, stream)
    if rc is None:
        rc = _general_window_attention_backward(q, k, v, out, lse, grad_out, out_grad_q, out_grad_k, out_grad_v, workspace, window, sinks, scale, q_starts, stream)
    if rc != 0:
        raise DafError(rc, "daf_window_attention_backward")


def _general_window_attention_backward(q, k, v, out, lse, grad_out, out_grad_q, out_grad_k, out_grad_v, workspace, window, sinks, scale, q_starts, stream):
    chk = _HeadChecks()
    p = _attention_parameters(chk, q, k, v, window, sinks, scale, q_starts, None, None, 1)
    for name, t in (("out", out), ("grad_out", grad_out), ("out_grad_q", out_grad_q)):
        chk.heads(name, t, q.dtype, *q.shape)
    for name, t in (("out_grad_k", out_grad_k), ("out_grad_v", out_grad_v)):
        chk.heads(name, t, q.dtype, *k.shape)
    chk.like("lse", lse, torch.float32, (q.shape[1], q.shape[0]))
    chk.workspace(workspace, daf_window_attention_backward_workspace_bytes(p.q_rows, p.q_heads, p.kv_heads, p.head_dim, p.sequences, window, sinks))
    chk.on_device()
    given = [_heads(t) for t in (q, k, v, out)]
    grads = [_heads(t) for t in (grad_out, out_grad_q, out_grad_k, out_grad_v)]
    return _library().daf_window_attention_backward(_at(p), *(_at(h) for h in given), lse.data_ptr(), *(_at(h) for h in grads), _pointer(workspace),
                                                    _stream_handle(stream))


def daf_window_attention_step_workspace_bytes(sequences: int, q_heads: int, kv_heads: int, head_dim: int, k_rows: int, window: int = 0,
                                              sinks: int = 0) -> int:
    """Enough for fewer sequences and rows of the cache too."""
    return int(_library().daf_window_attention_step_workspace_bytes(sequences, q_heads, kv_heads, head_dim, k_rows, window, sinks))


def daf_window_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, k_starts: torch.Tensor, k_lengths: torch.Tensor, out: torch.Tensor,
                              workspace: Optional[torch.Tensor] = None, *, window: int = 0, sinks: int = 0, scale: Optional[float] = None,
                              stream=None) -> None:
    """daf_window_attention for one query of each sequence, q [sequences, heads, head_dim], at the last of its keys."""
    rc = _fast.window_attention_step(q, k, v, out, k_starts, k_lengths, workspace, window, sinks, scale, stream)
    if rc is None:
        rc = _general_window_attention_step(q, k, v, out, k_starts, k_lengths, workspace, window, sinks, scale, stream)
    if rc == _EINVAL and workspace is None:                               # (a call may need none though fewer sequences do; it says so itself)
        need = daf_window_attention_step_workspace_bytes(*q.shape[:2], k.shape[1], q.shape[2], k.shape[0], window, sinks)
        if need > 0:
            raise ValueError(f"workspace: none, where {need} bytes serve such calls")
    if rc != 0:
        raise DafError(rc, "daf_window_attention_step")


def _general_window_attention_step(q, k, v, out, k_starts, k_lengths, workspace, window, sinks, scale, stream):
    chk = _HeadChecks()
    p = _attention_parameters(chk, q, k, v, window, sinks, scale, None, k_starts, k_lengths, q.shape[0] if isinstance(q, torch.Tensor) else 0)
    if k_starts is None:
        raise ValueError("k_starts and k_lengths: needed")
    chk.heads("out", out, q.dtype, *q.shape)
    if workspace is not None:
        chk.workspace(workspace, daf_window_attention_step_workspace_bytes(p.sequences, p.q_heads, p.kv_heads, p.head_dim, p.k_rows, window, sinks))
    chk.on_device()
    given = [_heads(t) for t in (q, k, v, out)]
    return _library().daf_window_attention_step(_at(p), *(_at(h) for h in given), _pointer(workspace), _stream_handle(stream))

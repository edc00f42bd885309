"""ctypes binding of include/daf_block.h: the operators of a transformer block's training step.  Same names as the C ABI; Python checks
and marshals arguments only."""
import ctypes
from typing import Optional

import torch

from .binding import _DTYPE_ID, _ELEM_DTYPES, DafError, _Args, _fast, _fast_calls, _stream_handle, load_library

_declared = None


def _library():
    """libdaf.so with the argument types of these calls."""
    global _declared
    if _declared is not None:
        return _declared
    L, c = load_library(), ctypes
    vp, i64, i32, f32 = c.c_void_p, c.c_int64, c.c_int32, c.c_float
    for name, result, arguments in (
            ("daf_grad_norm_workspace_bytes", i64, []),
            ("daf_grad_norm", c.c_int, [vp, i32, vp, vp, vp]),
            ("daf_clip_grad_norm", c.c_int, [vp, i32, f32, vp, vp, vp]),
            ("daf_gated_linear_workspace_bytes", i64, [i64, i64, i64, c.c_int]),
            ("daf_gated_linear", c.c_int, [vp, vp, vp, i64, i64, i64, c.c_int, c.c_int] + [vp] * 5),
            ("daf_gated_linear_schedule", c.c_int, [i64, i64, i64, c.c_int, vp]),
            ("daf_gated_linear_backward_workspace_bytes", i64, [i64, i64, i64, c.c_int]),
            ("daf_gated_linear_backward", c.c_int, [vp] * 6 + [i64, i64, i64, c.c_int, c.c_int] + [vp] * 6),
            ("daf_residual_norm", c.c_int, [vp] * 7),
            ("daf_residual_norm_backward_workspace_bytes", i64, [i64, i64, i64]),
            ("daf_residual_norm_backward", c.c_int, [vp] * 11)):
        getattr(L, name).restype = result
        getattr(L, name).argtypes = arguments
    if _fast_calls is not None:
        names = ("daf_clip_grad_norm", "daf_grad_norm_workspace_bytes", "daf_residual_norm", "daf_residual_norm_backward",
                 "daf_residual_norm_backward_workspace_bytes", "daf_gated_linear", "daf_gated_linear_workspace_bytes", "daf_gated_linear_backward",
                 "daf_gated_linear_backward_workspace_bytes")
        _fast_calls.bind_block({name: c.cast(getattr(L, name), vp).value for name in names})
    _declared = L
    return L


def _pointer(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


class _Checks(_Args):
    """The tensors of one call, as _Args; and that all are on one device."""

    def like(self, name: str, t, dtype, shape) -> None:
        self.tensor(name, t, dtype, 0)
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")

    def optional(self, name: str, t, dtype, shape) -> None:
        if t is not None:
            self.like(name, t, dtype, shape)

    def workspace(self, t, need: int) -> None:
        if t is None and need == 0:
            return
        if t is None:
            raise ValueError(f"workspace: {need} bytes are needed")
        self.tensor("workspace", t, t.dtype if isinstance(t, torch.Tensor) else None, 0)
        if t.numel() * t.element_size() < need:
            raise ValueError(f"workspace: {t.numel() * t.element_size()} bytes, {need} are needed")

    def on_device(self) -> None:
        super().on_device()
        for name, t in self.seen:
            if t.device != self.seen[0][1].device:
                raise ValueError(f"{name}: on {t.device}, {self.seen[0][0]} is on {self.seen[0][1].device}")


# ---- gradients ----
class _GradItem(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


def grad_items(items):
    """Marshals gradients, [grad, ...] (clipped in place), or [(grad, out), ...], once; the result can be passed to daf_grad_norm and
    daf_clip_grad_norm any number of times while the tensors stay alive and where they are."""
    pairs = [it if isinstance(it, (tuple, list)) else (it, it) for it in items]
    arr = (_GradItem * len(pairs))()
    chk = _Checks()
    for i, (it, (grad, out)) in enumerate(zip(arr, pairs)):
        chk.tensor(f"grad {i}", grad, _ELEM_DTYPES, 0)
        if out is not grad:
            chk.tensor(f"out {i}", out, grad.dtype, grad.numel(), exact=True)
        it.grad, it.out, it.n, it.dtype = grad.data_ptr(), out.data_ptr(), grad.numel(), _DTYPE_ID[grad.dtype]
    chk.on_device()
    arr.keep = pairs
    arr.on_device = pairs[0][0].get_device() if pairs else None
    return arr


def daf_grad_norm_workspace_bytes() -> int:
    return int(_library().daf_grad_norm_workspace_bytes())


def _grad_list(items, out_norm):
    """The array of grad_items, made or checked: of nothing else, and on out_norm's device."""
    try:
        if items.on_device == out_norm.get_device():
            return items
    except AttributeError:                       # a plain list, an array of something else, an out_norm that is no tensor
        if not isinstance(items, ctypes.Array):
            items = grad_items(items)
        elif items._type_ is not _GradItem:
            raise ValueError(f"items: an array of {items._type_.__name__}, not the result of grad_items") from None
    if isinstance(out_norm, torch.Tensor) and out_norm.is_cuda and len(items) > 0 and items.on_device != out_norm.get_device():
        raise ValueError(f"out_norm: on device {out_norm.get_device()}, the gradients are on {items.on_device}")
    return items


def _grad_call(items, out_norm, workspace):
    arr = _grad_list(items, out_norm)
    if not (isinstance(out_norm, torch.Tensor) and out_norm.dtype is torch.float32 and out_norm.is_cuda and out_norm.numel() == 1
            and isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.is_contiguous()
            and workspace.numel() * workspace.element_size() >= daf_grad_norm_workspace_bytes()):
        chk = _Checks()
        chk.tensor("out_norm", out_norm, torch.float32, 1, exact=True)
        chk.workspace(workspace, daf_grad_norm_workspace_bytes())
        chk.on_device()
    return arr


def daf_grad_norm(items, out_norm: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """The norm over all gradients of a list, or of the result of grad_items, into out_norm (one float on the device)."""
    arr = _grad_call(items, out_norm, workspace)
    rc = _library().daf_grad_norm(ctypes.addressof(arr), len(arr), out_norm.data_ptr(), workspace.data_ptr(), _stream_handle(stream))
    if rc != 0:
        raise DafError(rc, "daf_grad_norm")


def daf_clip_grad_norm(items, max_norm: float, out_norm: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """The norm into out_norm, and every gradient times min(1, max_norm / (norm + 1e-6)) into its `out`."""
    arr = _grad_list(items, out_norm)
    rc = _fast.clip_grad_norm(ctypes.addressof(arr), len(arr), max_norm, out_norm, workspace, stream)
    if rc is None:
        _grad_call(arr, out_norm, workspace)
        rc = _library().daf_clip_grad_norm(ctypes.addressof(arr), len(arr), max_norm, out_norm.data_ptr(), workspace.data_ptr(), _stream_handle(stream))
    if rc != 0:
        raise DafError(rc, "daf_clip_grad_norm")


# ---- norms, gate and residual sum ----
class _ResidualNorm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("gate_groups", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("kind", ctypes.c_int32), ("post", ctypes.c_int32), ("eps", ctypes.c_float), ("scale", ctypes.c_float),
                ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p), ("post_weight", ctypes.c_void_p), ("post_bias", ctypes.c_void_p),
                ("gate", ctypes.c_void_p)]


class _ResidualNormGrads(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("pre_weight", "pre_bias", "post_weight", "post_bias", "gate")]


NORM_KINDS = {"rms": 0, "layer": 1}


def _rows_of(t, name: str):
    if not isinstance(t, torch.Tensor) or t.dim() < 1:
        raise ValueError(f"{name}: expected a torch.Tensor of rows")
    cols = t.shape[-1]
    if cols < 1:
        raise ValueError(f"{name}: rows of no elements")
    return t.numel() // cols, cols


def _norm_parameters(chk, like, kind, eps, scale, post, pre_weight, pre_bias, post_weight, post_bias, gate, z):
    """The vectors checked against `like` (rows of the tensors), and the struct."""
    if kind not in NORM_KINDS:
        raise ValueError(f"kind: {kind!r} not in {tuple(NORM_KINDS)}")
    rows, cols = _rows_of(like, "residual")
    dtype, groups = like.dtype, 1
    for name, v in (("pre_weight", pre_weight), ("pre_bias", pre_bias), ("post_weight", post_weight), ("post_bias", post_bias)):
        chk.optional(name, v, dtype, (cols,))
    if gate is not None:
        chk.tensor("gate", gate, dtype, 0)
        if gate.dim() not in (1, 2) or gate.shape[-1] != cols:
            raise ValueError(f"gate: shape {tuple(gate.shape)}, expected ({cols},) or (groups, {cols})")
        groups = 1 if gate.dim() == 1 else gate.shape[0]
        if groups < 1 or rows % groups != 0:
            raise ValueError(f"gate: {groups} rows for {rows} rows of the tensors")
    if z is None and (post or gate is not None):
        raise ValueError("z: needed by `post` and by a gate")
    if not post and (post_weight is not None or post_bias is not None):
        raise ValueError("post_weight and post_bias belong to post=True")
    return rows, cols, groups, _ResidualNorm(rows, cols, groups, _DTYPE_ID[dtype], NORM_KINDS[kind], int(bool(post)), eps, scale, _pointer(pre_weight),
                                             _pointer(pre_bias), _pointer(post_weight), _pointer(post_bias), _pointer(gate))


def daf_residual_norm(residual: torch.Tensor, out_y: Optional[torch.Tensor], out_stats: Optional[torch.Tensor] = None, *, kind: str = "rms",
                      eps: float = 1e-5, z: Optional[torch.Tensor] = None, out_residual: Optional[torch.Tensor] = None, pre_weight=None,
                      pre_bias=None, post: bool = False, post_weight=None, post_bias=None, gate=None, scale: float = 1.0, stream=None) -> None:
    """out_residual = residual + scale * gate * post_norm(z); out_y = pre_norm(out_residual).  Tensors are [..., cols]; the norms are over the
    last dimension; gate is [cols] or [groups, cols]; out_stats is float32 [rows, 4]."""
    rc = _fast.residual_norm(residual, z, out_residual, out_y, out_stats, NORM_KINDS.get(kind), eps, scale, post, pre_weight, pre_bias, post_weight,
                             post_bias, gate, stream)
    if rc is None:
        rc = _general_residual_norm(residual, out_y, out_stats, kind, eps, z, out_residual, pre_weight, pre_bias, post, post_weight, post_bias, gate,
                                    scale, stream)
    if rc != 0:
        raise DafError(rc, "daf_residual_norm")


def _general_residual_norm(residual, out_y, out_stats, kind, eps, z, out_residual, pre_weight, pre_bias, post, post_weight, post_bias, gate, scale, stream):
    chk = _Checks()
    chk.tensor("residual", residual, _ELEM_DTYPES, 0)
    rows, cols, groups, p = _norm_parameters(chk, residual, kind, eps, scale, post, pre_weight, pre_bias, post_weight, post_bias, gate, z)
    for name, t in (("z", z), ("out_residual", out_residual), ("out_y", out_y)):
        chk.optional(name, t, residual.dtype, residual.shape)
    chk.optional("out_stats", out_stats, torch.float32, (rows, 4))
    chk.on_device()
    return _library().daf_residual_norm(ctypes.addressof(p), residual.data_ptr(), _pointer(z), _pointer(out_residual), _pointer(out_y),
                                        _pointer(out_stats), _stream_handle(stream))


def daf_residual_norm_backward_workspace_bytes(rows: int, cols: int, gate_groups: int = 1) -> int:
    return int(_library().daf_residual_norm_backward_workspace_bytes(rows, cols, gate_groups))


def daf_residual_norm_backward(sum: Optional[torch.Tensor], grad_y: Optional[torch.Tensor], stats: torch.Tensor, out_grad_residual: torch.Tensor,
                               workspace: Optional[torch.Tensor] = None, *, kind: str = "rms", z: Optional[torch.Tensor] = None,
                               grad_residual: Optional[torch.Tensor] = None, out_grad_z: Optional[torch.Tensor] = None, pre_weight=None,
                               post: bool = False, post_weight=None, post_bias=None, gate=None, scale: float = 1.0, out_grad_pre_weight=None,
                               out_grad_pre_bias=None, out_grad_post_weight=None, out_grad_post_bias=None, out_grad_gate=None, stream=None) -> None:
    """Backward of daf_residual_norm.  `sum` is its out_residual, `stats` its out_stats; grad_y and grad_residual are the gradients of out_y and
    out_residual (either may be None); the vectors' gradients are float32, those that are None are not computed."""
    vectors = (out_grad_pre_weight, out_grad_pre_bias, out_grad_post_weight, out_grad_post_bias)
    rc = _fast.residual_norm_backward(sum, z, stats, grad_y, grad_residual, out_grad_residual, out_grad_z, *vectors, out_grad_gate, workspace,
                                      NORM_KINDS.get(kind), 0.0, scale, post, pre_weight, None, post_weight, post_bias, gate, stream)
    if rc is None:
        rc = _general_residual_norm_backward(sum, grad_y, stats, out_grad_residual, workspace, kind, z, grad_residual, out_grad_z, pre_weight, post,
                                             post_weight, post_bias, gate, scale, vectors, out_grad_gate, stream)
    if rc != 0:
        raise DafError(rc, "daf_residual_norm_backward")


def _general_residual_norm_backward(sum, grad_y, stats, out_grad_residual, workspace, kind, z, grad_residual, out_grad_z, pre_weight, post, post_weight,
                                    post_bias, gate, scale, vectors, out_grad_gate, stream):
    chk = _Checks()
    chk.tensor("out_grad_residual", out_grad_residual, _ELEM_DTYPES, 0)
    rows, cols, groups, p = _norm_parameters(chk, out_grad_residual, kind, 0.0, scale, post, pre_weight, None, post_weight, post_bias, gate, z)
    dtype, shape = out_grad_residual.dtype, out_grad_residual.shape
    for name, t in (("sum", sum), ("grad_y", grad_y), ("z", z), ("grad_residual", grad_residual), ("out_grad_z", out_grad_z)):
        chk.optional(name, t, dtype, shape)
    chk.like("stats", stats, torch.float32, (rows, 4))
    for name, t in zip(("out_grad_pre_weight", "out_grad_pre_bias", "out_grad_post_weight", "out_grad_post_bias"), vectors):
        chk.optional(name, t, torch.float32, (cols,))
    if out_grad_gate is not None:
        if gate is not None:
            chk.like("out_grad_gate", out_grad_gate, torch.float32, gate.shape)
        else:
            chk.like("out_grad_gate", out_grad_gate, torch.float32, (cols,))
    if out_grad_gate is not None or any(t is not None for t in vectors):
        chk.workspace(workspace, daf_residual_norm_backward_workspace_bytes(rows, cols, groups))
    chk.on_device()
    grads = _ResidualNormGrads(*(_pointer(t) for t in vectors), _pointer(out_grad_gate))
    return _library().daf_residual_norm_backward(ctypes.addressof(p), _pointer(sum), _pointer(z), stats.data_ptr(), _pointer(grad_y),
                                                 _pointer(grad_residual), out_grad_residual.data_ptr(), _pointer(out_grad_z),
                                                 ctypes.addressof(grads), _pointer(workspace), _stream_handle(stream))


# ---- the gated feed-forward product ----
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}
_GATED_DTYPES = (torch.float16, torch.bfloat16)


def daf_gated_linear_workspace_bytes(M: int, N: int, K: int, dtype: torch.dtype) -> int:
    return int(_library().daf_gated_linear_workspace_bytes(M, N, K, _DTYPE_ID[dtype]))


def daf_gated_linear_backward_workspace_bytes(M: int, N: int, K: int, dtype: torch.dtype) -> int:
    return int(_library().daf_gated_linear_backward_workspace_bytes(M, N, K, _DTYPE_ID[dtype]))


class _GatedSchedule(ctypes.Structure):
    _fields_ = [("tile_rows", ctypes.c_int32), ("tile_cols", ctypes.c_int32), ("slices", ctypes.c_int32), ("tiles", ctypes.c_int64),
                ("whole_tiles", ctypes.c_int64)]


GATED_PRODUCTS = {"forward": 0, "grad_input": 1, "grad_weight": 2, "grad_input_of_both": 3, "grad_weight_of_both": 4}


def daf_gated_linear_schedule(M: int, N: int, K: int, product: str) -> dict:
    """How a product of these calls runs: tile_rows, tile_cols, slices, tiles, whole_tiles.  "grad_input" and "grad_weight": in a call that wants
    nothing of the other; with "_of_both": in one that wants both."""
    s = _GatedSchedule()
    rc = _library().daf_gated_linear_schedule(M, N, K, GATED_PRODUCTS[product], ctypes.addressof(s))
    if rc != 0:
        raise DafError(rc, "daf_gated_linear_schedule")
    return {name: getattr(s, name) for name, _ in s._fields_}


def _gated_operands(chk, x, w_gate, w_up, activation):
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation: {activation!r} not in {tuple(ACTIVATIONS)}")
    chk.tensor("x", x, _GATED_DTYPES, 0)
    chk.tensor("w_gate", w_gate, x.dtype, 0)
    if x.dim() != 2 or w_gate.dim() != 2 or x.shape[1] != w_gate.shape[1] or 0 in w_gate.shape:
        raise ValueError("x must be [M, K] and w_gate [N, K], N and K at least 1")
    chk.like("w_up", w_up, x.dtype, w_gate.shape)
    return x.shape[0], w_gate.shape[0], x.shape[1]


def daf_gated_linear(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, activation: str, out_h: torch.Tensor,
                     workspace: Optional[torch.Tensor] = None, out_gate: Optional[torch.Tensor] = None, out_up: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """out_h = act(x @ w_gate.T) * (x @ w_up.T); out_gate and out_up receive the two products, for the backward pass."""
    rc = _fast.gated_linear(x, w_gate, w_up, ACTIVATIONS.get(activation), out_h, workspace, out_gate, out_up, stream)
    if rc is None:
        rc = _general_gated_linear(x, w_gate, w_up, activation, out_h, workspace, out_gate, out_up, stream)
    if rc != 0:
        raise DafError(rc, "daf_gated_linear")


def _general_gated_linear(x, w_gate, w_up, activation, out_h, workspace, out_gate, out_up, stream):
    chk = _Checks()
    M, N, K = _gated_operands(chk, x, w_gate, w_up, activation)
    chk.like("out_h", out_h, x.dtype, (M, N))
    if (out_gate is None) != (out_up is None):
        raise ValueError("out_gate and out_up: both or neither")
    chk.optional("out_gate", out_gate, x.dtype, (M, N))
    chk.optional("out_up", out_up, x.dtype, (M, N))
    chk.workspace(workspace, daf_gated_linear_workspace_bytes(M, N, K, x.dtype))
    chk.on_device()
    return _library().daf_gated_linear(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), M, N, K, _DTYPE_ID[x.dtype], ACTIVATIONS[activation],
                                       out_h.data_ptr(), _pointer(out_gate), _pointer(out_up), _pointer(workspace), _stream_handle(stream))


def daf_gated_linear_backward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, grad_h: torch.Tensor, activation: str,
                              out_grad_x: Optional[torch.Tensor], out_grad_w_gate: Optional[torch.Tensor], out_grad_w_up: Optional[torch.Tensor],
                              workspace: torch.Tensor, gate: Optional[torch.Tensor] = None, up: Optional[torch.Tensor] = None,
                              out_h: Optional[torch.Tensor] = None, stream=None) -> None:
    """Backward of daf_gated_linear.  `gate` and `up` are its out_gate and out_up; without them they are computed again, and out_h receives h
    once more.  Outputs that are None are not computed."""
    rc = _fast.gated_linear_backward(x, w_gate, w_up, grad_h, ACTIVATIONS.get(activation), out_grad_x, out_grad_w_gate, out_grad_w_up, workspace, gate, up,
                                     out_h, stream)
    if rc is None:
        rc = _general_gated_linear_backward(x, w_gate, w_up, grad_h, activation, out_grad_x, out_grad_w_gate, out_grad_w_up, workspace, gate, up, out_h,
                                            stream)
    if rc != 0:
        raise DafError(rc, "daf_gated_linear_backward")


def _general_gated_linear_backward(x, w_gate, w_up, grad_h, activation, out_grad_x, out_grad_w_gate, out_grad_w_up, workspace, gate, up, out_h, stream):
    chk = _Checks()
    M, N, K = _gated_operands(chk, x, w_gate, w_up, activation)
    chk.like("grad_h", grad_h, x.dtype, (M, N))
    if (gate is None) != (up is None) or (out_grad_w_gate is None) != (out_grad_w_up is None):
        raise ValueError("gate and up, out_grad_w_gate and out_grad_w_up: both or neither")
    if gate is not None and out_h is not None:
        raise ValueError("out_h: only without gate and up")
    for name, t, shape in (("gate", gate, (M, N)), ("up", up, (M, N)), ("out_h", out_h, (M, N)), ("out_grad_x", out_grad_x, (M, K)),
                           ("out_grad_w_gate", out_grad_w_gate, (N, K)), ("out_grad_w_up", out_grad_w_up, (N, K))):
        chk.optional(name, t, x.dtype, shape)
    chk.workspace(workspace, daf_gated_linear_backward_workspace_bytes(M, N, K, x.dtype))
    chk.on_device()
    return _library().daf_gated_linear_backward(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), _pointer(gate), _pointer(up), grad_h.data_ptr(),
                                                M, N, K, _DTYPE_ID[x.dtype], ACTIVATIONS[activation], _pointer(out_grad_x), _pointer(out_grad_w_gate),
                                                _pointer(out_grad_w_up), _pointer(out_h), _pointer(workspace), _stream_handle(stream))

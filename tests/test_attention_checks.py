"""Host-side checks of daf_attention.h that need no GPU: what the C ABI refuses before it touches the device, and what the binding refuses."""
import ctypes

import pytest
import torch

import paper_2507_07149_amd as daf
from paper_2507_07149_amd import attention

EINVAL, EUNSUPPORTED = -1, -2
P, BIG = 1 << 20, 1 << 30            # addresses that are never used, far apart


@pytest.fixture(scope="module")
def lib():
    return attention._library()


def _h(at, token=64, head=16):
    return attention._Heads(at, token, head)


def _addresses(structs):
    return [None if s is None else ctypes.addressof(s) for s in structs]


def _rotation(lib, parameters=None, backward=False, **changes):
    """A call with addresses far apart and one thing changed: 6 tokens, 4 heads of queries and 2 of keys, of 16 elements."""
    fields = dict(tokens=6, positions=9, q_heads=4, kv_heads=2, head_dim=16, rotary_dim=16, dtype=2, pairing=0, norm=1, eps=1e-5, q_weight=P + 20 * BIG,
                  k_weight=P + 21 * BIG, cos=P + 22 * BIG, sin=P + 23 * BIG, position=P + 24 * BIG)
    fields.update(parameters or {})
    p = attention._HeadRotation(**fields)
    h = dict(q=_h(P), k=_h(P + BIG, 32), v=_h(P + 2 * BIG, 32), out_q=_h(P + 3 * BIG), out_k=_h(P + 4 * BIG, 32), out_v=_h(P + 5 * BIG, 32), rows=None, out_rows=6,
             grad_q=_h(P + 6 * BIG), grad_k=_h(P + 7 * BIG, 32), wq=P + 8 * BIG, wk=P + 9 * BIG, ws=P + 10 * BIG, p=p)
    h.update(changes)
    at = None if h["p"] is None else ctypes.addressof(h["p"])
    if backward:
        return lib.daf_head_rotation_backward(at, *_addresses([h["q"], h["k"], h["grad_q"], h["grad_k"], h["out_q"], h["out_k"]]), h["wq"], h["wk"], h["ws"], None)
    return lib.daf_head_rotation(at, *_addresses([h["q"], h["k"], h["v"], h["out_q"], h["out_k"], h["out_v"]]), h["rows"], h["out_rows"], None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("parameters,want", [
    (dict(tokens=-1), EINVAL), (dict(q_heads=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(head_dim=0), EINVAL), (dict(positions=-1), EINVAL),
    (dict(rotary_dim=-16), EINVAL), (dict(norm=2), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(position=None), EINVAL),
    (dict(position=P + 2), EINVAL), (dict(cos=None), EINVAL), (dict(sin=None), EINVAL), (dict(cos=P + 4), EINVAL), (dict(q_weight=P + 8), EINVAL),
    (dict(norm=0), EINVAL), (dict(dtype=3), EUNSUPPORTED), (dict(pairing=2), EUNSUPPORTED), (dict(head_dim=12), EUNSUPPORTED),
    (dict(head_dim=264), EUNSUPPORTED), (dict(rotary_dim=8), EUNSUPPORTED), (dict(rotary_dim=32), EUNSUPPORTED), (dict(tokens=1 << 31), EUNSUPPORTED),
    (dict(q_heads=4097), EUNSUPPORTED), (dict(positions=1 << 31), EUNSUPPORTED)])
def test_rotation_parameters(lib, backward, parameters, want):
    assert _rotation(lib, parameters, backward) == want


@pytest.mark.parametrize("changes,want", [
    (dict(p=None), EINVAL), (dict(q=None), EINVAL), (dict(q=_h(None)), EINVAL), (dict(q=_h(P + 8)), EINVAL), (dict(q=_h(P, 63)), EINVAL), (dict(q=_h(P, 8)), EINVAL),
    (dict(q=_h(P, 64, 8)), EINVAL), (dict(q=_h(P, 64, -16)), EINVAL), (dict(q=_h(P, 1 << 41)), EINVAL), (dict(out_q=_h(P + BIG, 64)), EINVAL), (dict(out_v=None), EINVAL), (dict(v=None), EINVAL),
    (dict(out_rows=7), EINVAL), (dict(out_rows=-1, rows=P + 26 * BIG), EINVAL), (dict(rows=P + 26 * BIG + 2), EINVAL), (dict(out_rows=1 << 31, rows=P + 26 * BIG), EUNSUPPORTED),
    (dict(out_q=_h(P + 16)), EINVAL), (dict(out_q=_h(P, 96)), EINVAL), (dict(out_k=_h(P + 3 * BIG + 64, 32)), EINVAL), (dict(out_q=_h(P + 3 * BIG, 32)), EINVAL),
    (dict(out_k=_h(P + 20 * BIG, 32)), EINVAL), (dict(out_v=_h(P + 24 * BIG, 32)), EINVAL), (dict(out_k=_h(P + BIG, 32), rows=P + 26 * BIG), EINVAL),
    (dict(q=_h(P, 128), out_q=_h(P, 128), k=_h(P + 96, 128)), EINVAL)])
def test_rotation_heads(lib, changes, want):
    assert _rotation(lib, **changes) == want


def test_rotation_of_more_than_any_memory(lib):
    far = _h(P + 4 * BIG, 1 << 40)
    assert _rotation(lib, out_k=far, out_rows=(1 << 31) - 65536, rows=P + 26 * BIG) == EINVAL


@pytest.mark.parametrize("changes,want", [
    (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(grad_q=None), EINVAL), (dict(out_k=None), EINVAL), (dict(ws=None), EINVAL), (dict(ws=P + 8), EINVAL),
    (dict(wq=P + 2), EINVAL), (dict(wk=P + 8 * BIG), EINVAL), (dict(ws=P + 3 * BIG), EINVAL), (dict(out_q=_h(P)), EINVAL), (dict(out_q=_h(P + 6 * BIG + 32)), EINVAL),
    (dict(out_k=_h(P + 6 * BIG, 32)), EINVAL), (dict(wq=P + 20 * BIG), EINVAL)])
def test_rotation_backward_heads(lib, changes, want):
    assert _rotation(lib, backward=True, **changes) == want


def test_rotation_backward_without_norm_has_no_weights(lib):
    assert _rotation(lib, dict(norm=0, q_weight=None, k_weight=None), True, q=None, k=None) == EINVAL


def test_rotation_workspace_sizes():
    assert daf.daf_head_rotation_backward_workspace_bytes(0, 4, 2, 64) == 0
    assert daf.daf_head_rotation_backward_workspace_bytes(5, 4, 2, 64) == 2 * 2 * 64 * 4
    for bad in ((-1, 4, 2, 64), (5, 0, 2, 64), (5, 4, 0, 64), (5, 4, 2, 0), (5, 4, 2, 65), (5, 4, 2, 512), (1 << 31, 4, 2, 64)):
        assert daf.daf_head_rotation_backward_workspace_bytes(*bad) == -1


def _attention(lib, kind="forward", parameters=None, **changes):
    """A call of `kind`: 6 queries of 4 heads, 2 heads of keys, of 16 elements."""
    step = kind == "step"
    fields = dict(q_rows=6, k_rows=20 if step else 6, sequences=6 if step else 2, window=3, sinks=1, q_heads=4, kv_heads=2, head_dim=16, dtype=2, scale=0.25,
                  q_starts=None if step else P + 20 * BIG, k_starts=P + 21 * BIG if step else None, k_lengths=P + 22 * BIG if step else None)
    fields.update(parameters or {})
    p = attention._WindowAttention(**fields)
    h = dict(p=p, q=_h(P), k=_h(P + BIG, 32), v=_h(P + 2 * BIG, 32), out=_h(P + 3 * BIG), lse=P + 4 * BIG, grad=_h(P + 5 * BIG), gq=_h(P + 6 * BIG), gk=_h(P + 7 * BIG, 32),
             gv=_h(P + 8 * BIG, 32), ws=P + 9 * BIG)
    h.update(changes)
    at = None if h["p"] is None else ctypes.addressof(h["p"])
    tensors = _addresses([h["q"], h["k"], h["v"], h["out"]])
    if kind == "forward":
        return lib.daf_window_attention(at, *tensors, h["lse"], None)
    if kind == "step":
        return lib.daf_window_attention_step(at, *tensors, h["ws"], None)
    return lib.daf_window_attention_backward(at, *tensors, h["lse"], *_addresses([h["grad"], h["gq"], h["gk"], h["gv"]]), h["ws"], None)


@pytest.mark.parametrize("kind", ["forward", "backward", "step"])
@pytest.mark.parametrize("parameters,want", [
    (dict(q_rows=-1), EINVAL), (dict(k_rows=-1), EINVAL), (dict(q_heads=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(kv_heads=3), EINVAL), (dict(head_dim=0), EINVAL),
    (dict(sequences=0), EINVAL), (dict(window=-1), EINVAL), (dict(sinks=-1), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(q_starts=P + 2), EINVAL), (dict(k_starts=P + 1, k_lengths=P + 4), EINVAL), (dict(k_starts=P, k_lengths=None), EINVAL), (dict(k_starts=None, k_lengths=P), EINVAL),
    (dict(dtype=0), EUNSUPPORTED), (dict(dtype=7), EUNSUPPORTED), (dict(head_dim=20), EUNSUPPORTED), (dict(head_dim=136), EUNSUPPORTED),
    (dict(q_rows=1 << 30), EUNSUPPORTED), (dict(k_rows=1 << 30), EUNSUPPORTED), (dict(q_rows=(1 << 20) + 1, sequences=(1 << 20) + 1), EUNSUPPORTED),
    (dict(q_heads=4096, kv_heads=2, sequences=1024), EUNSUPPORTED), (dict(q_heads=4098), EUNSUPPORTED)])
def test_attention_parameters(lib, kind, parameters, want):
    assert _attention(lib, kind, parameters) == want


@pytest.mark.parametrize("kind", ["forward", "backward"])
def test_sequences_of_a_call(lib, kind):
    assert _attention(lib, kind, dict(sequences=(1 << 16) + 1)) == EUNSUPPORTED


@pytest.mark.parametrize("kind", ["forward", "backward", "step"])
@pytest.mark.parametrize("changes,want", [
    (dict(p=None), EINVAL), (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=_h(None)), EINVAL), (dict(out=None), EINVAL), (dict(q=_h(P + 4)), EINVAL), (dict(k=_h(P + BIG, 36)), EINVAL),
    (dict(v=_h(P + 2 * BIG, 32, 8)), EINVAL), (dict(q=_h(P, 1 << 23)), EUNSUPPORTED), (dict(k=_h(P + BIG, 1 << 23)), EUNSUPPORTED)])
def test_attention_heads(lib, kind, changes, want):
    assert _attention(lib, kind, **changes) == want


def test_attention_outputs(lib):
    for changes in (dict(lse=P + 2), dict(out=_h(P)), dict(out=_h(P + BIG + 16)), dict(out=_h(P + 3 * BIG, 48)), dict(lse=P + 3 * BIG + 16), dict(lse=P + 20 * BIG), dict(lse=P)):
        assert _attention(lib, **changes) == EINVAL, changes
    assert _attention(lib, parameters=dict(q_starts=None)) == EINVAL                    # several sequences of no known rows
    assert _attention(lib, parameters=dict(k_rows=7)) == EINVAL                         # keys that are the queries' rows
    for changes in (dict(lse=None), dict(ws=None), dict(ws=P + 8), dict(grad=None), dict(gq=None), dict(gk=_h(P + 6 * BIG, 32)), dict(gv=_h(P + 7 * BIG + 16, 32)), dict(gq=_h(P)),
                    dict(gk=_h(P + BIG, 32)), dict(ws=P + 8 * BIG), dict(gq=_h(P + 5 * BIG)), dict(gv=_h(P + 2 * BIG, 32)), dict(gq=_h(P + 3 * BIG)), dict(gq=_h(P + 4 * BIG))):
        assert _attention(lib, "backward", **changes) == EINVAL, changes
    assert _attention(lib, "backward", dict(k_starts=P + 21 * BIG, k_lengths=P + 22 * BIG)) == EINVAL
    assert _attention(lib, "backward", dict(k_rows=7)) == EINVAL
    for parameters in (dict(q_starts=P + 20 * BIG), dict(sequences=5), dict(k_starts=None, k_lengths=None)):
        assert _attention(lib, "step", parameters) == EINVAL
    for changes in (dict(out=_h(P)), dict(out=_h(P + 2 * BIG, 64)), dict(out=_h(P + 22 * BIG))):
        assert _attention(lib, "step", **changes) == EINVAL, changes


def test_attention_workspace_sizes():
    for bad in ((-1, 4, 2, 64), (5, 4, 3, 64), (5, 4, 2, 65), (5, 4, 2, 136), (1 << 31, 4, 2, 64), (5, 4, 2, 64, 0), (5, 4, 2, 64, 1, -1), (5, 4, 2, 64, 1, 0, -1)):
        assert daf.daf_window_attention_backward_workspace_bytes(*bad) == -1
    for bad in ((-1, 4, 2, 64, 9), (5, 4, 3, 64, 9), (5, 4, 2, 65, 9), (5, 4, 2, 64, -1), (5, 4, 2, 64, 9, -1), (5, 4, 2, 64, 9, 0, -1)):
        assert daf.daf_window_attention_step_workspace_bytes(*bad) == -1
    assert daf.daf_window_attention_step_workspace_bytes(0, 4, 2, 64, 9) == 0
    assert daf.daf_window_attention_backward_workspace_bytes(100, 4, 2, 64) >= 100 * 4 * 4


def test_workspaces_serve_smaller_calls():
    """What a query says for some sequences and rows is enough for fewer of either: a program asks once, for its largest call."""
    from random import Random
    r = Random(1)
    size = lambda most: max(1, int(most ** r.random()))
    for _ in range(4000):
        kv = r.choice((1, 2, 5, 8, 12, 30, 64))
        heads, dim = kv * r.choice((1, 2, 4, 8, 40)), r.choice((8, 64, 80, 128))
        window, sinks = r.choice((0, 1, 100, size(1 << 14), size(1 << 40))), r.choice((0, 0, 1, 4, 40, 200, size(1 << 14)))
        rows, sequences = size(1 << 17), size(1 << 10)
        few, short = r.choice((1, size(sequences), sequences)), r.choice((1, size(rows), rows // 2, rows))
        large = daf.daf_window_attention_backward_workspace_bytes(rows, heads, kv, dim, sequences, window, sinks)
        case = (rows, short, sequences, few, heads, kv, dim, window, sinks)
        assert -1 < daf.daf_window_attention_backward_workspace_bytes(short, heads, kv, dim, few, window, sinks) <= large or large == -1, case
        assert -1 < daf.daf_head_rotation_backward_workspace_bytes(short, heads, kv, dim) <= daf.daf_head_rotation_backward_workspace_bytes(rows, heads, kv, dim), case
        large = daf.daf_window_attention_step_workspace_bytes(sequences, heads, kv, dim, rows, window, sinks)
        assert -1 < daf.daf_window_attention_step_workspace_bytes(few, heads, kv, dim, short, window, sinks) <= large or large == -1, case


def test_workspaces_are_bounded():
    """What sums of pieces and far queries may take does not grow without end."""
    stats = 2 * 4 * (1 << 20) * 32
    assert daf.daf_window_attention_backward_workspace_bytes(1 << 20, 32, 8, 128, 64, 4096, 4) <= stats + 16 + (3 << 28)
    assert daf.daf_window_attention_step_workspace_bytes(1 << 16, 32, 8, 128, 1 << 26) <= 1 << 26
    assert daf.daf_window_attention_step_workspace_bytes(1 << 16, 32, 8, 128, 1 << 26, 160) == 0


# ---- the binding ----
def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def _rotation_call(**changes):
    a = dict(q=_t(6, 4, 32), k=_t(6, 2, 32), position=_t(6, dtype=torch.int32), cos=_t(9, 8, dtype=torch.float32), sin=_t(9, 8, dtype=torch.float32), out_q=_t(6, 4, 32),
             out_k=_t(6, 2, 32))
    a.update(changes)
    daf.daf_head_rotation(**a)


@pytest.mark.parametrize("changes,what", [
    (dict(), "device"), (dict(q=1), "torch.Tensor"), (dict(q=_t(6, 128)), "shape"), (dict(q=_t(6, 32, 4).transpose(1, 2)), "strides"),
    (dict(q=_t(6, 4, 36)[:, :, :32]), "strides"), (dict(q=_t(1, 4, 32).expand(6, 4, 32)), "strides"),
    (dict(k=_t(5, 2, 32)), "k: shape"), (dict(k=_t(6, 2, 32, dtype=torch.float16)), "k: dtype"), (dict(position=_t(6, dtype=torch.int64)), "position: dtype"),
    (dict(position=_t(5, dtype=torch.int32)), "position: shape"), (dict(cos=_t(9, 8)), "cos: dtype"), (dict(cos=_t(72, dtype=torch.float32)), "cos: shape"),
    (dict(sin=_t(9, 4, dtype=torch.float32)), "sin: shape"), (dict(out_q=_t(6, 3, 32)), "out_q: shape"), (dict(out_k=_t(8, 2, 32)), "out_k: shape"),
    (dict(v=_t(6, 2, 32)), "both or neither"), (dict(v=_t(6, 2, 32), out_v=_t(7, 2, 32)), "out_v: shape"), (dict(rows=_t(5, dtype=torch.int32)), "rows: shape"),
    (dict(q_weight=_t(32), norm=False), "norm"), (dict(q_weight=_t(16)), "q_weight: shape"), (dict(pairing="thirds"), "pairing")])
def test_rotation_binding(changes, what):
    with pytest.raises(ValueError, match=what):
        _rotation_call(**changes)


def _backward_call(**changes):
    a = dict(q=_t(6, 4, 32), k=_t(6, 2, 32), position=_t(6, dtype=torch.int32), cos=_t(9, 8, dtype=torch.float32), sin=_t(9, 8, dtype=torch.float32), grad_q=_t(6, 4, 32),
             grad_k=_t(6, 2, 32), out_grad_q=_t(6, 4, 32), out_grad_k=_t(6, 2, 32))
    a.update(changes)
    daf.daf_head_rotation_backward(**a)


@pytest.mark.parametrize("changes,what", [
    (dict(), "device"), (dict(q=None), "q: expected"), (dict(q=None, k=None, norm=False), "device"), (dict(k=_t(6, 4, 32)), "k: shape"), (dict(out_grad_k=_t(6, 4, 32)), "out_grad_k: shape"),
    (dict(out_grad_q_weight=_t(32, dtype=torch.float32)), "workspace"), (dict(out_grad_k_weight=_t(32)), "out_grad_k_weight: dtype"),
    (dict(out_grad_q_weight=_t(32, dtype=torch.float32), workspace=_t(4)), "workspace"), (dict(out_grad_q_weight=_t(32, dtype=torch.float32), norm=False), "norm")])
def test_rotation_backward_binding(changes, what):
    with pytest.raises(ValueError, match=what):
        _backward_call(**changes)


def _attention_call(kind, **changes):
    starts = torch.tensor([0, 2, 6], dtype=torch.int32)
    a = dict(q=_t(6, 4, 32), k=_t(6, 2, 32), v=_t(6, 2, 32), out=_t(6, 4, 32))
    if kind == "forward":
        a |= dict(q_starts=starts)
    elif kind == "backward":
        a |= dict(q_starts=starts, lse=_t(4, 6, dtype=torch.float32), grad_out=_t(6, 4, 32), out_grad_q=_t(6, 4, 32), out_grad_k=_t(6, 2, 32), out_grad_v=_t(6, 2, 32),
                  workspace=_t(1 << 20))
    else:
        a |= dict(k_starts=_t(6, dtype=torch.int32), k_lengths=_t(6, dtype=torch.int32), workspace=_t(1 << 20))
    a.update(changes)
    {"forward": daf.daf_window_attention, "backward": daf.daf_window_attention_backward, "step": daf.daf_window_attention_step}[kind](**a)


@pytest.mark.parametrize("kind", ["forward", "backward", "step"])
@pytest.mark.parametrize("changes,what", [
    (dict(), "device"), (dict(q=_t(6, 4, 32, dtype=torch.float32)), "dtype"), (dict(k=_t(6, 2, 64)), "k: shape"), (dict(v=_t(6, 1, 32)), "v: shape"), (dict(q=_t(6, 3, 32)), "3 heads"),
    (dict(out=_t(6, 2, 32)), "out: shape"), (dict(k=_t(2, 6, 32).transpose(0, 1), q=_t(6, 4, 33)[:, :, :32]), "q: strides")])
def test_attention_binding(kind, changes, what):
    with pytest.raises(ValueError, match=what):
        _attention_call(kind, **changes)


@pytest.mark.parametrize("kind,changes,what", [
    ("forward", dict(q_starts=torch.zeros(3, dtype=torch.int64)), "q_starts: dtype"), ("forward", dict(q_starts=torch.zeros(1, dtype=torch.int32)), "q_starts"),
    ("forward", dict(q_starts=torch.zeros(2, 2, dtype=torch.int32)), "q_starts: shape"), ("forward", dict(k=_t(7, 2, 32), v=_t(7, 2, 32)), "7 rows"),
    ("forward", dict(k_starts=torch.zeros(2, dtype=torch.int32)), "both or neither"), ("forward", dict(k_starts=torch.zeros(3, dtype=torch.int32), k_lengths=torch.zeros(3, dtype=torch.int32)), "k_starts: shape"),
    ("forward", dict(out_lse=_t(6, 4, dtype=torch.float32)), "out_lse: shape"), ("backward", dict(lse=_t(6, 4, dtype=torch.float32)), "lse: shape"),
    ("backward", dict(workspace=_t(2)), "workspace"), ("backward", dict(out_grad_k=_t(6, 4, 32)), "out_grad_k: shape"), ("backward", dict(k=_t(7, 2, 32), v=_t(7, 2, 32)), "7 rows"),
    ("forward", dict(window=1 << 63), "window"), ("step", dict(sinks=1 << 64), "sinks"), ("backward", dict(window=3.0), "window"),
    ("step", dict(k_starts=None, k_lengths=None, k=_t(6, 2, 32)), "needed"), ("step", dict(k_lengths=torch.zeros(5, dtype=torch.int32)), "k_lengths: shape")])
def test_attention_binding_of_each(kind, changes, what):
    with pytest.raises(ValueError, match=what):
        _attention_call(kind, **changes)

"""Host-side checks of daf_block.h that need no GPU: what the C ABI refuses before it touches the device, and what the binding refuses."""
import ctypes

import pytest
import torch

import paper_2507_07149_amd as daf
from paper_2507_07149_amd import block

EINVAL, EUNSUPPORTED = -1, -2
P = 1 << 20                       # an address that is never used


@pytest.fixture(scope="module")
def lib():
    return block._library()


def _items(*fields):
    arr = (block._GradItem * len(fields))()
    for it, f in zip(arr, fields):
        it.grad, it.out, it.n, it.dtype = f
    return ctypes.addressof(arr), arr


@pytest.mark.parametrize("item,want", [
    ((None, P, 4, 0), EINVAL), ((P, None, 4, 0), EINVAL), ((P + 2, P, 4, 0), EINVAL), ((P, P + 1, 4, 1), EINVAL), ((P, P, -1, 0), EINVAL),
    ((P, P, 4, 3), EUNSUPPORTED), ((P, P + 4, 4, 0), EINVAL), ((P, P - 4, 4, 0), EINVAL), ((P, P, 1 << 50, 0), EUNSUPPORTED)])
def test_gradient_lists(lib, item, want):
    at, keep = _items((P, P, 8, 0), item)
    assert lib.daf_clip_grad_norm(at, 2, 1.0, P, P, None) == want


def test_gradient_arguments(lib):
    at, keep = _items((P, P, 8, 0))
    assert lib.daf_clip_grad_norm(None, 1, 1.0, P, P, None) == EINVAL
    assert lib.daf_clip_grad_norm(at, 0, 1.0, P, P, None) == EINVAL
    assert lib.daf_clip_grad_norm(at, 1, 1.0, None, P, None) == EINVAL
    assert lib.daf_clip_grad_norm(at, 1, 1.0, P + 2, P, None) == EINVAL
    assert lib.daf_clip_grad_norm(at, 1, 1.0, P, None, None) == EINVAL
    assert lib.daf_clip_grad_norm(at, 1, 1.0, P, P + 8, None) == EINVAL
    assert lib.daf_clip_grad_norm(at, 1, -1.0, P, P, None) == EINVAL
    assert lib.daf_clip_grad_norm(at, 1, float("nan"), P, P, None) == EINVAL
    assert lib.daf_grad_norm(at, 1, None, P, None) == EINVAL


def _norm(**changes):
    fields = dict(rows=6, cols=32, gate_groups=1, dtype=0, kind=0, post=0, eps=1e-5, scale=1.0, pre_weight=None, pre_bias=None, post_weight=None,
                  post_bias=None, gate=None)
    fields.update(changes)
    return block._ResidualNorm(**fields)


BIG = 1 << 30                     # tensors far apart


@pytest.mark.parametrize("changes,want", [
    (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(cols=16385), EUNSUPPORTED), (dict(rows=1 << 31), EUNSUPPORTED), (dict(dtype=3), EUNSUPPORTED),
    (dict(kind=2), EUNSUPPORTED), (dict(post=2), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(gate_groups=0), EINVAL),
    (dict(gate_groups=4, gate=P), EINVAL), (dict(gate_groups=2), EINVAL), (dict(pre_weight=P + 4), EINVAL), (dict(gate=P + 8), EINVAL)])
def test_norm_parameters(lib, changes, want):
    parameters = _norm(**changes)
    p = ctypes.addressof(parameters)
    assert lib.daf_residual_norm(p, P, P + BIG, P + 2 * BIG, P + 3 * BIG, None, None) == want
    grads = block._ResidualNormGrads()
    assert lib.daf_residual_norm_backward(p, P, P + BIG, P + 2 * BIG, P + 3 * BIG, None, P + 4 * BIG, P + 5 * BIG, ctypes.addressof(grads), None, None) == want


def test_norm_tensors(lib):
    plain, posted = _norm(), _norm(post=1)
    n, q = ctypes.addressof(plain), ctypes.addressof(posted)
    call = lambda p, *t: lib.daf_residual_norm(p, *t, None)
    r, z, s, y, st = P, P + BIG, P + 2 * BIG, P + 3 * BIG, P + 4 * BIG
    assert lib.daf_residual_norm(None, r, z, s, y, st, None) == EINVAL
    assert call(n, None, z, s, y, st) == EINVAL and call(n, r, z, None, None, st) == EINVAL
    assert call(q, r, None, s, y, st) == EINVAL                                # a norm of nothing
    assert call(n, r + 4, z, s, y, st) == EINVAL and call(n, r, z, s, y, st + 4) == EINVAL
    assert call(n, r, z, r + 16, y, st) == EINVAL and call(n, r, z, s, z - 16, st) == EINVAL
    assert call(n, r, z, s, s, st) == EINVAL and call(n, r, z, s, y, y) == EINVAL


def test_norm_backward_tensors(lib):
    plain, posted, none = _norm(), _norm(post=1), block._ResidualNormGrads()
    n, g = ctypes.addressof(plain), ctypes.addressof(none)
    s, z, st, dy, ds, dr, dz = (P + i * BIG for i in range(7))

    def call(p=n, sum=s, z=z, stats=st, dy=dy, ds=ds, dr=dr, dz=dz, grads=g, ws=None):
        return lib.daf_residual_norm_backward(p, sum, z, stats, dy, ds, dr, dz, grads, ws, None)

    assert call(p=None) == EINVAL and call(grads=None) == EINVAL and call(dy=None, ds=None) == EINVAL and call(sum=None) == EINVAL
    assert call(stats=None) == EINVAL and call(dr=None) == EINVAL and call(dz=None) == EINVAL and call(z=None) == EINVAL
    assert call(dr=s) == EINVAL and call(dr=z) == EINVAL and call(dr=dz) == EINVAL and call(dr=dy + 16) == EINVAL and call(dz=s) == EINVAL
    for name, more in (("pre_weight", dict(dy=None)), ("post_weight", {}), ("post_bias", {}), ("gate", dict(z=None, dz=None)), ("pre_weight", {})):
        wanted = block._ResidualNormGrads(**{name: P})                          # (the last: a workspace is needed)
        assert call(grads=ctypes.addressof(wanted), **more) == EINVAL, name
    wanted = block._ResidualNormGrads(pre_weight=P + 2)
    assert call(grads=ctypes.addressof(wanted), ws=P) == EINVAL


def test_norm_workspace_sizes():
    assert daf.daf_residual_norm_backward_workspace_bytes(0, 5) == 0
    assert daf.daf_residual_norm_backward_workspace_bytes(4, 5) == 5 * 5 * 4
    for bad in ((-1, 5, 1), (4, 0, 1), (4, 5, 3), (4, 5, 0), (4, 20000, 1)):
        assert daf.daf_residual_norm_backward_workspace_bytes(*bad) == -1


def test_binding_refuses():
    t, w = torch.zeros(4, 8), torch.zeros(8)
    for call, text in (
            (lambda: daf.grad_items([t.double()]), "dtype"),
            (lambda: daf.grad_items([(t, t[:2])]), "elements"),
            (lambda: daf.grad_items([t.t()]), "contiguous"),
            (lambda: daf.grad_items([t]), "device"),
            (lambda: daf.daf_residual_norm(t, t, kind="batch"), "kind"),
            (lambda: daf.daf_residual_norm(t, t[:2]), "shape"),
            (lambda: daf.daf_residual_norm(t, t, pre_weight=w[:4]), "shape"),
            (lambda: daf.daf_residual_norm(t, t, pre_weight=w.half()), "dtype"),
            (lambda: daf.daf_residual_norm(t, t, z=t, gate=torch.zeros(3, 8)), "gate"),
            (lambda: daf.daf_residual_norm(t, t, gate=w), "z:"),
            (lambda: daf.daf_residual_norm(t, t, z=t, post_weight=w), "post=True"),
            (lambda: daf.daf_residual_norm(t, t, torch.zeros(4, 3)), "shape"),
            (lambda: daf.daf_residual_norm(t, t), "device"),
            (lambda: daf.daf_residual_norm_backward(t, t, torch.zeros(4, 4), t, None, out_grad_pre_weight=w), "workspace"),
            (lambda: daf.daf_residual_norm_backward(t, t, torch.zeros(4, 4), t, torch.zeros(3), out_grad_pre_weight=w), "workspace"),
            (lambda: daf.daf_residual_norm_backward(t, t[:1], torch.zeros(4, 4), t), "shape")):
        with pytest.raises(ValueError, match=text):
            call()

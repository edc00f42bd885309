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


def _gated(lib, backward=False, **changes):
    """A forward (backward) call with addresses far apart and one thing changed."""
    a = dict(x=P, wg=P + BIG, wu=P + 2 * BIG, M=40, N=6, K=9, dtype=2, act=0, ws=P + 9 * BIG)
    if backward:
        a |= dict(gate=None, up=None, gh=P + 3 * BIG, dx=P + 4 * BIG, dwg=P + 5 * BIG, dwu=P + 6 * BIG, h=P + 7 * BIG)
    else:
        a |= dict(h=P + 3 * BIG, gate=None, up=None)
    a |= changes
    first = [a["x"], a["wg"], a["wu"]]
    sizes = [a["M"], a["N"], a["K"], a["dtype"], a["act"]]
    if backward:
        return lib.daf_gated_linear_backward(*first, a["gate"], a["up"], a["gh"], *sizes, a["dx"], a["dwg"], a["dwu"], a["h"], a["ws"], None)
    return lib.daf_gated_linear(*first, *sizes, a["h"], a["gate"], a["up"], a["ws"], None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("changes,want", [
    (dict(dtype=0), EUNSUPPORTED), (dict(dtype=5), EUNSUPPORTED), (dict(act=4), EUNSUPPORTED), (dict(act=-1), EUNSUPPORTED), (dict(M=-1), EINVAL), (dict(N=0), EINVAL),
    (dict(K=0), EINVAL), (dict(M=1 << 24), EUNSUPPORTED), (dict(N=1 << 20), EUNSUPPORTED), (dict(K=1 << 21), EUNSUPPORTED), (dict(x=None), EINVAL),
    (dict(wg=None), EINVAL), (dict(wu=None), EINVAL), (dict(ws=None), EINVAL), (dict(x=P + 8), EINVAL), (dict(ws=P + 9 * BIG + 4), EINVAL),
    (dict(gate=P + 8 * BIG), EINVAL), (dict(h=P), EINVAL), (dict(h=P + BIG + 16), EINVAL), (dict(ws=P + 2 * BIG - 16), EINVAL)])
def test_gated_arguments(lib, backward, changes, want):
    assert _gated(lib, backward, **changes) == want


def test_gated_outputs(lib):
    assert _gated(lib, h=None) == EINVAL
    assert _gated(lib, gate=P + 4 * BIG, up=P + 4 * BIG) == EINVAL
    both = dict(gate=P + 8 * BIG, up=P + 10 * BIG)
    for changes in (dict(gh=None), dict(dwu=None), dict(dwg=None), dict(dx=None, dwg=None, dwu=None, h=None), dict(**both), dict(dx=P + 3 * BIG),
                    dict(dwg=P + 6 * BIG + 32), dict(dx=P), dict(h=None, dx=P + 8 * BIG, **both)):
        assert _gated(lib, True, **changes) == EINVAL, changes
    assert _gated(lib, True, M=0, dwu=P + 5 * BIG + 16) == EINVAL
    assert _gated(lib, M=0, x=None, h=None, ws=None) == 0


def test_gated_workspace_sizes():
    bf16 = torch.bfloat16
    assert daf.daf_gated_linear_workspace_bytes(8192, 11008, 4096, bf16) == 0            # whole loads, more tiles than compute units
    assert daf.daf_gated_linear_workspace_bytes(0, 5, 7, bf16) == 0 == daf.daf_gated_linear_backward_workspace_bytes(0, 5, 7, bf16)
    assert daf.daf_gated_linear_backward_workspace_bytes(8192, 11008, 4096, bf16) >= 8192 * 2 * 11008 * 2
    for bad in ((-1, 5, 5), (5, 0, 5), (5, 5, 0), (1 << 24, 5, 5)):
        assert daf.daf_gated_linear_workspace_bytes(*bad, bf16) == -1 == daf.daf_gated_linear_backward_workspace_bytes(*bad, bf16)
    assert daf.daf_gated_linear_workspace_bytes(5, 5, 5, torch.float32) == -1


def test_gated_schedule():
    for m, n, k in ((1, 1, 1), (1, 11008, 4096), (1576, 2048, 768), (8192, 11008, 4096), (40, 64, 4096), (1000, 3001, 511)):
        for product, rows, cols in (("forward", m, 2 * -(-n // 64) * 64), ("grad_input", m, k), ("grad_weight", 2 * -(-n // 64) * 64, k)):
            s = daf.daf_gated_linear_schedule(m, n, k, product)
            large = -(-rows // 256) * -(-cols // 256)
            tiles = -(-rows // s["tile_rows"]) * -(-cols // s["tile_cols"])
            if s["whole_tiles"]:
                assert s["whole_tiles"] % 256 == 0 and s["whole_tiles"] < large
                tiles = (large - s["whole_tiles"]) * (256 // s["tile_rows"]) * (256 // s["tile_cols"])
            assert s["tiles"] == tiles and s["slices"] >= 1
    with pytest.raises(daf.DafError):
        daf.daf_gated_linear_schedule(0, 5, 5, "forward")


def test_binding_refuses_gated():
    x, w, h = (torch.zeros(*s, dtype=torch.bfloat16) for s in ((4, 8), (6, 8), (4, 6)))
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    for call, text in (
            (lambda: daf.daf_gated_linear(x, w, w, "tanh", h, ws), "activation"),
            (lambda: daf.daf_gated_linear(x.float(), w, w, "silu", h, ws), "dtype"),
            (lambda: daf.daf_gated_linear(x, w.half(), w, "silu", h, ws), "dtype"),
            (lambda: daf.daf_gated_linear(x, w[:, :7], w, "silu", h, ws), "contiguous"),
            (lambda: daf.daf_gated_linear(x, w[:5], w, "silu", h, ws), "shape"),
            (lambda: daf.daf_gated_linear(x, w, w, "silu", h[:3], ws), "shape"),
            (lambda: daf.daf_gated_linear(x, w, w, "silu", h, ws, out_gate=h), "both or neither"),
            (lambda: daf.daf_gated_linear(x, w, w, "silu", h, ws), "device"),
            (lambda: daf.daf_gated_linear_backward(x, w, w, h, "silu", x, w, w, ws[:64]), "workspace"),
            (lambda: daf.daf_gated_linear_backward(x, w, w, h, "silu", x, w, None, ws), "both or neither"),
            (lambda: daf.daf_gated_linear_backward(x, w, w, h, "silu", x, w, w, ws, gate=h, up=h, out_h=h), "only without")):
        with pytest.raises(ValueError, match=text):
            call()


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


def test_sums_of_gate_rows_fit_a_launch():
    """Only rows of the gate that several workgroups share are added up by a launch of their own, of 1024 threads to 32 columns of one: below 2^32 threads."""
    for cols in (1, 512, 513, 1024, 1025, 2048, 4096, 4097, 16384):
        for groups in (1, 2, 255, 256, 1023, 1024, 2047, 2048, 8192, 32768, 1 << 20):
            for rows in (1, 2, 3, 5, 64, 2047):
                blocks, rest = divmod(daf.daf_residual_norm_backward_workspace_bytes(rows * groups, cols, groups), cols * 5 * 4)
                assert rest == 0 and blocks % groups == 0
                assert blocks == groups or -(-cols // 32) * (4 + groups) * 1024 < 1 << 32


def test_products_fit_a_launch():
    """2^24 tiles of 256 threads each are refused, fewer are taken; and both gradients side by side are fewer too."""
    bf16 = torch.bfloat16
    for m, n, k in ((1 << 20, 1 << 19, 8), (1 << 23, 64, 1 << 17), (8, 1 << 19, 1 << 20)):
        assert daf.daf_gated_linear_workspace_bytes(m, n, k, bf16) == -1 == daf.daf_gated_linear_backward_workspace_bytes(m, n, k, bf16)
    for m, n, k in (((1 << 20) - 256, 1 << 19, 8), ((1 << 23) - 300, 64, 1 << 17), (8, (1 << 19) - 128, 1 << 20)):
        assert daf.daf_gated_linear_workspace_bytes(m, n, k, bf16) >= 0 and daf.daf_gated_linear_backward_workspace_bytes(m, n, k, bf16) > 0
        for product in block.GATED_PRODUCTS:
            s = daf.daf_gated_linear_schedule(m, n, k, product)
            assert s["whole_tiles"] < 1 << 24 and s["tiles"] * s["slices"] < 1 << 24


def test_norm_outputs_that_meet_something_else(lib):
    """Every output of the norms' calls against everything that a call reads or writes beside it, at its first and its last bytes."""
    rows, cols, groups = 6, 32, 3
    row_bytes, vector, gate_bytes = rows * cols * 4, cols * 4, groups * cols * 4
    tensors = {name: (P + i * BIG, row_bytes) for i, name in enumerate(("residual", "z", "out_residual", "out_y", "dy", "ds", "dr", "dz"))}
    vectors = {name: (P + (10 + i) * BIG, vector) for i, name in enumerate(("pre_weight", "pre_bias", "post_weight", "post_bias"))}
    vectors["gate"] = (P + 15 * BIG, gate_bytes)
    grads = {"grad_" + name: (P + (20 + i) * BIG, gate_bytes if name == "gate" else vector) for i, name in enumerate(vectors)}
    stats, ws = (P + 30 * BIG, rows * 16), (P + 31 * BIG, lib.daf_residual_norm_backward_workspace_bytes(rows, cols, groups))
    everything = {**tensors, **vectors, **grads, "stats": stats, "ws": ws}

    def forward(at):
        p = _norm(rows=rows, cols=cols, gate_groups=groups, post=1, **{name: at[name] for name in vectors})
        return lib.daf_residual_norm(ctypes.addressof(p), *(at[name] for name in ("residual", "z", "out_residual", "out_y", "stats")), None)

    def backward(at):
        p = _norm(rows=rows, cols=cols, gate_groups=groups, post=1, **{name: at[name] for name in vectors})
        g = block._ResidualNormGrads(**{name: at["grad_" + name] for name in vectors})
        return lib.daf_residual_norm_backward(ctypes.addressof(p), *(at[name] for name in ("out_residual", "z", "stats", "dy", "ds", "dr", "dz")),
                                              ctypes.addressof(g), at["ws"], None)

    forward_reads = ("residual", "z", *vectors)
    backward_reads = ("out_residual", "z", "stats", "dy", "ds", "pre_weight", "post_weight", "post_bias", "gate")
    same = {("out_residual", "residual"), ("out_residual", "z"), ("out_y", "residual"), ("out_y", "z"), ("dr", "dy"), ("dr", "ds"), ("dz", "dy"), ("dz", "ds"),
            ("dz", "z")}
    for call, outs, reads in ((forward, ("out_residual", "out_y", "stats"), forward_reads), (backward, ("dr", "dz", *grads, "ws"), backward_reads)):
        for out in outs:
            for other in (*reads, *(o for o in outs if o != out)):
                start, size = everything[other]
                own = everything[out][1]
                for at in {start, start + (size - 1) // 16 * 16, start - (own - 1) // 16 * 16}:
                    if at == start and (out, other) in same:
                        continue
                    places = {name: place for name, (place, _) in everything.items()}
                    places[out] = at
                    assert call(places) == EINVAL, (call.__name__, out, other, at - start)


def test_lists_that_are_no_gradients():
    """An array of something else is not taken for a list of gradients."""
    t, ws = torch.zeros(1), torch.zeros(daf.daf_grad_norm_workspace_bytes(), dtype=torch.uint8)
    for other in ((ctypes.c_int64 * 8)(), (block._ResidualNorm * 2)()):
        with pytest.raises(ValueError, match="items"):
            daf.daf_clip_grad_norm(other, 1.0, t, ws)
        with pytest.raises(ValueError, match="items"):
            daf.daf_grad_norm(other, t, ws)


def test_gradients_on_another_device():
    class OnDevice(torch.Tensor):                                         # what a tensor of a device says of itself
        is_cuda = True
        get_device = lambda self: 1

    elsewhere, ws = (block._GradItem * 1)(), torch.zeros(daf.daf_grad_norm_workspace_bytes(), dtype=torch.uint8)
    elsewhere.on_device = 0
    norm = torch.zeros(1).as_subclass(OnDevice)
    with pytest.raises(ValueError, match="gradients are on 0"):
        daf.daf_clip_grad_norm(elsewhere, 1.0, norm, ws)
    with pytest.raises(ValueError, match="gradients are on 0"):
        daf.daf_grad_norm(elsewhere, norm, ws)


def test_schedule_of_both_gradients():
    """Gradients that share a launch have tiles of one size and no whole rounds in front; each covers its output."""
    shared = 0
    for m, n, k in ((1, 1, 1), (1576, 2048, 768), (32768, 2048, 768), (8192, 11008, 4096), (4095, 75, 4090), (1731, 1365, 511), (40, 64, 4096)):
        both = [daf.daf_gated_linear_schedule(m, n, k, f"grad_{of}_of_both") for of in ("input", "weight")]
        alone = [daf.daf_gated_linear_schedule(m, n, k, f"grad_{of}") for of in ("input", "weight")]
        if both == alone:
            continue
        shared += 1
        assert both[0]["tile_rows"] == both[1]["tile_rows"] and both[0]["tile_cols"] == both[1]["tile_cols"]
        for s, rows, cols in zip(both, (m, 2 * -(-n // 64) * 64), (k, k)):
            assert s["whole_tiles"] == 0 and s["slices"] >= 1 and s["tiles"] == -(-rows // s["tile_rows"]) * -(-cols // s["tile_cols"])
    assert shared >= 3
    for bad in (-1, 5):
        assert block._library().daf_gated_linear_schedule(40, 64, 64, bad, ctypes.addressof(block._GatedSchedule())) == EINVAL

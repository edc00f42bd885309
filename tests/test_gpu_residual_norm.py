"""daf_residual_norm and its backward pass against the formulas in 64 bits.

Bounds: one rounding to the element's format, and binary32 arithmetic, of which every operation on the way may add 2^-24 of what it works on.
A value is at most 64 such operations deep (a thread's 32 columns or rows, the wave, the workgroup, the formula)."""
import itertools

import pytest
import torch

import paper_2507_07149_amd as daf
from tests.block_reference import TINY, UNIT, assert_within, residual_norm, residual_norm_backward

pytestmark = pytest.mark.gpu
DEPTH = 64 * 2.0 ** -24


def _data(rows, cols, dtype, groups, post, bias, seed):
    g = torch.Generator().manual_seed(seed)
    n = lambda *shape: torch.randn(*shape, generator=g, dtype=torch.float64).to(dtype)
    d = {"r": n(rows, cols) * 2 + 1, "z": n(rows, cols) + 3, "dy": n(rows, cols), "ds": n(rows, cols), "pre_w": 1 + n(cols) / 4, "pre_b": None,
         "post_w": None, "post_b": None, "gate": None}
    if bias:
        d["pre_b"] = n(cols)
    if post:
        d["post_w"], d["post_b"] = 1 + n(cols) / 4, n(cols) if bias else None
    if groups:
        d["gate"] = n(cols) if groups == 1 else n(groups, cols)
    return d


def _wide(t):
    return None if t is None else t.double()


def _check(rows, cols, dtype, kind, post, groups, bias, scale=0.75, eps=1e-5, seed=0):
    print("case", rows, cols, dtype, kind, post, groups, bias, flush=True)
    d = _data(rows, cols, dtype, groups, post, bias, seed)
    c = {k: None if v is None else v.cuda() for k, v in d.items()}
    w = {k: _wide(v) for k, v in d.items()}
    layer = kind == "layer"
    s, y = torch.full_like(c["r"], float("nan")), torch.full_like(c["r"], float("nan"))
    stats = torch.full((rows, 4), float("nan"), device="cuda")
    daf.daf_residual_norm(c["r"], y, stats, kind=kind, eps=eps, z=c["z"], out_residual=s, pre_weight=c["pre_w"], pre_bias=c["pre_b"], post=post,
                          post_weight=c["post_w"], post_bias=c["post_b"], gate=c["gate"], scale=scale)
    ws, wy, wstats, size, size_y = residual_norm(w["r"], w["z"], layer, eps, post, w["pre_w"], w["pre_b"], w["post_w"], w["post_b"], w["gate"], scale)
    u = UNIT[dtype]
    assert_within(s, ws, u * ws.abs() + DEPTH * size + TINY[dtype], "sum")
    assert_within(y, wy, u * wy.abs() + DEPTH * size_y + TINY[dtype], "y")
    row_size = torch.stack([w["z"].abs().amax(1), wstats[:, 1] * (1 + w["z"].abs().amax(1) * wstats[:, 1]), size.amax(1),
                            wstats[:, 3] * (1 + size.amax(1) * wstats[:, 3])], 1) if rows else wstats
    assert_within(stats, wstats, DEPTH * row_size, "stats")

    outs = {"residual": torch.full_like(s, float("nan")), "z": torch.full_like(s, float("nan"))}
    vector = lambda *shape: torch.full(shape, float("nan"), device="cuda")
    outs["pre_weight"], outs["pre_bias"] = vector(cols), vector(cols) if bias else None
    outs["post_weight"], outs["post_bias"] = (vector(cols) if post else None), (vector(cols) if post and bias else None)
    outs["gate"] = vector(*d["gate"].shape) if groups else None
    ws_bytes = daf.daf_residual_norm_backward_workspace_bytes(rows, cols, max(groups, 1))
    workspace = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    daf.daf_residual_norm_backward(s, c["dy"], stats, outs["residual"], workspace, kind=kind, z=c["z"], grad_residual=c["ds"], out_grad_z=outs["z"],
                                   pre_weight=c["pre_w"], post=post, post_weight=c["post_w"], post_bias=c["post_b"], gate=c["gate"], scale=scale,
                                   out_grad_pre_weight=outs["pre_weight"], out_grad_pre_bias=outs["pre_bias"],
                                   out_grad_post_weight=outs["post_weight"], out_grad_post_bias=outs["post_bias"], out_grad_gate=outs["gate"])
    want, size = residual_norm_backward(s.cpu().double(), w["z"], stats.cpu().double(), w["dy"], w["ds"], layer, post, w["pre_w"], w["post_w"],
                                        w["post_b"], w["gate"], scale)
    for name, got in outs.items():
        if got is None:
            continue
        rounding = u * want[name].abs() + TINY[dtype] if name in ("residual", "z") else 0.0
        # (a row's means are as large as its largest parts)
        bound = size[name] + size[name].amax(-1, keepdim=True) if name in ("residual", "z") and rows else size[name]
        assert_within(got.reshape(want[name].shape), want[name], rounding + DEPTH * bound, "gradient of " + name)


SHAPES = [(1, 1), (3, 7), (5, 64), (9, 512), (6, 513), (7, 1001), (2, 1024), (5, 1025), (130, 768), (3, 2048), (2, 2055), (3, 4096), (2, 5003),
          (2, 8192), (3, 8193), (2, 11008), (1, 16384), (2, 16383)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_lengths(rows, cols, dtype):
    _check(rows, cols, dtype, "layer", True, 1, True)
    _check(rows, cols, dtype, "rms", False, 0, False, seed=1)


@pytest.mark.parametrize("kind,post,groups,bias", itertools.product(["rms", "layer"], [False, True], [0, 1, 6], [False, True]))
def test_forms(kind, post, groups, bias):
    for dtype, (rows, cols) in ((torch.bfloat16, (60, 200)), (torch.float32, (18, 1500)), (torch.float16, (24, 4100)), (torch.float32, (6, 9000))):
        _check(rows, cols, dtype, kind, post, groups, bias, seed=2)


@pytest.mark.parametrize("rows,groups", [(4100, 1), (4099, 4099), (6000, 3), (3000, 1500)])
def test_many_rows(rows, groups):
    """Chunks of several rows, and runs that do not fill one."""
    _check(rows, 96, torch.bfloat16, "layer", True, groups, True)
    _check(rows, 1100, torch.float32, "rms", True, groups, False)


def test_no_rows():
    empty = torch.empty(0, 40, device="cuda", dtype=torch.bfloat16)
    daf.daf_residual_norm(empty, empty.clone(), torch.empty(0, 4, device="cuda"), z=empty.clone(), out_residual=empty.clone())
    w, gate = torch.full((40,), 5.0, device="cuda"), torch.full((2, 40), 5.0, device="cuda")
    daf.daf_residual_norm_backward(empty, empty.clone(), torch.empty(0, 4, device="cuda"), empty.clone(), None, z=empty.clone(),
                                   gate=torch.ones(2, 40, device="cuda", dtype=torch.bfloat16), out_grad_z=empty.clone(), out_grad_pre_weight=w,
                                   out_grad_gate=gate)
    assert torch.equal(w, torch.zeros_like(w)) and torch.equal(gate, torch.zeros_like(gate))


def _forward(c, s, y, stats, **more):
    daf.daf_residual_norm(c["r"], y, stats, kind="layer", z=c["z"], out_residual=s, pre_weight=c["pre_w"], post=True, post_weight=c["post_w"], **more)


@pytest.mark.parametrize("cols,dtype", [(768, torch.bfloat16), (3333, torch.float32), (10000, torch.float16), (6000, torch.float32), (9000, torch.float32)])
def test_in_place(cols, dtype):
    """Outputs that are inputs hold what other outputs would."""
    c = {k: None if v is None else v.cuda() for k, v in _data(70, cols, dtype, 0, True, False, 3).items()}
    s, y, stats = torch.empty_like(c["r"]), torch.empty_like(c["r"]), torch.empty(70, 4, device="cuda")
    _forward(c, s, y, stats)
    for first in ("r", "z"):
        e = {k: None if v is None else v.clone() for k, v in c.items()}
        other = "z" if first == "r" else "r"
        _forward(e, e[first], e[other], torch.empty_like(stats))
        assert torch.equal(e[first], s) and torch.equal(e[other], y)
    ws = torch.empty(daf.daf_residual_norm_backward_workspace_bytes(70, cols), dtype=torch.uint8, device="cuda")

    def backward(e, to_r, to_z):
        w = torch.empty(cols, device="cuda")
        daf.daf_residual_norm_backward(s, e["dy"], stats, to_r, ws, kind="layer", z=e["z"], grad_residual=e["ds"], out_grad_z=to_z, pre_weight=e["pre_w"],
                                       post=True, post_weight=e["post_w"], out_grad_post_weight=w)
        return w

    dr, dz = torch.empty_like(s), torch.empty_like(s)
    w = backward(c, dr, dz)
    for to_r, to_z in (("dy", "ds"), ("ds", "dy"), ("ds", "z"), ("dy", "z")):
        e = {k: None if v is None else v.clone() for k, v in c.items()}
        assert torch.equal(backward(e, e[to_r], e[to_z]), w) and torch.equal(e[to_r], dr) and torch.equal(e[to_z], dz)


@pytest.mark.parametrize("cols", [200, 3000, 9001])
def test_parts_left_out(cols):
    """The norm alone, the sum alone, gradients of one of the two outputs alone."""
    for dtype in (torch.float32, torch.bfloat16):
        d = _data(33, cols, dtype, 1, True, False, 4)
        c = {k: None if v is None else v.cuda() for k, v in d.items()}
        w = {k: _wide(v) for k, v in d.items()}
        u = UNIT[dtype]
        y, stats = torch.empty_like(c["r"]), torch.empty(33, 4, device="cuda")
        daf.daf_residual_norm(c["r"], y, stats)
        _, wy, wstats, _, size_y = residual_norm(w["r"], None, False, 1e-5, False, None, None, None, None, None, 1.0)
        assert_within(y, wy, u * wy.abs() + DEPTH * size_y, "y")
        s = torch.empty_like(c["r"])
        daf.daf_residual_norm(c["r"], None, z=c["z"], out_residual=s, gate=c["gate"], scale=0.5)
        ws_, _, _, size, _ = residual_norm(w["r"], w["z"], False, 1e-5, False, None, None, None, None, w["gate"], 0.5)
        assert_within(s, ws_, u * ws_.abs() + DEPTH * size, "sum")
        dr, dz = torch.empty_like(s), torch.empty_like(s)
        daf.daf_residual_norm_backward(c["r"], c["dy"], stats, dr)
        want, size = residual_norm_backward(w["r"], None, stats.cpu().double(), w["dy"], None, False, False, None, None, None, None, 1.0)
        assert_within(dr, want["residual"], u * want["residual"].abs() + DEPTH * 2 * size["residual"].amax(-1, keepdim=True), "gradient of the norm alone")
        daf.daf_residual_norm_backward(None, None, stats, dr, z=c["z"], out_grad_z=dz, grad_residual=c["ds"], gate=c["gate"], scale=0.5)
        want, size = residual_norm_backward(None, w["z"], stats.cpu().double(), None, w["ds"], False, False, None, None, None, w["gate"], 0.5)
        assert torch.equal(dr, c["ds"])
        assert_within(dz, want["z"], u * want["z"].abs() + DEPTH * size["z"], "gradient of z")


def test_rows_of_nan_and_infinity_stay_alone():
    for dtype, cols in ((torch.float32, 300), (torch.bfloat16, 5000)):
        c = {k: None if v is None else v.cuda() for k, v in _data(9, cols, dtype, 0, True, False, 5).items()}
        s, y, stats = torch.empty_like(c["r"]), torch.empty_like(c["r"]), torch.empty(9, 4, device="cuda")
        _forward(c, s, y, stats)
        c["z"][3, 7], c["r"][5, 1] = float("nan"), float("inf")
        s2, y2 = torch.empty_like(s), torch.empty_like(y)
        _forward(c, s2, y2, stats)
        rest = [0, 1, 2, 4, 6, 7, 8]
        assert torch.equal(s2[rest], s[rest]) and torch.equal(y2[rest], y[rest])
        assert s2[3].isnan().all() and y2[3].isnan().all() and s2[5, 1] == float("inf") and torch.equal(s2[5, 2:], s[5, 2:]) and y2[5].isnan().all()


def test_large_offsets_and_small_spread():
    """A row far from zero: its variance is not lost in the square of its mean (a spread of 1 at 1000, within what binary32 holds of the row)."""
    r = (1000 + torch.randn(40, 3001, generator=torch.Generator().manual_seed(6), dtype=torch.float64)).float().cuda()
    y, stats = torch.empty_like(r), torch.empty(40, 4, device="cuda")
    daf.daf_residual_norm(r, y, stats, kind="layer")
    _, wy, wstats, _, _ = residual_norm(r.cpu().double(), None, True, 1e-5, False, None, None, None, None, None, 1.0)
    # the mean is off by a few roundings of 1000, which shifts all of the row by that; its square is added to the variance, not its product
    assert_within(stats[:, 2], wstats[:, 2], torch.tensor(8 * 1000 * 2.0 ** -24), "mean")
    assert_within(stats[:, 3], wstats[:, 3], torch.tensor(64 * 2.0 ** -24), "rstd")
    assert_within(y, wy, 10 * 1000 * 2.0 ** -24 + 64 * 2.0 ** -24 * wy.abs(), "y")


def test_gradient_against_differences():
    """Central differences of sum(y * dy + s * ds) along a random direction, in binary32 with steps of 2^-6: the third derivative's part is
    below 2^-12 of the terms, a binary32 output's error over the step 2^-17 of them."""
    rows, cols = 12, 700
    c = {k: None if v is None else v.cuda() for k, v in _data(rows, cols, torch.float32, 3, True, True, 7).items()}
    g = torch.Generator().manual_seed(8)
    names = {"r": "residual", "z": "z", "pre_w": "pre_weight", "pre_b": "pre_bias", "post_w": "post_weight", "post_b": "post_bias", "gate": "gate"}
    stats = torch.empty(rows, 4, device="cuda")

    def loss(c):
        s, y = torch.empty_like(c["r"]), torch.empty_like(c["r"])
        daf.daf_residual_norm(c["r"], y, stats, kind="layer", z=c["z"], out_residual=s, pre_weight=c["pre_w"], pre_bias=c["pre_b"], post=True,
                              post_weight=c["post_w"], post_bias=c["post_b"], gate=c["gate"], scale=0.5)
        return s, (y.double() * c["dy"].double() + s.double() * c["ds"].double())

    s, terms = loss(c)
    outs = {n: torch.empty(c[k].shape, device="cuda") for k, n in names.items()}
    ws = torch.empty(daf.daf_residual_norm_backward_workspace_bytes(rows, cols, 3), dtype=torch.uint8, device="cuda")
    daf.daf_residual_norm_backward(s, c["dy"], stats, outs["residual"], ws, kind="layer", z=c["z"], grad_residual=c["ds"], out_grad_z=outs["z"],
                                   pre_weight=c["pre_w"], post=True, post_weight=c["post_w"], post_bias=c["post_b"], gate=c["gate"], scale=0.5,
                                   **{"out_grad_" + n: outs[n] for n in names.values() if n not in ("residual", "z")})
    h = 2.0 ** -6
    for k, n in names.items():
        direction = torch.randn(c[k].shape, generator=g).cuda()
        plus, minus = dict(c), dict(c)
        plus[k], minus[k] = c[k] + h * direction, c[k] - h * direction
        difference = (loss(plus)[1] - loss(minus)[1]) / (2 * h)
        slope = (outs[n].double() * direction.double()).sum()
        assert abs(difference.sum() - slope) <= 2.0 ** -10 * difference.abs().sum(), n


def test_graph_and_other_stream():
    c = {k: None if v is None else v.cuda() for k, v in _data(257, 1500, torch.bfloat16, 0, True, False, 9).items()}
    s, y, stats = torch.empty_like(c["r"]), torch.empty_like(c["r"]), torch.empty(257, 4, device="cuda")
    dr, dz, w = torch.empty_like(s), torch.empty_like(s), torch.empty(1500, device="cuda")
    ws = torch.empty(daf.daf_residual_norm_backward_workspace_bytes(257, 1500), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        _forward(c, s, y, stats, stream=stream)
        daf.daf_residual_norm_backward(s, c["dy"], stats, dr, ws, kind="layer", z=c["z"], grad_residual=c["ds"], out_grad_z=dz, pre_weight=c["pre_w"],
                                       post=True, post_weight=c["post_w"], out_grad_post_weight=w, stream=stream)

    outs = (s, y, stats, dr, dz, w)
    step()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    for t in outs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("rows,cols,groups", [(32768, 4096, 32768), (8192, 16384, 8192), (16386, 8200, 8193)])
def test_a_gate_row_for_every_row_or_two(rows, cols, groups):
    """As many rows of the gate as rows, and longest rows: the gate's gradient is scale * grad_s * z, exact in binary32 for bfloat16 factors and one
    row; two rows add up with one rounding."""
    print("case", rows, cols, groups, flush=True)
    g = torch.Generator(device="cuda").manual_seed(10)
    n = lambda *shape: torch.randn(*shape, generator=g, device="cuda").bfloat16()
    z, ds, gate = n(rows, cols), n(rows, cols), n(groups, cols)
    dr, dz = torch.empty_like(z), torch.empty_like(z)
    grad = torch.full((groups, cols), float("nan"), device="cuda")
    stats = torch.zeros(rows, 4, device="cuda")
    ws = torch.full((daf.daf_residual_norm_backward_workspace_bytes(rows, cols, groups),), 255, dtype=torch.uint8, device="cuda")
    daf.daf_residual_norm_backward(None, None, stats, dr, ws, z=z, grad_residual=ds, out_grad_z=dz, gate=gate, scale=0.5, out_grad_gate=grad)
    want = (0.5 * ds.float() * z.float()).view(groups, rows // groups, cols).sum(1)
    assert torch.equal(grad, want) and torch.equal(dr, ds)


def test_no_rows_and_more_gradients_than_threads_in_a_launch():
    groups, cols = 1 << 20, 4100                         # more than 2^32 elements
    empty = torch.empty(0, cols, device="cuda", dtype=torch.bfloat16)
    gate, grad = torch.empty(groups, cols, device="cuda", dtype=torch.bfloat16), torch.full((groups, cols), 5.0, device="cuda")
    daf.daf_residual_norm_backward(empty, empty.clone(), torch.empty(0, 4, device="cuda"), empty.clone(), None, z=empty.clone(), gate=gate,
                                   out_grad_z=empty.clone(), out_grad_gate=grad)
    assert all(not part.any() for part in grad.split(1 << 16))
    del gate, grad
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(9, 5), (5, 40), (6, 1001), (3, 5000), (3, 9000)])
def test_constant_rows_far_from_zero(rows, cols, dtype):
    """A row of one value everywhere is its bias after a layer norm, whatever the value: 2^114 gives what 1 gives, forward and backward, though the mean
    times 1 / deviation, 2^114 * 10^5, is beyond binary32 (the row's sum is not)."""
    d = {k: None if v is None else v.cuda() for k, v in _data(rows, cols, dtype, 1, True, True, 11).items()}
    results = []
    for value in (1.0, 2.0 ** 114):
        flat = torch.full_like(d["z"], value)
        s, y, dr, dz = (torch.empty_like(flat) for _ in range(4))
        stats, ws = torch.empty(rows, 4, device="cuda"), torch.empty(daf.daf_residual_norm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        daf.daf_residual_norm(d["r"], y, stats, kind="layer", eps=1e-10, z=flat, out_residual=s, pre_weight=d["pre_w"], pre_bias=d["pre_b"], post=True,
                              post_weight=d["post_w"], post_bias=d["post_b"], gate=d["gate"])
        assert (stats[:, 0] == value).all() and (stats[:, 1] - 1e5).abs().max() < 1.0
        stats[:, 2:] = stats[:, :2]                                       # as if the sum were as flat
        vectors = [torch.empty(cols, device="cuda") for _ in range(5)]
        daf.daf_residual_norm_backward(flat, d["dy"], stats, dr, ws, kind="layer", z=flat, grad_residual=d["ds"], out_grad_z=dz, pre_weight=d["pre_w"], post=True,
                                       post_weight=d["post_w"], post_bias=d["post_b"], gate=d["gate"], out_grad_pre_weight=vectors[0],
                                       out_grad_pre_bias=vectors[1], out_grad_post_weight=vectors[2], out_grad_post_bias=vectors[3],
                                       out_grad_gate=vectors[4])
        results.append((s, y, dr, dz, *vectors))
        assert all(t.isfinite().all() for t in results[-1]), value
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes and 2^31 elements to a tensor: the last rows are what they are alone."""
    rows, cols, last = (1 << 19) + 77, 4104, 33
    g = torch.Generator(device="cuda").manual_seed(12)
    d = {name: torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda") for name in ("r", "z", "dy", "ds")}
    for t in d.values():
        t[-last:] = torch.randn(last, cols, generator=g, device="cuda").bfloat16()
    weight = torch.randn(cols, generator=g, device="cuda").bfloat16()
    results = []
    for at in (0, rows - last):
        c = {name: t[at:].clone() if at else t for name, t in d.items()}           # (their own allocation: rows of 4104 begin anywhere)
        n = rows - at
        s, y, dr, dz = (torch.empty_like(c["r"]) for _ in range(4))
        stats, grad = torch.empty(n, 4, device="cuda"), torch.empty(cols, device="cuda")
        ws = torch.empty(daf.daf_residual_norm_backward_workspace_bytes(n, cols), dtype=torch.uint8, device="cuda")
        daf.daf_residual_norm(c["r"], y, stats, kind="layer", z=c["z"], out_residual=s, pre_weight=weight, post=True, post_weight=weight)
        daf.daf_residual_norm_backward(s, c["dy"], stats, dr, ws, kind="layer", z=c["z"], grad_residual=c["ds"], out_grad_z=dz, pre_weight=weight, post=True,
                                       post_weight=weight, out_grad_pre_weight=grad)
        results.append([t[-last:].clone() for t in (s, y, dr, dz)] + [grad])
    (*whole, grad), (*alone, grad_alone) = results
    assert all(torch.equal(a, b) for a, b in zip(whole, alone))
    assert_within(grad, grad_alone.double(), DEPTH * (d["dy"][-last:].double().abs().sum(0) * 8).cpu(), "gradient of pre_weight")
    del d, c, s, y, dr, dz
    torch.cuda.empty_cache()

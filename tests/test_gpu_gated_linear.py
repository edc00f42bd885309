"""daf_gated_linear and its backward pass against the formulas in 64 bits.

Bounds: a sum of L products on the matrix cores is off by at most 2 (L / 16 + 32) 2^-24 of the sum of the products' sizes (16 products to an
instruction, one rounding of the running sum each, a factor of two for how the instruction adds its 16 up); the activation and its slope by 32
roundings of binary32 of their argument's size, and by 1.2 times (silu, gelu: the largest slopes and curvatures are below 1.2) what the argument is
off; every rounding to the format by half of its last place."""
import pytest
import torch

import paper_2507_07149_amd as daf
from tests.block_reference import TINY, UNIT, activation, assert_within

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
EPS = 2.0 ** -24


def _sum_error(length):
    return 2 * (length / 16 + 32) * EPS


def _data(m, n, k, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *shape: torch.randn(*shape, generator=g, dtype=torch.float64)
    return {"x": r(m, k).to(dtype), "wg": (r(n, k) / k ** 0.5).to(dtype), "wu": (r(n, k) / k ** 0.5).to(dtype), "gh": r(m, n).to(dtype)}


def _workspace(m, n, k, dtype, backward):
    size = daf.daf_gated_linear_backward_workspace_bytes if backward else daf.daf_gated_linear_workspace_bytes
    return torch.full((max(size(m, n, k, dtype), 16),), 255, dtype=torch.uint8, device="cuda")       # NaN in either format


def _nan(*shape, dtype):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


class _Expected:
    """Values and bounds of one case; a and u as computed from x, or as given (exact then)."""

    def __init__(self, d, act, dtype, kept=None):
        x, wg, wu, gh = (d[name].double() for name in ("x", "wg", "wu", "gh"))
        m, k = x.shape
        n, unit, tiny = wg.shape[0], UNIT[dtype], TINY[dtype]
        if kept is None:
            a, u = x @ wg.t(), x @ wu.t()
            ea, eu = (_sum_error(k) * (x.abs() @ w.abs().t()) for w in (wg, wu))
        else:
            a, u = (t.double() for t in kept)
            ea = eu = torch.zeros_like(a)
        f, slope = activation(a, act)
        # a jump of relu's slope within the error of a is not the kernel's
        jump = (a.abs() <= ea).double() if act == "relu" else 0.0
        ef = 1.2 * ea + 32 * EPS * a.abs()
        eslope = 1.2 * ea + 32 * EPS * (1 + a.abs()) + jump
        self.a, self.u, self.h = a, u, f * u
        self.bound_a, self.bound_u = (unit * t.abs() + e + tiny for t, e in ((a, ea), (u, eu)))
        eh = ef * u.abs() + f.abs() * eu + ef * eu + 2 * EPS * self.h.abs()
        self.bound_h = unit * self.h.abs() + (1 + unit) * eh + tiny
        da, du = gh * u * slope, gh * f
        eda = gh.abs() * (u.abs() * eslope + eu * (slope.abs() + eslope)) + 3 * EPS * da.abs()
        edu = gh.abs() * ef + 2 * EPS * du.abs()
        eda, edu = (unit * t.abs() + (1 + unit) * e + tiny for t, e in ((da, eda), (du, edu)))
        self.dx = da @ wg + du @ wu
        self.bound_dx = (1 + unit) * ((eda @ wg.abs() + edu @ wu.abs()) + _sum_error(2 * n + 128) * ((da.abs() + eda) @ wg.abs() + (du.abs() + edu) @ wu.abs()))
        self.bound_dx += unit * self.dx.abs() + tiny
        self.dw = [t.t() @ x for t in (da, du)]
        self.bound_dw = [(1 + unit) * (e.t() @ x.abs() + _sum_error(m) * ((t.abs() + e).t() @ x.abs())) + unit * w.abs() + tiny
                         for t, e, w in ((da, eda, self.dw[0]), (du, edu, self.dw[1]))]


def _backward(c, act, dtype, kept=(None, None), h=False, want="xw"):
    m, k = c["x"].shape
    n = c["wg"].shape[0]
    out = {"h": _nan(m, n, dtype=dtype) if h else None, "dx": _nan(m, k, dtype=dtype) if "x" in want else None,
           "dwg": _nan(n, k, dtype=dtype) if "w" in want else None, "dwu": _nan(n, k, dtype=dtype) if "w" in want else None}
    daf.daf_gated_linear_backward(c["x"], c["wg"], c["wu"], c["gh"], act, out["dx"], out["dwg"], out["dwu"], _workspace(m, n, k, dtype, True),
                                  gate=kept[0], up=kept[1], out_h=out["h"])
    return out


def _check(m, n, k, dtype, act="silu", seed=0):
    print("case", m, n, k, dtype, act, flush=True)
    d = _data(m, n, k, dtype, seed)
    c = {name: t.cuda() for name, t in d.items()}
    e = _Expected(d, act, dtype)
    h, a, u = (_nan(m, n, dtype=dtype) for _ in range(3))
    daf.daf_gated_linear(c["x"], c["wg"], c["wu"], act, h, _workspace(m, n, k, dtype, False), out_gate=a, out_up=u)
    assert_within(h, e.h, e.bound_h, "h")
    assert_within(a, e.a, e.bound_a, "a")
    assert_within(u, e.u, e.bound_u, "u")
    alone = _nan(m, n, dtype=dtype)
    daf.daf_gated_linear(c["x"], c["wg"], c["wu"], act, alone, _workspace(m, n, k, dtype, False))
    assert torch.equal(alone, h)

    got = _backward(c, act, dtype, h=True)
    assert torch.equal(got["h"], h)
    kept = _backward(c, act, dtype, (a, u))
    for out, e in ((got, e), (kept, _Expected(d, act, dtype, (a.cpu(), u.cpu())))):
        assert_within(out["dx"], e.dx, e.bound_dx, "grad_x")
        assert_within(out["dwg"], e.dw[0], e.bound_dw[0], "grad_w_gate")
        assert_within(out["dwu"], e.dw[1], e.bound_dw[1], "grad_w_up")
    # one gradient alone (its sums may be cut in other places)
    x_alone, w_alone = _backward(c, act, dtype, want="x"), _backward(c, act, dtype, want="w")
    e = _Expected(d, act, dtype)
    assert_within(x_alone["dx"], e.dx, e.bound_dx, "grad_x alone")
    assert_within(w_alone["dwg"], e.dw[0], e.bound_dw[0], "grad_w_gate alone")
    assert_within(w_alone["dwu"], e.dw[1], e.bound_dw[1], "grad_w_up alone")
    again = _backward(c, act, dtype, h=True)
    assert all(torch.equal(again[name], got[name]) for name in got)


# one token, a few, parts of a tile and a little more than whole ones; widths of one column, odd ones, whole tiles and steps
SIZES = [(1, 1, 1), (1, 64, 64), (2, 3, 5), (1, 129, 320), (7, 65, 8), (16, 130, 72), (31, 64, 65), (33, 66, 127), (64, 128, 128), (65, 127, 129), (100, 200, 191),
         (129, 63, 192), (128, 256, 256), (257, 192, 64), (300, 257, 136), (190, 512, 511), (513, 70, 96)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_sizes(m, n, k, dtype):
    _check(m, n, k, dtype)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("m,n,k", [(40, 72, 80), (130, 200, 33)])
def test_activations(act, m, n, k):
    _check(m, n, k, BF16, act, seed=1)
    _check(m, n, k, F16, act, seed=2)


@pytest.mark.parametrize("m,n,k", [(1, 2048, 1024), (3, 1000, 2000), (40, 64, 4096), (64, 700, 1000), (2000, 96, 64), (3000, 33, 40), (1100, 640, 520)])
def test_long_sums_and_many_tiles(m, n, k):
    """Sums over few tiles are cut into slices; tiles of every size."""
    _check(m, n, k, BF16, seed=3)


@pytest.mark.parametrize("m,n,k,product", [(4000, 2017, 100, "forward"), (4096, 2048, 64, "forward"), (4095, 75, 4090, "grad_input"), (90, 2040, 4090, "grad_weight"),
                                           (200, 2048, 4001, "grad_weight")])
def test_largest_tiles(m, n, k, product):
    assert daf.daf_gated_linear_schedule(m, n, k, product)["tile_rows"] == 256
    _check(m, n, k, BF16, seed=9)


@pytest.mark.parametrize("m,n,k,tile", [(1, 4100, 520, (16, 32)), (5, 37, 7, (16, 16)), (9, 50, 31, (16, 16)), (16, 4090, 33, (16, 32)), (17, 4065, 300, (32, 32)),
                                        (32, 300, 1031, (32, 16)), (3, 5000, 4, (16, 32)), (2, 64, 9001, (16, 16))])
def test_few_rows(m, n, k, tile):
    """Rows that begin at any element, whole instructions and the rest, fewer values than a load has, columns that do not fill a workgroup."""
    how = daf.daf_gated_linear_schedule(m, n, k, "forward")
    assert (how["tile_rows"], how["tile_cols"]) == tile and daf.daf_gated_linear_workspace_bytes(m, n, k, BF16) == 0
    _check(m, n, k, BF16, "gelu", seed=10)
    _check(m, n, k, F16, "silu", seed=11)


@pytest.mark.parametrize("m,n,k", [(5, 45, 39), (20, 4050, 6)])
def test_few_rows_touch_nothing_outside(m, n, k):
    d = _data(m, n, k, BF16, 12)
    c = {}
    for name, t in d.items():
        whole = torch.full((t.numel() + 2048,), float("nan"), dtype=BF16, device="cuda")
        c[name] = whole[1024:1024 + t.numel()].view(t.shape)
        c[name].copy_(t)
    outs = [torch.full((m * n + 2048,), 3.0, dtype=BF16, device="cuda") for _ in range(3)]
    h, a, u = (t[1024:1024 + m * n].view(m, n) for t in outs)
    daf.daf_gated_linear(c["x"], c["wg"], c["wu"], "silu", h, out_gate=a, out_up=u)
    e = _Expected(d, "silu", BF16)
    assert_within(h, e.h, e.bound_h, "h")
    for whole in outs:
        assert (whole[:1024] == 3.0).all() and (whole[-1024:] == 3.0).all() and whole.isfinite().all()


def test_no_rows():
    w = torch.ones(5, 6, device="cuda", dtype=BF16)
    x, gh = torch.empty(0, 6, device="cuda", dtype=BF16), torch.empty(0, 5, device="cuda", dtype=BF16)
    daf.daf_gated_linear(x, w, w, "silu", gh)
    a, b = w.clone(), w.clone()
    daf.daf_gated_linear_backward(x, w, w, gh, "silu", x.clone(), a, b, torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert not a.any() and not b.any()


def test_nothing_outside_is_touched():
    """Outputs in the middle of a larger buffer, odd sizes: what lies around them stays as it is, and NaN around the inputs does not get in."""
    m, n, k = 67, 45, 39
    d = _data(m, n, k, BF16, 4)

    def framed(shape, fill):
        size = shape[0] * shape[1]
        whole = torch.full((size + 2048,), fill, dtype=BF16, device="cuda")
        return whole, whole[1024:1024 + size].view(shape)

    c = {}
    for name, t in d.items():
        _, c[name] = framed(t.shape, float("nan"))
        c[name].copy_(t)
    outs = {"h": framed((m, n), 3.0), "dx": framed((m, k), 3.0), "dwg": framed((n, k), 3.0), "dwu": framed((n, k), 3.0)}
    daf.daf_gated_linear(c["x"], c["wg"], c["wu"], "silu", outs["h"][1], _workspace(m, n, k, BF16, False))
    daf.daf_gated_linear_backward(c["x"], c["wg"], c["wu"], c["gh"], "silu", outs["dx"][1], outs["dwg"][1], outs["dwu"][1], _workspace(m, n, k, BF16, True))
    e = _Expected(d, "silu", BF16)
    for name, want, bound in (("h", e.h, e.bound_h), ("dx", e.dx, e.bound_dx), ("dwg", e.dw[0], e.bound_dw[0]), ("dwu", e.dw[1], e.bound_dw[1])):
        whole, inside = outs[name]
        assert_within(inside, want, bound, name)
        assert (whole[:1024] == 3.0).all() and (whole[-1024:] == 3.0).all(), name


def test_rows_of_nan_and_infinity_stay_alone():
    m, n, k = 70, 80, 72
    d = _data(m, n, k, BF16, 5)
    c = {name: t.cuda() for name, t in d.items()}
    run = lambda: (_backward(c, "silu", BF16, h=True), _nan(m, n, dtype=BF16))
    clean, _ = run()
    c["x"][11, 3], c["x"][40, 71] = float("nan"), float("inf")
    got, h = run()
    daf.daf_gated_linear(c["x"], c["wg"], c["wu"], "silu", h, _workspace(m, n, k, BF16, False))
    rest = [i for i in range(m) if i not in (11, 40)]
    assert torch.equal(h[rest], clean["h"][rest]) and torch.equal(got["dx"][rest], clean["dx"][rest]) and h[11].isnan().all()
    assert not h[40].isfinite().any() and got["dwg"].isnan().all()


def test_large_arguments():
    """Far out the activations and slopes are 0 or 1 times their factors, without NaN."""
    for dtype, big in ((BF16, 3e4), (F16, 100.0)):
        x = torch.tensor([[1.0], [-1.0], [0.0]], dtype=dtype, device="cuda")
        wg, wu = torch.full((4, 1), big, dtype=dtype, device="cuda"), torch.full((4, 1), 0.5, dtype=dtype, device="cuda")
        for act in ("silu", "gelu", "gelu_tanh", "relu"):
            c = {"x": x, "wg": wg, "wu": wu, "gh": torch.ones(3, 4, dtype=dtype, device="cuda")}
            got = _backward(c, act, dtype, h=True)
            a = x.double() @ wg.double().t()
            want = a.clamp(min=0) * (x.double() @ wu.double().t())
            assert_within(got["h"], want.cpu(), 2 * UNIT[dtype] * want.cpu().abs() + TINY[dtype], act)
            assert all(got[name].isfinite().all() for name in ("dx", "dwg", "dwu")), act


def test_gradient_against_differences():
    """Central differences of sum(h * gh) along random directions.  h is rounded to binary16: with steps of 2^-5 its error over the step is below 2^-6 of
    each term, and random over the terms; the third derivative's part below 2^-8."""
    m, n, k = 60, 70, 48
    c = {name: t.cuda() for name, t in _data(m, n, k, F16, 6).items()}
    got = _backward(c, "gelu", F16)

    def loss(c):
        h = _nan(m, n, dtype=F16)
        daf.daf_gated_linear(c["x"], c["wg"], c["wu"], "gelu", h, _workspace(m, n, k, F16, False))
        return h.double() * c["gh"].double()

    g = torch.Generator().manual_seed(7)
    for name, grad in (("x", "dx"), ("wg", "dwg"), ("wu", "dwu")):
        direction = (torch.randint(0, 2, c[name].shape, generator=g).double() * 2 - 1).cuda() * (1.0 if name == "x" else k ** -0.5)
        plus, minus = dict(c), dict(c)
        plus[name] = (c[name].double() + 2.0 ** -5 * direction).half()
        minus[name] = (c[name].double() - 2.0 ** -5 * direction).half()
        moved = plus[name].double() - minus[name].double()                 # the steps as binary16 has them
        difference = loss(plus) - loss(minus)
        slope = (got[grad].double() * moved).sum()
        assert abs(difference.sum() - slope) <= 2.0 ** -6 * difference.abs().sum(), name


def test_same_bits_graph_and_other_stream():
    m, n, k = 333, 200, 1001
    c = {name: t.cuda() for name, t in _data(m, n, k, BF16, 8).items()}
    h, a, u = (_nan(m, n, dtype=BF16) for _ in range(3))
    dx, dwg, dwu = _nan(m, k, dtype=BF16), _nan(n, k, dtype=BF16), _nan(n, k, dtype=BF16)
    fw, bw = _workspace(m, n, k, BF16, False), _workspace(m, n, k, BF16, True)

    def step(stream=None):
        daf.daf_gated_linear(c["x"], c["wg"], c["wu"], "silu", h, fw, out_gate=a, out_up=u, stream=stream)
        daf.daf_gated_linear_backward(c["x"], c["wg"], c["wu"], c["gh"], "silu", dx, dwg, dwu, bw, stream=stream)

    outs = (h, a, u, dx, dwg, dwu)
    step()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        for t in outs + (fw, bw):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(outs, want))
    for t in outs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(outs, want))


def test_no_rows_and_more_elements_than_threads_in_a_launch():
    n, k = 1 << 17, (1 << 15) + 8                        # more than 2^32 elements of a weight
    w = torch.empty(n, k, device="cuda", dtype=BF16)
    x, gh = torch.empty(0, k, device="cuda", dtype=BF16), torch.empty(0, n, device="cuda", dtype=BF16)
    a, b = (torch.full((n, k), 5.0, device="cuda", dtype=BF16) for _ in range(2))
    daf.daf_gated_linear_backward(x, w, w, gh, "silu", x.clone(), a, b, torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert all(not part.any() for t in (a, b) for part in t.split(1 << 13))
    del w, a, b
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m,n,k", [(70, 45, 39), (9, 45, 39), (500, 300, 72), (4000, 2017, 100)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_infinity_goes_through_the_gradients(m, n, k, dtype):
    """relu, weights and gradients above zero: an infinite input makes its row of a, u, da, du and grad_x +infinity, at any number of columns, and leaves the
    other rows alone."""
    print("case", m, n, k, dtype, flush=True)
    c = {name: t.cuda().abs() for name, t in _data(m, n, k, dtype, 13).items()}
    c["wg"], c["wu"] = c["wg"] + 0.0625, c["wu"] + 0.0625
    c["gh"] = c["gh"] / 64 + 2.0 ** -10
    clean = _backward(c, "relu", dtype, h=True)
    c["x"][5, 3] = float("inf")
    got = _backward(c, "relu", dtype, h=True)
    rest = [i for i in range(m) if i != 5]
    for name in ("h", "dx"):
        assert (got[name][5] == float("inf")).all() and clean[name].isfinite().all() and torch.equal(got[name][rest], clean[name][rest]), name


@pytest.mark.parametrize("dtype,values,factor", [(BF16, [-2.0, -2.5, -3.0, -4.0, -5.0, -6.5, -8.0, -9.0, -10.0], 1.0),
                                                 (F16, [-2.0, -2.25, -2.5, -3.0, -3.5, -4.0, -4.5, -5.0, -5.5, -6.0], -4096.0)])
@pytest.mark.parametrize("rows", [1, 64])
def test_gelu_far_below_zero(dtype, values, factor, rows):
    """gelu and its slope to a relative error: the argument is exact (one product to a sum), so h and da are off by their roundings to the format and 2^-13 for
    the function, a quarter of binary16's and a 32nd of bfloat16's."""
    k = len(values)
    x = torch.diag(torch.tensor(values, dtype=torch.float64)).repeat(-(-rows // k) if rows > 1 else 1, 1)[:max(rows, k)]
    x = x if rows > 1 else x[:k]
    m, n = x.shape[0], 64
    c = {"x": x.to(dtype).cuda(), "wg": torch.ones(n, k, dtype=dtype, device="cuda"), "wu": torch.full((n, k), factor, dtype=dtype, device="cuda"),
         "gh": torch.ones(m, n, dtype=dtype, device="cuda")}
    a = x.to(dtype).double().sum(1, keepdim=True).expand(m, n)
    f, slope = activation(a, "gelu")
    h = torch.empty(m, n, dtype=dtype, device="cuda")
    daf.daf_gated_linear(c["x"], c["wg"], c["wu"], "gelu", h, _workspace(m, n, k, dtype, False))
    want = f * a * factor
    assert_within(h, want, (UNIT[dtype] + 2.0 ** -13) * want.abs() + TINY[dtype], "h")
    for kept in ((None, None), (a.to(dtype).cuda().contiguous(), (a * factor).to(dtype).cuda().contiguous())):
        one = {name: (t[:k] if name in ("x", "gh") else t) for name, t in c.items()}       # every value once: a column of x^T each
        got = _backward(one, "gelu", dtype, tuple(t if t is None else t[:k].contiguous() for t in kept))
        da = (a * factor * slope)[:k]
        want = da.t() * a[:k, 0]
        assert_within(got["dwg"], want, (2.01 * UNIT[dtype] + 2.0 ** -13) * want.abs() + TINY[dtype] * (1 + a[:k, 0].abs()), "grad_w_gate")

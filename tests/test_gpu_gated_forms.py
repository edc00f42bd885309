"""daf_gated_linear and its backward pass in every form that they are cut into: each size of tile, sums whole and in slices, whole rounds of the largest tiles in
front, both gradients side by side.  Bounds as in test_gpu_gated_linear.py; expected values in binary64 on the GPU."""
import pytest
import torch

import paper_2507_07149_amd as daf
from tests.test_gpu_gated_linear import BF16, F16, _backward, _Expected, _nan, _workspace

pytestmark = pytest.mark.gpu

# product, tile, in slices, whole rounds in front (or more than a round of the largest tiles): rows, columns of h, columns of x
ALONE = [
    ("forward", (64, 128), False, False, (34, 33, 8)), ("forward", (64, 128), True, False, (33, 34, 962)), ("forward", (64, 128), False, True, (28159, 770, 66)),
    ("forward", (64, 128), True, True, (32910, 132, 1423)), ("forward", (128, 128), False, False, (65, 6620, 8)), ("forward", (128, 128), True, False, (65, 2689, 2019)),
    ("forward", (128, 128), False, True, (15508, 1051, 258)), ("forward", (128, 128), True, True, (22950, 257, 2214)),
    ("forward", (128, 256), False, False, (25131, 65, 8)), ("forward", (128, 256), True, False, (65, 8205, 3599)), ("forward", (128, 256), False, True, (28628, 258, 1219)),
    ("forward", (128, 256), True, True, (1056, 7319, 3737)), ("forward", (256, 256), False, False, (24933, 196, 8)), ("forward", (256, 256), True, False, (16618, 69, 3521)),
    ("forward", (256, 256), False, True, (32901, 264, 840)), ("forward", (256, 256), True, True, (1040, 8220, 3591)),
    ("grad_input", (64, 128), False, True, (14510, 65, 2192)), ("grad_input", (64, 128), True, False, (34, 513, 8)), ("grad_input", (64, 128), True, True, (32922, 833, 261)),
    ("grad_input", (128, 128), False, False, (14099, 33, 8)), ("grad_input", (128, 128), True, False, (5522, 1217, 8)), ("grad_input", (128, 128), False, True, (20144, 130, 1629)),
    ("grad_input", (128, 128), True, True, (22532, 1251, 558)), ("grad_input", (128, 256), False, False, (23287, 33, 130)), ("grad_input", (128, 256), True, False, (5511, 3100, 129)),
    ("grad_input", (128, 256), False, True, (27810, 718, 513)), ("grad_input", (128, 256), True, True, (25127, 2258, 518)),
    ("grad_input", (256, 256), False, False, (25332, 33, 389)), ("grad_input", (256, 256), False, True, (32817, 875, 519)), ("grad_input", (256, 256), True, False, (16419, 2050, 133)),
    ("grad_input", (256, 256), True, True, (27613, 2070, 524)),
    ("grad_weight", (64, 128), True, False, (1154, 34, 8)), ("grad_weight", (64, 128), False, True, (129, 10905, 2072)), ("grad_weight", (64, 128), True, True, (1465, 10982, 517)),
    ("grad_weight", (128, 128), False, False, (34, 6415, 8)), ("grad_weight", (128, 128), True, False, (2483, 2696, 8)), ("grad_weight", (128, 128), False, True, (328, 10192, 1537)),
    ("grad_weight", (128, 128), True, True, (2473, 8470, 782)), ("grad_weight", (128, 256), False, False, (33, 6341, 392)), ("grad_weight", (128, 256), True, False, (6038, 2761, 134)),
    ("grad_weight", (128, 256), False, True, (1576, 10242, 778)), ("grad_weight", (128, 256), True, True, (4399, 9309, 771)),
    ("grad_weight", (256, 256), False, False, (33, 10235, 514)), ("grad_weight", (256, 256), False, True, (850, 9832, 1031)), ("grad_weight", (256, 256), True, False, (4172, 8273, 132)),
    ("grad_weight", (256, 256), True, True, (4340, 10269, 787))]
# tile, slices of grad_x, slices of the weights' gradients
BOTH = [((64, 128), False, False, (1155, 129, 8)), ((64, 128), False, True, (1112, 33, 8)), ((64, 128), True, False, (33, 578, 8)), ((64, 128), True, True, (456, 654, 8)),
        ((128, 128), False, False, (65, 67, 4039)), ((128, 128), False, True, (11075, 129, 8)), ((128, 128), True, False, (258, 5677, 8)),
        ((128, 128), True, True, (1952, 1098, 8)), ((128, 256), False, False, (619, 141, 4100)), ((128, 256), False, True, (2691, 34, 3207)),
        ((128, 256), True, False, (33, 1494, 3786)), ((128, 256), True, True, (3085, 2429, 129)), ((256, 256), False, False, (1059, 386, 4100)),
        ((256, 256), False, True, (6814, 66, 2331)), ((256, 256), False, True, (32907, 856, 262)), ((256, 256), True, False, (131, 3055, 2720)),
        ((256, 256), True, True, (3438, 4751, 129))]


def _data(m, n, k, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    return {"x": r(m, k).to(dtype), "wg": (r(n, k) / k ** 0.5).to(dtype), "wu": (r(n, k) / k ** 0.5).to(dtype), "gh": r(m, n).to(dtype)}


def _within(got, want, bound, what):
    """|got - want| <= bound for every element, all of them numbers."""
    off = (got.double() - want).abs()
    assert (off <= bound).all(), f"{what}: the worst {float((off / bound).nan_to_num(nan=float('inf')).max()):.3g} times its bound"


def _gradients(got, e, names):
    for name, want, bound in (("dx", e.dx, e.bound_dx), ("dwg", e.dw[0], e.bound_dw[0]), ("dwu", e.dw[1], e.bound_dw[1])):
        if name in names:
            _within(got[name], want, bound, name)


def _forward(c, act, dtype, e):
    m, k = c["x"].shape
    n = c["wg"].shape[0]
    h, a, u = (_nan(m, n, dtype=dtype) for _ in range(3))
    daf.daf_gated_linear(c["x"], c["wg"], c["wu"], act, h, _workspace(m, n, k, dtype, False), out_gate=a, out_up=u)
    for name, got, want, bound in (("h", h, e.h, e.bound_h), ("a", a, e.a, e.bound_a), ("u", u, e.u, e.bound_u)):
        _within(got, want, bound, name)
    return h


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("product,tile,sliced,whole,size", ALONE)
def test_products(product, tile, sliced, whole, size, dtype):
    m, n, k = size
    print("case", product, tile, sliced, whole, size, dtype, flush=True)
    s = daf.daf_gated_linear_schedule(m, n, k, product)
    assert (s["tile_rows"], s["tile_cols"]) == tile and (s["slices"] > 1) == sliced
    assert (s["whole_tiles"] > 0) == whole or (whole and tile == (256, 256) and s["tiles"] > 256)
    c = _data(m, n, k, dtype, 20)
    e = _Expected(c, "silu", dtype)
    if product == "forward":
        h = _forward(c, "silu", dtype, e)
        got = _backward(c, "silu", dtype, h=True, want="x")               # the same product again, with the slopes behind it
        assert torch.equal(got["h"], h)
        _gradients(got, e, ("dx",))
    else:
        names = ("dx",) if product == "grad_input" else ("dwg", "dwu")
        got = _backward(c, "silu", dtype, want=names[0][1])
        _gradients(got, e, names)
        again = _backward(c, "silu", dtype, want=names[0][1])
        assert all(torch.equal(got[name], again[name]) for name in names)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tile,input_sliced,weight_sliced,size", BOTH)
def test_both_gradients(tile, input_sliced, weight_sliced, size, dtype):
    m, n, k = size
    print("case both", tile, input_sliced, weight_sliced, size, dtype, flush=True)
    s, w = (daf.daf_gated_linear_schedule(m, n, k, f"grad_{of}_of_both") for of in ("input", "weight"))
    assert all((p["tile_rows"], p["tile_cols"]) == tile and p["whole_tiles"] == 0 for p in (s, w))
    assert (s["slices"] > 1, w["slices"] > 1) == (input_sliced, weight_sliced)
    assert (s, w) != tuple(daf.daf_gated_linear_schedule(m, n, k, f"grad_{of}") for of in ("input", "weight"))
    c = _data(m, n, k, dtype, 21)
    got = _backward(c, "gelu", dtype)
    _gradients(got, _Expected(c, "gelu", dtype), ("dx", "dwg", "dwu"))
    again = _backward(c, "gelu", dtype)
    assert all(torch.equal(got[name], again[name]) for name in ("dx", "dwg", "dwu"))
    kept = tuple((c["x"].double() @ c[w].double().t()).to(dtype) for w in ("wg", "wu"))
    _gradients(_backward(c, "gelu", dtype, kept), _Expected(c, "gelu", dtype, kept), ("dx", "dwg", "dwu"))


def test_offsets_beyond_32_bits():
    """h, a, u and [da du] of more than 2^32 bytes each, from more than 2^31 elements of h on: the last rows, and the weights' gradients, which only those
    rows give something to."""
    m, n, k, last = (1 << 18) + 300, 8200, 72, 300
    c = _data(last, n, k, BF16, 22)
    x, gh = torch.zeros(m, k, dtype=BF16, device="cuda"), torch.zeros(m, n, dtype=BF16, device="cuda")
    x[-last:], gh[-last:] = c["x"], c["gh"]
    whole = dict(c, x=x, gh=gh)
    e = _Expected(c, "silu", BF16)
    h, a, u = (_nan(m, n, dtype=BF16) for _ in range(3))
    daf.daf_gated_linear(x, c["wg"], c["wu"], "silu", h, _workspace(m, n, k, BF16, False), out_gate=a, out_up=u)
    for name, got, want, bound in (("h", h, e.h, e.bound_h), ("a", a, e.a, e.bound_a), ("u", u, e.u, e.bound_u)):
        _within(got[-last:], want, bound, name)
        assert not got[:-last].any(), name
    for kept in ((None, None), (a, u)):
        got = _backward(whole, "silu", BF16, kept)
        at = _Expected(c, "silu", BF16) if kept[0] is None else _Expected(c, "silu", BF16, (a[-last:], u[-last:]))
        got["dx"], rest = got["dx"][-last:], got["dx"][:-last]
        _gradients(got, at, ("dx", "dwg", "dwu"))
        assert not rest.any()
    del x, gh, whole, h, a, u, got, rest
    torch.cuda.empty_cache()

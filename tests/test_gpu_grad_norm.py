"""daf_grad_norm and daf_clip_grad_norm against sums in 64 bits."""
import math

import pytest
import torch

import paper_2507_07149_amd as daf
from tests.block_reference import TINY, UNIT, assert_within

pytestmark = pytest.mark.gpu


def _workspace():
    return torch.empty(daf.daf_grad_norm_workspace_bytes(), dtype=torch.uint8, device="cuda")


def _grads(sizes, seed, scale=0.1):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g, dtype=torch.float64) * scale).to(dt).cuda() for n, dt in sizes]


def _check(sizes, max_norm, seed=0, in_place=False):
    print("case", len(sizes), sizes[:4], max_norm, flush=True)
    grads = _grads(sizes, seed)
    before = [t.clone() for t in grads]
    outs = grads if in_place else [torch.full_like(t, float("nan")) for t in grads]
    norm = torch.full((1,), float("nan"), device="cuda")
    ws = _workspace()
    daf.daf_clip_grad_norm(list(zip(grads, outs)), max_norm, norm, ws)
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in before))
    # one rounding; the sums are exact to far below it
    assert abs(float(norm) - want) <= 2.0 ** -23 * want + 1e-300
    factor = min(1.0, max_norm / (want + 1e-6))
    for got, t in zip(outs, before):
        exact = t.double() * factor
        # norm, sum, quotient and product: four roundings of binary32, then one to the format
        assert_within(got, exact, (UNIT[t.dtype] + 6 * 2.0 ** -24) * exact.abs() + TINY[t.dtype], str(t.dtype))
        if factor == 1.0:
            assert torch.equal(got, t)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(grads, before))
    alone = torch.empty(1, device="cuda")
    daf.daf_grad_norm(before, alone, ws)
    assert torch.equal(alone, norm)


F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("max_norm", [1e-3, 1.0, 1e9, float("inf"), 0.0])
def test_mixed_list(max_norm, in_place):
    _check([(1, F32), (7, F16), (100_003, BF16), (0, F32), (8192, F32), (8193, F32), (16_384, F16), (16_385, BF16), (3, BF16), (0, F16)], max_norm,
           in_place=in_place)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 4095, 8191, 8192, 16_383, 16_385, 1 << 20])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_lengths(n, dtype):
    _check([(n, dtype)], 0.01)


@pytest.mark.parametrize("count", [95, 96, 97, 200, 301])
def test_long_lists(count):
    """More tensors than a launch carries; some of no elements at the ends of launches."""
    _check([((i * 37) % 5000 if i not in (0, 95, 96, 191) else 0, (F32, F16, BF16)[i % 3]) for i in range(count)], 0.5)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("count", [143, 144, 145, 199, 200, 201, 405])
def test_lists_around_what_a_launch_carries(count, in_place):
    _check([((i * 37) % 5000 if i not in (143, 144, 199, 200) else 0, (F32, F16, BF16)[i % 3]) for i in range(count)], 0.5, in_place=in_place)


def test_more_chunks_than_workgroups():
    _check([(30_000_001, F32), (11, BF16), (50_000_000, BF16)], 1.0)


def test_empty_list_of_elements():
    norm = torch.full((1,), 5.0, device="cuda")
    daf.daf_clip_grad_norm([torch.empty(0, device="cuda")], 1.0, norm, _workspace())
    assert float(norm) == 0.0


def test_unaligned_views():
    """Tensors that begin at any element, and gradients and outputs at different places of a vector."""
    for dtype in (F32, F16, BF16):
        flat, out = _grads([(50_000, dtype), (50_000, dtype)], 3)
        for a, b, n in ((1, 0, 40_001), (3, 5, 9000), (0, 7, 16), (2, 2, 33_333)):
            norm = torch.empty(1, device="cuda")
            daf.daf_clip_grad_norm([(flat[a:a + n], out[b:b + n])], 0.5, norm, _workspace())
            want = flat[a:a + n].double() * min(1.0, 0.5 / (float((flat[a:a + n].double() ** 2).sum().sqrt()) + 1e-6))
            assert_within(out[b:b + n], want, (UNIT[dtype] + 6 * 2.0 ** -24) * want.abs() + TINY[dtype], "view")


def test_huge_and_tiny_values():
    """Squares that binary32 cannot hold."""
    for value, dtype in ((3e38, BF16), (1e30, F32), (1e-30, F32), (2.0 ** -149, F32), (2.0 ** -24, F16)):
        t = torch.full((1000,), value, device="cuda", dtype=dtype)
        norm = torch.empty(1, device="cuda")
        daf.daf_grad_norm([t], norm, _workspace())
        want = torch.tensor(math.sqrt(1000) * float(t[0])).float()
        assert abs(float(norm) - float(want)) <= 2.0 ** -22 * float(want) + 2.0 ** -149 or float(want) == float(norm) == float("inf")


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_no_numbers(value):
    """An infinity: the norm is infinite and the others become zero; NaN: everything does."""
    t = torch.ones(20_000, device="cuda")
    t[777] = value
    out, norm = torch.empty_like(t), torch.empty(1, device="cuda")
    daf.daf_clip_grad_norm([(t, out)], 1.0, norm, _workspace())
    if math.isnan(value):
        assert norm.isnan().all() and out.isnan().all()
    else:
        assert float(norm) == float("inf") and out[777].isnan() and int((out == 0).sum()) == 19_999


def test_same_bits_and_graph():
    grads = _grads([(1_000_003, BF16), (77_777, F32), (5, F16)] * 40, 4)
    outs = [torch.empty_like(t) for t in grads]
    items, norm, ws = daf.grad_items(list(zip(grads, outs))), torch.empty(1, device="cuda"), _workspace()
    daf.daf_clip_grad_norm(items, 1.0, norm, ws)
    want = [t.clone() for t in outs + [norm]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        daf.daf_clip_grad_norm(items, 1.0, norm, ws)
    for _ in range(3):
        for t in outs + [norm]:
            t.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + [norm], want))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("in_place", [False, True])
def test_no_limit_leaves_infinite_gradients_as_they_are(dtype, in_place):
    """A max_norm of infinity clips nothing, whatever the norm; NaN still makes everything NaN."""
    for value, what in ((float("inf"), "inf"), (float("-inf"), "-inf"), (float("nan"), "nan")):
        t = torch.randn(20_001, generator=torch.Generator().manual_seed(5)).to(dtype).cuda()
        t[777] = value
        before = t.clone()
        out, norm = t if in_place else torch.empty_like(t), torch.empty(1, device="cuda")
        daf.daf_clip_grad_norm([(t, out)], float("inf"), norm, _workspace())
        if what == "nan":
            assert norm.isnan().all() and out.isnan().all()
        else:
            assert float(norm) == float("inf") and torch.equal(out, before)

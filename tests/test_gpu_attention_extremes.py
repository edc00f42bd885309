"""Attention whose scores are far from 0: up to the largest numbers of binary32, where a score times log2(e) is none of them any more.

Queries and keys have one element that is not zero, a power of two times a number of few bits, so that every score is exact, and the distance of two that differ is
thousands at least: what a query gets is the mean of the values of its largest scores.  Bounds are those of test_gpu_window_attention.py for scores without an error; a
gradient of more than the format holds may come of what dP and delta are off alone, and is not looked at."""
import math

import pytest
import torch

import paper_2507_07149_amd as daf
from tests import attention_reference as ref
from tests.block_reference import TINY, UNIT, assert_within

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
NAN = float("nan")
# dtype, powers of two of queries, keys and scale
SIZES = [(BF16, 12, 14, 0), (BF16, 16, 15, 0), (BF16, 20, 20, 0), (BF16, 60, 50, 16), (BF16, 61, 66, -1), (BF16, 63, 63, 0), (BF16, 63, 64, 0),
         (F16, 13, 13, 0), (F16, 14, 14, 1), (F16, 15, 14, 2), (F16, 14, 14, 20), (F16, 14, 14, 99)]
BEYOND = [(BF16, 63, 65, -2)]                                           # (the products alone are none of binary32's numbers; a step has them infinite)


def _int32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _inputs(dtype, rows, k_rows, heads, kv, dim, powers, sign, distinct=0):
    """Queries of 1 or 1.0625, keys of 1.40625 ... 1.875 (`distinct` steps to 1: no two the same), times their powers; the sign is the queries'."""
    g = torch.Generator().manual_seed(1)
    q, k = torch.zeros(rows, heads, dim, dtype=torch.float64), torch.zeros(k_rows, kv, dim, dtype=torch.float64)
    more = 0 if sum(powers) == 127 and distinct else 1                   # (there 1.0625 times the largest key would be none of binary32's numbers)
    q[:, :, 3] = sign * 2.0 ** powers[0] * (1 + more * torch.randint(0, 2, (rows, heads), generator=g).double() / 16)
    steps = torch.arange(k_rows).double()[:, None] / distinct if distinct else torch.randint(0, 4, (k_rows, kv), generator=g).double() * 0.15625
    k[:, :, 3] = 2.0 ** powers[1] * (1.40625 + steps)
    v, grad = (torch.randn(n, h, dim, generator=g, dtype=torch.float64).to(dtype).double() for n, h in ((k_rows, kv), (rows, heads)))
    for t in (q, k, q[:, :, 3].max() * k[:, :, 3].max() * 2.0 ** powers[2]):
        assert torch.equal(t.to(torch.float32 if t.dim() == 0 else dtype).double(), t)
    return q, k, v, grad


def _check(q, k, v, got, got_lse, window, sinks, scale, seqs, dtype):
    """(Exponentials of scores less the largest: less lse, the logarithm of how many are the largest would be lost in 64 bits too.)"""
    out, size, lse = torch.zeros_like(q), torch.zeros_like(q), torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64)
    for begin, rows, k_begin, keys in seqs:
        for h in range(q.shape[1] if keys else 0):
            x, (y, z) = q[begin:begin + rows, h], (t[k_begin:k_begin + keys, h // (q.shape[1] // k.shape[1])] for t in (k, v))
            s = (x @ y.T * scale).masked_fill(~ref.seen(rows, keys, window, sinks), -math.inf)
            p = (s - s.amax(1, keepdim=True)).exp()
            lse[h, begin:begin + rows] = s.amax(1) + p.sum(1).log()
            for t, value in ((out, p @ z), (size, p @ z.abs())):
                t[begin:begin + rows, h] = value / p.sum(1, keepdim=True)
    u, n, e = UNIT[dtype], max(keys for *_, keys in seqs) + 8, 2.0 ** -22
    assert_within(got, out, u * out.abs() + (u + 2 * e + n * 2.0 ** -24) * size + TINY[dtype], "out")
    if got_lse is not None:
        assert_within(got_lse, lse, 2 * e + n * 2.0 ** -24 + 4 * 2.0 ** -24 * lse.abs(), "lse")


@pytest.mark.parametrize("heads,kv,dim", [(2, 1, 64), (130, 130, 32), (80, 80, 128)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,a,b,c", SIZES + BEYOND)
def test_forward(dtype, a, b, c, sign, heads, kv, dim):
    """With the waves' shared keys, and with 128 queries to a workgroup."""
    print("case", dtype, a, b, c, sign, heads, flush=True)
    n = 300
    q, k, v, _ = _inputs(dtype, n, n, heads, kv, dim, (a, b, c), sign)
    for window, sinks in ((0, 0), (40, 2)):
        out, lse = torch.full((n, heads, dim), NAN, dtype=dtype, device="cuda"), torch.full((heads, n), NAN, device="cuda")
        daf.daf_window_attention(*(t.to(dtype).cuda() for t in (q, k, v)), out, lse, window=window, sinks=sinks, scale=2.0 ** c)
        _check(q, k, v, out, lse, window, sinks, 2.0 ** c, [(0, n, 0, n)], dtype)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,a,b,c", SIZES)
def test_step(dtype, a, b, c, sign):
    """In one piece and in several."""
    print("case", dtype, a, b, c, sign, flush=True)
    lengths = [100, 1, 0, 900]
    starts = [0, 100, 101, 101]
    q, k, v, _ = _inputs(dtype, 4, 1001, 4, 2, 64, (a, b, c), sign)
    for window, sinks in ((60, 2), (0, 0)):
        ws = torch.full((max(16, daf.daf_window_attention_step_workspace_bytes(4, 4, 2, 64, 1001, window, sinks)),), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((4, 4, 64), NAN, dtype=dtype, device="cuda")
        daf.daf_window_attention_step(*(t.to(dtype).cuda() for t in (q, k, v)), _int32(starts), _int32(lengths), out, ws, window=window, sinks=sinks, scale=2.0 ** c)
        _check(q, k, v, out, None, window, sinks, 2.0 ** c, [(i, 1, a, n) for i, (a, n) in enumerate(zip(starts, lengths))], dtype)


@pytest.mark.parametrize("powers", [(63, 64, -126), (63, 64, -128), (60, 60, -118), (0, 0, 0)])
def test_products_far_apart(powers):
    """Products whose distance is none of binary32's numbers, of a scale that leaves scores of 1 to 7 on both sides of 0."""
    heads, kv, dim, n, scale = 4, 2, 64, 400, 2.0 ** powers[2]
    q, k, v, _ = _inputs(BF16, n, n, heads, kv, dim, powers, 1, 0)
    q[:, :, 3], k[::3, :, 3] = 2.0 ** powers[0], -k[::3, :, 3]
    x, at = [t.to(BF16).cuda() for t in (q, k, v)], [0, 150, 0]
    for window, sinks in ((0, 0), (60, 3)):
        out, lse = torch.full((n, heads, dim), NAN, dtype=BF16, device="cuda"), torch.full((heads, n), NAN, device="cuda")
        daf.daf_window_attention(*x, out, lse, window=window, sinks=sinks, scale=scale)
        _check(q, k, v, out, lse, window, sinks, scale, [(0, n, 0, n)], BF16)
        ws = torch.full((max(16, daf.daf_window_attention_step_workspace_bytes(3, heads, kv, dim, n, window, sinks)),), 255, dtype=torch.uint8, device="cuda")
        out = torch.full((3, heads, dim), NAN, dtype=BF16, device="cuda")
        daf.daf_window_attention_step(x[0][:3], *x[1:], _int32(at), _int32([400, 33, 200]), out, ws, window=window, sinks=sinks, scale=scale)
        _check(q[:3], k, v, out, None, window, sinks, scale, [(i, 1, a, m) for i, (a, m) in enumerate(zip(at, (400, 33, 200)))], BF16)


def _backward(dtype, powers, sign, n, heads, kv, dim, window, sinks, distinct):
    print("case", dtype, powers, sign, n, heads, dim, window, sinks, flush=True)
    q, k, v, grad = _inputs(dtype, n, n, heads, kv, dim, powers, sign, distinct)
    dev, scale, u = lambda t: t.to(dtype).cuda(), 2.0 ** powers[2], UNIT[dtype]
    out, lse = torch.zeros_like(q), torch.zeros(heads, n, dtype=torch.float64)
    ref.attention(q, k, v, window, sinks, scale, [(0, n, 0, n)], out, lse)
    assert torch.equal(lse.float().double(), lse) and torch.equal(out.to(dtype).double(), out)
    want, sizes, inner, of_delta, _ = ref.attention_backward(q, k, v, out, lse, grad, window, sinks, scale, [(0, n, 0, n)])
    grads = [torch.full(t.shape, NAN, dtype=dtype, device="cuda") for t in (q, k, v)]
    ws = torch.full((daf.daf_window_attention_backward_workspace_bytes(n, heads, kv, dim, 1, window, sinks),), 255, dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_backward(dev(q), dev(k), dev(v), dev(out), lse.float().cuda(), dev(grad), *grads, ws, window=window, sinks=sinks, scale=scale)
    terms, e = n * heads // kv + 8, 2.0 ** -22
    for name, got, w, size, parts, rounded in zip(("grad_v", "grad_q", "grad_k"), *((t[2], t[0], t[1]) for t in (grads, want, sizes, inner, of_delta))):
        bound = u * w.abs() + (u + 2 * e + terms * 2.0 ** -24) * size + (dim + 16) * 2.0 ** -23 * parts + u * rounded + TINY[dtype]
        assert not got.isnan().any(), name
        if bound.max() < torch.finfo(dtype).max:
            assert_within(got, w, bound, name)
        else:
            assert name != "grad_v"


@pytest.mark.parametrize("heads,kv,dim", [(2, 1, 64), (8, 2, 128), (330, 330, 32), (164, 82, 128)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,a,b,c", SIZES + BEYOND)
def test_backward(dtype, a, b, c, sign, heads, kv, dim):
    """Every query has one largest score, its lse, and P of 1 there: grad_v is what the queries give that have the key as theirs, dS is 0 but for what dP and delta are off."""
    for window, sinks in ((0, 0), (20, 3)):
        _backward(dtype, (a, b, c), sign, 70, heads, kv, dim, window, sinks, 128)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (6, 2, 128)])
def test_backward_far_queries_and_pieces(heads, kv, dim, sign):
    """Queries that see only sinks and their window; and all keys, in pieces."""
    _backward(F16, (14, 14, 1), sign, 600, heads, kv, dim, 10, 3, 1024)
    _backward(F16, (14, 14, 1), sign, 600, heads, kv, dim, 0, 0, 1024)

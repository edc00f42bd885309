"""daf_window_attention, its backward pass and its form for single tokens against the formulas in 64 bits.

Bounds.  A score is a sum of `dim` products in binary32, each operation off by 2^-24 of the sum of absolute values at most, then a few more operations and an
exponential of 2^-22: E below is what p = exp(s - lse) may be off, relative to itself.  p (dS) is rounded to the format for its product, and the result once:
half a step each (UNIT); so is out, of which the backward pass makes delta.  Sums over n keys or queries add n 2^-24 of their terms' absolute values.  Binary16 has no steps below 2^-24: a p is off by half
of that, of a largest p of 1 at least (forward), or of 2^8 times p and dS (backward)."""
import math

import pytest
import torch

import paper_2507_07149_amd as daf
from tests import attention_reference as ref
from tests.block_reference import TINY, UNIT, assert_within

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
NAN = float("nan")


def _exponent(dim, score_size):
    return (dim + 16) * 2.0 ** -24 * (score_size + 16) + 2.0 ** -22


def _int32(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def _fused(tensors, dtype, device="cuda"):
    """The tensors [rows, heads, dim] as views beside each other in one buffer [rows, all heads, dim], as a projection leaves them."""
    whole = torch.cat(tensors, 1).to(dtype).to(device)
    at, views = 0, []
    for t in tensors:
        views.append(whole[:, at:at + t.shape[1]])
        at += t.shape[1]
    return views


def _empty(rows, heads, dim, dtype):
    return torch.full((rows, heads, dim), NAN, dtype=dtype, device="cuda")


def _check_forward(q, k, v, got, got_lse, window, sinks, scale, seqs, dtype):
    """`got` [rows, heads, dim] and `got_lse` against q, k, v (64 bits, on the CPU); rows of no sequence are NaN as they were."""
    dim, u = q.shape[2], UNIT[dtype]
    out, lse = torch.full_like(q, NAN), torch.full((q.shape[1], q.shape[0]), NAN, dtype=torch.float64)
    size, score = ref.attention(q, k, v, window, sinks, scale, seqs, out, lse)
    n = max(keys for *_, keys in seqs) + 8
    e = _exponent(dim, score)
    small = n * 2.0 ** -25 * v[torch.isfinite(v)].abs().max() if dtype == F16 else 0.0
    size = torch.nan_to_num(size)
    assert_within(got, out, u * torch.nan_to_num(out).abs() + (u + 2 * e + n * 2.0 ** -24) * size + small + TINY[dtype], "out")
    if got_lse is not None:
        size = torch.nan_to_num(lse, neginf=0.0).abs()
        assert_within(got_lse, lse, 2 * e + n * 2.0 ** -24 + 4 * 2.0 ** -24 * size, "lse")


def _forward(dtype, heads, kv, dim, starts, window, sinks, rows=None, keys=None, scale=None, seed=0, lse=True):
    """`keys`: (first row, keys) of each sequence in a cache of its own; else the queries' rows."""
    print("case", dtype, heads, kv, dim, starts, window, sinks, keys, flush=True)
    g = torch.Generator().manual_seed(seed)
    rows = starts[-1] + 3 if rows is None else rows
    k_rows = rows if keys is None else max(a + n for a, n in keys) + 2
    r = lambda *s: _randn(g, *s).to(dtype).double()
    q, k, v = r(rows, heads, dim), r(k_rows, kv, dim), r(k_rows, kv, dim)
    if keys is None:
        dq, dk, dv = _fused([q, k, v], dtype)
        where = {}
    else:
        dq, (dk, dv) = q.to(dtype).cuda(), _fused([k, v], dtype)
        where = {"k_starts": _int32(a for a, _ in keys), "k_lengths": _int32(n for _, n in keys)}
    out, got_lse = _empty(rows, heads, dim, dtype), torch.full((heads, rows), NAN, device="cuda") if lse else None
    daf.daf_window_attention(dq, dk, dv, out, got_lse, window=window, sinks=sinks, scale=scale, q_starts=_int32(starts), **where)
    seqs = list(ref.sequences(rows, starts, *(zip(*keys) if keys else (None, None))))
    _check_forward(q, k, v, out, got_lse, window, sinks, dim ** -0.5 if scale is None else scale, seqs, dtype)
    return out, got_lse


STARTS = [[0, 1], [0, 5], [2, 66, 66, 67, 197], [0, 31, 64, 193, 450], [1, 258], [0, 513]]


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 4, 2, 128), (F16, 3, 3, 64), (BF16, 5, 1, 80), (F16, 2, 1, 8), (BF16, 2, 2, 40), (F16, 4, 1, 96), (BF16, 1, 1, 120)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (64, 4), (100, 70), (129, 1), (0, 9)])
def test_forward(dtype, heads, kv, dim, window, sinks):
    for starts in STARTS:
        _forward(dtype, heads, kv, dim, starts, window, sinks)


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 4, 2, 128), (F16, 3, 1, 64), (BF16, 2, 1, 72)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 2), (200, 130), (1, 1)])
def test_forward_over_a_cache(dtype, heads, kv, dim, window, sinks):
    """More keys than queries, as many, fewer (the first queries see nothing), none at all; sequences that share rows."""
    keys = [(3, 300), (200, 64), (3, 40), (500, 0), (320, 129)]
    _forward(dtype, heads, kv, dim, [0, 1, 65, 165, 170, 300], window, sinks, keys=keys)


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 48, 8, 128), (F16, 80, 80, 64), (BF16, 50, 10, 80), (F16, 90, 90, 24)])
def test_forward_of_many_tiles(dtype, heads, kv, dim):
    """Enough tiles of 128 queries for the kernel that takes those."""
    for window, sinks in ((0, 0), (100, 70), (1, 3)):
        _forward(dtype, heads, kv, dim, [0, 31, 64, 193, 450, 800], window, sinks)
    _forward(dtype, heads, kv, dim, [0, 1, 65, 165, 170, 500], 50, 40, keys=[(3, 300), (200, 64), (3, 40), (500, 0), (320, 400)])


def test_order_of_many_tiles():
    """More than 64 sequences of 0 to 9 tiles, with a window of some of them: every tile is found once."""
    g = torch.Generator().manual_seed(10)
    lengths = torch.randint(0, 1200, (90,), generator=g).tolist()
    lengths[7:60:9] = [0] * 6
    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    rows, dim = starts[-1], 8
    q, k, v = (_randn(g, rows, 1, dim).to(BF16).double() for _ in range(3))
    for window in (1, 300, 0):
        out, lse = _empty(rows, 1, dim, BF16), torch.full((1, rows), NAN, device="cuda")
        daf.daf_window_attention(*(t.to(BF16).cuda() for t in (q, k, v)), out, lse, window=window, sinks=1, q_starts=_int32(starts))
        _check_forward(q, k, v, out, lse, window, 1, dim ** -0.5, list(ref.sequences(rows, starts)), BF16)


def test_forward_many_sequences():
    lengths = [1, 2, 0, 33, 7] * 40
    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    _forward(BF16, 2, 1, 64, starts, 5, 1)


@pytest.mark.parametrize("scale", [-0.125, 0.0, 0.7])
def test_forward_scales(scale):
    _forward(F16, 2, 1, 64, [0, 150], 70, 2, scale=scale)


def test_forward_long():
    _forward(BF16, 2, 1, 128, [0, 2500], 700, 5, lse=False)


def test_scores_that_grow():
    """Every key's score is larger than those before: the running maximum moves all the time; and large ones."""
    g = torch.Generator().manual_seed(3)
    n, dim = 400, 64
    for dtype, most in ((BF16, 90.0), (F16, 300.0)):
        q = _randn(g, n, 2, dim).sign() * 2
        k = q[:, :1].mean(0, keepdim=True).sign().expand(n, 1, dim) * torch.linspace(0.1, most / 16, n, dtype=torch.float64)[:, None, None]
        q, k, v = (t.to(dtype).double() for t in (q, k, _randn(g, n, 1, dim)))
        out, lse = _empty(n, 2, dim, dtype), torch.full((2, n), NAN, device="cuda")
        daf.daf_window_attention(*(t.to(dtype).cuda() for t in (q, k, v)), out, lse, window=0, sinks=0)
        _check_forward(q, k, v, out, lse, 0, 0, dim ** -0.5, [(0, n, 0, n)], dtype)


@pytest.mark.parametrize("heads,dim", [(2, 64), (80, 128)])
def test_what_is_not_seen_has_no_influence(heads, dim):
    """NaN and infinities in keys and values behind the window, behind the query and behind the cache's end: only the queries that see them change."""
    g = torch.Generator().manual_seed(4)
    n, window, sinks = 300, 90, 2
    q, k, v = (_randn(g, n, heads, dim).to(BF16).double() for _ in range(3))
    k[40], v[41, :, 3], k[170, 0, 0], v[171, 1] = NAN, math.inf, math.inf, -math.inf
    out, lse = _empty(n, heads, dim, BF16), torch.full((heads, n), NAN, device="cuda")
    daf.daf_window_attention(*(t.to(BF16).cuda() for t in (q, k, v)), out, lse, window=window, sinks=sinks)
    mask = ref.seen(n, n, window, sinks)
    touched = mask[:, [40, 41, 170, 171]].any(1)
    clean = [torch.where(torch.isfinite(t), t, 0.0) for t in (q, k, v)]
    want, want_lse = torch.zeros_like(q), torch.zeros(heads, n, dtype=torch.float64)
    size, score = ref.attention(*clean, window, sinks, dim ** -0.5, [(0, n, 0, n)], want, want_lse)
    e = _exponent(dim, score)
    free = ~touched
    bound = UNIT[BF16] * want.abs() + (UNIT[BF16] + 2 * e + n * 2.0 ** -24) * size
    assert_within(out[free.cuda()], want[free], bound[free], "out of queries that do not see them")
    assert_within(lse[:, free.cuda()], want_lse[:, free], 2 * e + n * 2.0 ** -24 + 2.0 ** -22 * want_lse[:, free].abs(), "lse")
    assert torch.isnan(out[mask[:, 40].cuda()]).all() and not torch.isfinite(out[mask[:, 41].cuda()][:, :, 3]).any()
    assert not torch.isfinite(out[mask[:, 171].cuda()][:, 1]).any()
    assert torch.isfinite(out[(mask[:, 41] & ~mask[:, [40, 170, 171]].any(1)).cuda()][:, :, :3]).all()


def _backward(dtype, heads, kv, dim, starts, window, sinks, rows=None, scale=None, seed=0, fused=True):
    print("case backward", dtype, heads, kv, dim, starts, window, sinks, flush=True)
    g = torch.Generator().manual_seed(seed)
    rows = starts[-1] + 2 if rows is None else rows
    r = lambda *s: _randn(g, *s).to(dtype).double()
    q, k, v, grad = r(rows, heads, dim), r(rows, kv, dim), r(rows, kv, dim), r(rows, heads, dim)
    factor = dim ** -0.5 if scale is None else scale
    seqs = list(ref.sequences(rows, starts))
    out, lse = torch.zeros_like(q), torch.zeros(heads, rows, dtype=torch.float64)
    ref.attention(q, k, v, window, sinks, factor, seqs, out, lse)
    out, lse = out.to(dtype).double(), lse.float().double()
    want, sizes, inner, of_delta, score = ref.attention_backward(q, k, v, out, lse, grad, window, sinks, factor, seqs)
    dq, dk, dv = _fused([q, k, v], dtype)
    if fused:
        gq, gk, gv = _fused([torch.full_like(q, NAN), torch.full_like(k, NAN), torch.full_like(v, NAN)], dtype)
    else:
        gq, gk, gv = _empty(rows, heads, dim, dtype), _empty(rows, kv, dim, dtype), _empty(rows, kv, dim, dtype)
    ws = torch.full((daf.daf_window_attention_backward_workspace_bytes(rows, heads, kv, dim, len(starts) - 1, window, sinks),), 255, dtype=torch.uint8, device="cuda")
    dout, dlse, dgrad = out.to(dtype).cuda(), lse.float().cuda(), grad.to(dtype).cuda()
    daf.daf_window_attention_backward(dq, dk, dv, dout, dlse, dgrad, gq, gk, gv, ws, window=window, sinks=sinks, scale=scale, q_starts=_int32(starts))
    u, n = UNIT[dtype], max(m for _, m, *_ in seqs) * (heads // kv) + 8
    e = _exponent(dim, score)
    inside = torch.zeros(rows, dtype=torch.bool)
    inside[starts[0]:starts[-1]] = True
    for name, got, w, size, parts, rounded, other in (("grad_q", gq, want[0], sizes[0], inner[0], of_delta[0], k),
                                                      ("grad_k", gk, want[1], sizes[1], inner[1], of_delta[1], q),
                                                      ("grad_v", gv, want[2], sizes[2], inner[2], of_delta[2], grad)):
        small = n * 2.0 ** -33 * other.abs().max() if dtype == F16 else 0.0
        bound = u * w.abs() + (u + 2 * e + n * 2.0 ** -24) * size + (dim + 16) * 2.0 ** -23 * parts + u * rounded + small + TINY[dtype]
        assert_within(got[inside.cuda()], w[inside], bound[inside], name)
        assert torch.isnan(got[(~inside).cuda()]).all(), name + ": rows of no sequence"
    return gq, gk, gv


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 4, 2, 128), (F16, 3, 3, 64), (BF16, 5, 1, 80), (F16, 2, 1, 8), (BF16, 2, 2, 40), (F16, 4, 1, 96)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (64, 4), (100, 70), (129, 1)])
def test_backward(dtype, heads, kv, dim, window, sinks):
    for starts in STARTS:
        _backward(dtype, heads, kv, dim, starts, window, sinks)


def test_backward_sinks_of_a_long_sequence():
    _backward(BF16, 2, 1, 64, [0, 1500], 100, 3)
    _backward(F16, 6, 2, 128, [0, 700, 1500], 60, 200, fused=False)
    _backward(BF16, 4, 2, 128, [0, 900, 901, 1700, 1710, 2400], 64, 40)
    _backward(F16, 3, 1, 80, [3, 800, 1300], 1, 128)
    _backward(BF16, 2, 2, 32, [0, 1111], 7, 1)


def test_backward_without_pieces():
    """As many key tiles as fill the chip: no tile's work is shared out (and, in the first, with far queries)."""
    _backward(F16, 48, 48, 64, [0, 700, 1300], 100, 3)
    _backward(BF16, 40, 20, 128, [1, 1400], 0, 0)
    _backward(BF16, 44, 22, 128, [0, 700, 1300], 64, 33)
    _backward(F16, 48, 48, 96, [0, 400, 1000], 1, 128)
    _backward(BF16, 60, 60, 24, [0, 900], 200, 0)


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 8, 2, 128), (F16, 8, 2, 64), (BF16, 6, 1, 80), (F16, 12, 1, 24), (F16, 4, 1, 120), (F16, 22, 22, 64), (BF16, 11, 11, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 0), (600, 30), (128, 2)])
def test_backward_in_pieces(dtype, heads, kv, dim, window, sinks):
    """Few key tiles, of long sequences: a tile's queries, of all heads that share it, are shared out."""
    starts = [1, 1301, 1303, 1500]
    if window == 0 or (window != 128 and kv <= 2):
        assert daf.daf_window_attention_backward_workspace_bytes(1502, heads, kv, dim, 3, window, 0) > 2 * 1502 * heads * 4 + 16
    _backward(dtype, heads, kv, dim, starts, window, sinks)


def test_backward_many_sequences():
    lengths = [1, 2, 0, 33, 7] * 40
    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    _backward(BF16, 2, 1, 64, starts, 5, 1)
    # one of them long, its far queries' chunks fewer than sequences
    _backward(F16, 2, 1, 64, starts + [starts[-1] + 800, starts[-1] + 810], 5, 2)


@pytest.mark.parametrize("scale", [-0.125, 0.0])
def test_backward_scales(scale):
    _backward(F16, 2, 1, 64, [0, 150], 70, 2, scale=scale)


def test_backward_large_gradients():
    """Binary16: 2^8 P (dP - delta) leaves the format's range; the rows are done again without it."""
    g = torch.Generator().manual_seed(9)
    n, heads, kv, dim = 140, 4, 2, 64
    q, k, v, grad = _randn(g, n, heads, dim) * 2, _randn(g, n, kv, dim) * 2, _randn(g, n, kv, dim) * 8, _randn(g, n, heads, dim) * 40
    grad[100:] /= 400
    q, k, v, grad = (t.to(F16).double() for t in (q, k, v, grad))
    seqs, scale = [(0, n, 0, n)], 2.0 ** -6
    out, lse = torch.zeros_like(q), torch.zeros(heads, n, dtype=torch.float64)
    ref.attention(q, k, v, 0, 0, scale, seqs, out, lse)
    out, lse = out.to(F16).double(), lse.float().double()
    want, sizes, inner, of_delta, score = ref.attention_backward(q, k, v, out, lse, grad, 0, 0, scale, seqs)
    dev = lambda t: t.to(F16).cuda()
    grads = [torch.full(t.shape, NAN, dtype=F16, device="cuda") for t in (q, k, v)]
    ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(n, heads, kv, dim), dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_backward(dev(q), dev(k), dev(v), dev(out), lse.float().cuda(), dev(grad), *grads, ws, scale=scale)
    u, e, terms = UNIT[F16], _exponent(dim, score), 2 * n + 8
    for name, got, w, size, parts, rounded, other in zip(("grad_q", "grad_k", "grad_v"), grads, want, sizes, inner, of_delta, (k, q, grad)):
        assert w.abs().max() < 65504, name
        bound = u * w.abs() + (u + 2 * e + terms * 2.0 ** -24) * size + (dim + 16) * 2.0 ** -23 * parts + u * rounded + terms * 2.0 ** -33 * other.abs().max() + TINY[F16]
        assert_within(got, w, bound, name)


def test_gradients_against_differences():
    """The forward pass twice, a step to each side: the slope of sum(out * grad) along a direction of q, k and v together.  Steps are whole numbers of the
    format's, so that the inputs are what they are taken for; out's rounding is the bound (every element off by half a step on both sides)."""
    g = torch.Generator().manual_seed(5)
    n, heads, kv, dim, window, sinks = 150, 4, 2, 64, 40, 2
    draw = lambda *s: torch.randint(-64, 65, s, generator=g).double() / 32
    q, k, v, grad = draw(n, heads, dim), draw(n, kv, dim), draw(n, kv, dim), draw(n, heads, dim) / 4
    step = [torch.randint(-1, 2, t.shape, generator=g).double() / 32 for t in (q, k, v)]
    side = []
    for sign in (1, -1):
        x = [(t + sign * s).to(F16).cuda() for t, s in zip((q, k, v), step)]
        out = torch.zeros(n, heads, dim, dtype=F16, device="cuda")
        daf.daf_window_attention(*x, out, window=window, sinks=sinks)
        side.append(out.double().cpu())
    slope = ((side[0] - side[1]) * grad).sum().item() / 2
    x = [t.to(F16).cuda() for t in (q, k, v)]
    out, lse = torch.zeros(n, heads, dim, dtype=F16, device="cuda"), torch.zeros(heads, n, device="cuda")
    daf.daf_window_attention(*x, out, lse, window=window, sinks=sinks)
    grads = [torch.zeros_like(t) for t in x]
    ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(n, heads, kv, dim, 1, window, sinks), dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_backward(*x, out, lse, grad.to(F16).cuda(), *grads, ws, window=window, sinks=sinks)
    got = sum((a.double().cpu() * b).sum().item() for a, b in zip(grads, step))
    # the same difference in 64 bits says how far it is from the slope by itself
    exact = []
    for sign in (1, -1):
        o, l = torch.zeros_like(q), torch.zeros(heads, n, dtype=torch.float64)
        ref.attention(q + sign * step[0], k + sign * step[1], v + sign * step[2], window, sinks, dim ** -0.5, [(0, n, 0, n)], o, l)
        exact.append(o)
    curvature = abs(((exact[0] - exact[1]) * grad).sum().item() / 2 - got)
    rounding = 3 * UNIT[F16] * (side[0].abs() * grad.abs()).sum().item()
    assert abs(slope - got) <= rounding + curvature and curvature <= 0.02 * abs(got) + rounding, (slope, got, curvature, rounding)


@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_slopes_of_differences(which):
    """The forward pass a step to each side of q, of k, of v alone, every element's step in the direction of its gradient (in 64 bits, from the formula), so that
    all of them add up to a slope of many times what it may be off: out's and the gradient's bounds, added up without regard to sign, and what the difference is off in 64 bits.
    (Inputs and steps are whole 64ths, which binary16 holds.)  A gradient of zeros, of the other sign, or of twice the size is off by the slope at least."""
    g = torch.Generator().manual_seed(12)
    n, heads, kv, dim, window, sinks = 150, 4, 2, 64, 40, 2
    draw = lambda *s: torch.randint(-64, 65, s, generator=g).double() / 32
    inputs, grad = dict(q=draw(n, heads, dim), k=draw(n, kv, dim), v=draw(n, kv, dim)), draw(n, heads, dim) / 4
    scale, seqs, u = dim ** -0.5, [(0, n, 0, n)], UNIT[F16]

    def exact(inputs):
        out, lse = torch.zeros(n, heads, dim, dtype=torch.float64), torch.zeros(heads, n, dtype=torch.float64)
        size, score = ref.attention(*inputs.values(), window, sinks, scale, seqs, out, lse)
        return out, lse, size, score

    out, lse, size, score = exact(inputs)
    # delta is made of the rounded out
    want, sizes, inner, of_delta, _ = ref.attention_backward(*inputs.values(), out, lse, grad, window, sinks, scale, seqs)
    at, e, terms = "qkv".index(which), _exponent(dim, score), 2 * n + 8
    other = (inputs["k"], inputs["q"], grad)[at]
    off = u * want[at].abs() + (u + 2 * e + terms * 2.0 ** -24) * sizes[at] + (dim + 16) * 2.0 ** -23 * inner[at] + u * of_delta[at] + terms * 2.0 ** -33 * other.abs().max() + TINY[F16]
    off_out = u * out.abs() + (u + 2 * e + n * 2.0 ** -24) * size + n * 2.0 ** -25 * inputs["v"].abs().max() + TINY[F16]
    step = want[at].sign() / 64
    sides = [dict(inputs, **{which: inputs[which] + s * step}) for s in (1, -1)]
    slope = (want[at] * step).sum().item()
    difference = ((exact(sides[0])[0] - exact(sides[1])[0]) * grad).sum().item() / 2
    bound = (off * step.abs()).sum().item() + 1.1 * (off_out * grad.abs()).sum().item() + abs(difference - slope)
    assert 0 < bound < slope / 2, (slope, bound)
    dev = lambda i: [t.to(F16).cuda() for t in i.values()]
    outs = []
    for side in sides:
        outs.append(torch.zeros(n, heads, dim, dtype=F16, device="cuda"))
        daf.daf_window_attention(*dev(side), outs[-1], window=window, sinks=sinks)
    got_difference = ((outs[0].double().cpu() - outs[1].double().cpu()) * grad).sum().item() / 2
    x, got_out, got_lse = dev(inputs), torch.zeros(n, heads, dim, dtype=F16, device="cuda"), torch.zeros(heads, n, device="cuda")
    daf.daf_window_attention(*x, got_out, got_lse, window=window, sinks=sinks)
    grads = [torch.zeros_like(t) for t in x]
    ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(n, heads, kv, dim, 1, window, sinks), dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_backward(*x, got_out, got_lse, grad.to(F16).cuda(), *grads, ws, window=window, sinks=sinks)
    got = (grads[at].double().cpu() * step).sum().item()
    assert abs(got_difference - got) <= bound, (got_difference, got, slope, bound)


@pytest.mark.parametrize("heads,dim", [(2, 64), (130, 128)])
def test_backward_what_is_not_seen_has_no_influence(heads, dim):
    g = torch.Generator().manual_seed(6)
    n, window, sinks = 260, 70, 2
    q, k, v, grad = (_randn(g, n, heads, dim).to(BF16).double() for _ in range(4))
    out, lse = torch.zeros_like(q), torch.zeros(heads, n, dtype=torch.float64)
    ref.attention(q, k, v, window, sinks, dim ** -0.5, [(0, n, 0, n)], out, lse)
    bad_k, bad_grad = k.clone(), grad.clone()
    bad_k[33, 0, 5], bad_grad[150, 1] = math.inf, NAN
    dev = lambda t: t.to(BF16).cuda()
    ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(n, heads, heads, dim, 1, window, sinks), dtype=torch.uint8, device="cuda")
    results = []
    for kk, gg in ((k, grad), (bad_k, bad_grad)):
        grads = [torch.zeros(n, heads, dim, dtype=BF16, device="cuda") for _ in range(3)]
        daf.daf_window_attention_backward(dev(q), dev(kk), dev(v), dev(out), lse.float().cuda(), dev(gg), *grads, ws, window=window, sinks=sinks)
        results.append([t.double().cpu() for t in grads])
    mask = ref.seen(n, n, window, sinks)
    # head 0: key 33 is infinite: the queries that see it, and through their dS the keys that those see.  head 1: query 150's gradient is NaN: the keys that it sees
    q_free = torch.stack([~mask[:, 33], torch.arange(n) != 150], 1)
    touched = mask[mask[:, 33]].any(0)
    k_free = torch.stack([~touched, ~mask[150]], 1)
    for i, free in enumerate((q_free, k_free, k_free)):
        a, b = results[0][i][:, :2][free], results[1][i][:, :2][free]
        assert torch.isfinite(b).all(), i
        assert (a - b).abs().max() <= 4 * UNIT[BF16] * results[0][i].abs().max(), i      # (rows that are done again row by row round less)
        assert not torch.isfinite(results[1][i][:, 1][~free[:, 1]]).all(), i


def _step(dtype, sequences, heads, kv, dim, lengths, window, sinks, seed=0, workspace=True):
    print("case step", dtype, heads, kv, dim, lengths, window, sinks, flush=True)
    g = torch.Generator().manual_seed(seed)
    starts, at = [], 1
    for n in lengths:
        starts.append(at)
        at += n + 2
    r = lambda *s: _randn(g, *s).to(dtype).double()
    q, k, v = r(sequences, heads, dim), r(at, kv, dim), r(at, kv, dim)
    dead = torch.ones(at, dtype=torch.bool)
    for a, n in zip(starts, lengths):
        dead[a:a + n] = False
    dk, dv = _fused([k.masked_fill(dead[:, None, None], NAN), v.masked_fill(dead[:, None, None], NAN)], dtype)
    out = _empty(sequences, heads, dim, dtype)
    need = daf.daf_window_attention_step_workspace_bytes(sequences, heads, kv, dim, at, window, sinks)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_step(q.to(dtype).cuda(), dk, dv, _int32(starts), _int32(lengths), out, ws, window=window, sinks=sinks)
    seqs = [(i, 1, a, n) for i, (a, n) in enumerate(zip(starts, lengths))]
    _check_forward(q, k, v, out, None, window, sinks, dim ** -0.5, seqs, dtype)


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 32, 8, 128), (F16, 12, 12, 64), (BF16, 5, 1, 80), (F16, 40, 2, 8), (BF16, 17, 1, 96), (F16, 2, 2, 40)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (64, 4), (300, 130), (17, 1)])
def test_step(dtype, heads, kv, dim, window, sinks):
    _step(dtype, 7, heads, kv, dim, [1, 0, 700, 64, 65, 2, 333], window, sinks)
    _step(dtype, 1, heads, kv, dim, [1500], window, sinks)


def test_step_one_long_sequence():
    _step(BF16, 1, 8, 2, 128, [9000], 0, 0)
    _step(F16, 2, 4, 4, 64, [5000, 9000], 4000, 100)


def test_step_what_is_not_seen_has_no_influence():
    g = torch.Generator().manual_seed(8)
    n, window, sinks = 500, 100, 3
    q, k, v = _randn(g, 1, 4, 64), _randn(g, n, 2, 64), _randn(g, n, 2, 64)
    q, k, v = (t.to(F16).double() for t in (q, k, v))
    k[3:400], v[3:400] = NAN, math.inf
    out = _empty(1, 4, 64, F16)
    need = daf.daf_window_attention_step_workspace_bytes(1, 4, 2, 64, n, window, sinks)
    ws = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_step(*(t.to(F16).cuda() for t in (q, k, v)), _int32([0]), _int32([n]), out, ws, window=window, sinks=sinks)
    _check_forward(q, k, v, out, None, window, sinks, 64 ** -0.5, [(0, 1, 0, n)], F16)


def _three_calls(stream=None):
    """A forward and a backward pass and a step on buffers of their own: a function that makes the calls, and the outputs."""
    g = torch.Generator(device="cuda").manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)
    n, heads, kv, dim = 333, 4, 2, 64
    q, k, v, grad = r(n, heads, dim), r(n, kv, dim), r(n, kv, dim), r(n, heads, dim)
    out, lse, token = torch.zeros_like(q), torch.zeros(heads, n, device="cuda"), r(3, heads, dim)
    gq, gk, gv, token_out = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros(3, heads, dim, dtype=BF16, device="cuda")
    starts, k_starts, k_lengths = _int32([0, 100, n]), _int32([0, 5, 100]), _int32([333, 200, 1])
    ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(n, heads, kv, dim, 2, 90, 3), dtype=torch.uint8, device="cuda")
    ws2 = torch.zeros(max(16, daf.daf_window_attention_step_workspace_bytes(3, heads, kv, dim, n, 90, 3)), dtype=torch.uint8, device="cuda")
    how = dict(window=90, sinks=3, stream=stream)

    def calls():
        daf.daf_window_attention(q, k, v, out, lse, q_starts=starts, **how)
        daf.daf_window_attention_backward(q, k, v, out, lse, grad, gq, gk, gv, ws, q_starts=starts, **how)
        daf.daf_window_attention_step(token, k, v, k_starts, k_lengths, token_out, ws2, **how)
    return calls, [out, lse, gq, gk, gv, token_out], [q, k, v]


def test_captured_and_replayed():
    calls, outs, ins = _three_calls()
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(3):
        ins[turn % 3].mul_(-0.5)
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        calls()
        torch.cuda.synchronize()
        for a, b in zip(replayed, outs):
            assert torch.equal(a, b)


def test_another_stream_and_the_same_bits():
    calls, outs, _ = _three_calls()
    calls()
    torch.cuda.synchronize()
    first = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    calls, outs, _ = _three_calls(side)
    torch.cuda.synchronize()
    calls()
    side.synchronize()
    for a, b in zip(first, outs):
        assert torch.equal(a, b)


def test_nothing_to_do():
    e = lambda *s: torch.zeros(*s, dtype=BF16, device="cuda")
    daf.daf_window_attention(e(0, 4, 64), e(0, 2, 64), e(0, 2, 64), e(0, 4, 64))
    ws = torch.zeros(16, dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_backward(e(0, 4, 64), e(0, 2, 64), e(0, 2, 64), e(0, 4, 64), torch.zeros(4, 0, device="cuda"), e(0, 4, 64), e(0, 4, 64),
                                      e(0, 2, 64), e(0, 2, 64), ws)
    daf.daf_window_attention_step(e(0, 4, 64), e(5, 2, 64), e(5, 2, 64), _int32([]), _int32([]), e(0, 4, 64))
    torch.cuda.synchronize()


def test_no_keys():
    r = lambda *s: torch.randn(*s, device="cuda").to(BF16)
    out, lse = _empty(40, 4, 64, BF16), torch.zeros(4, 40, device="cuda")
    daf.daf_window_attention(r(40, 4, 64), r(0, 2, 64), r(0, 2, 64), out, lse, q_starts=_int32([0, 30, 40]), k_starts=_int32([0, 0]), k_lengths=_int32([0, 7]))
    assert not out.any() and (lse == -math.inf).all()
    out = _empty(3, 4, 64, BF16)
    ws = torch.zeros(max(16, daf.daf_window_attention_step_workspace_bytes(3, 4, 2, 64, 0)), dtype=torch.uint8, device="cuda")
    daf.daf_window_attention_step(r(3, 4, 64), r(0, 2, 64), r(0, 2, 64), _int32([0] * 3), _int32([0, 3, 0]), out, ws)
    assert not out.any()


@pytest.mark.parametrize("heads,dim", [(2, 64), (2, 128), (80, 128), (24, 64), (13, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 2)])
def test_all_that_overflowed(heads, dim, window, sinks):
    """Queries that are all NaN, and gradients that are: all that they reach is NaN, and nothing else is."""
    n = 1400
    r = lambda: torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(3)).to(F16).cuda()
    q, k, v, grad, out = r(), r(), r(), r(), torch.zeros(n, heads, dim, dtype=F16, device="cuda")
    lse = torch.zeros(heads, n, device="cuda")
    bad = torch.full_like(q, NAN)
    daf.daf_window_attention(bad, k, v, out, lse, window=window, sinks=sinks)
    assert out.isnan().all() and lse.isnan().all()
    daf.daf_window_attention(q, k, v, out, lse, window=window, sinks=sinks)
    ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(n, heads, heads, dim, 1, window, sinks), dtype=torch.uint8, device="cuda")
    grads = [torch.zeros_like(q) for _ in range(3)]
    daf.daf_window_attention_backward(q, k, v, out, lse, bad, *grads, ws, window=window, sinks=sinks)
    assert all(t.isnan().all() for t in grads)
    bad = grad.clone()
    bad[-1, 0] = NAN                                                     # (the last query of one head)
    daf.daf_window_attention_backward(q, k, v, out, lse, bad, *grads, ws, window=window, sinks=sinks)
    seen = ref.seen(n, n, window, sinks)[-1].cuda()
    assert not grads[0][:-1].isnan().any() and grads[0][-1, 0].isnan().all() and not grads[0][-1, 1:].isnan().any()
    for t in grads[1:]:
        assert t[seen, 0].isnan().all() and not t[~seen, 0].isnan().any() and not t[:, 1:].isnan().any()


def test_a_cache_beyond_32_bits():
    """Keys that lie 5 GB into their cache: as those of a small cache."""
    far, rows, kv, dim = 1300000, 3000, 8, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)
    small = r(rows, 2 * kv, dim)
    large = torch.empty(far + rows, 2 * kv, dim, dtype=BF16, device="cuda")
    assert far * 2 * kv * dim * 2 > 1 << 32
    large[far:] = small
    q, starts, lengths, how = r(300, 16, dim), [0, 900, 2000], [800, 1100, 1000], dict(window=500, sinks=3)
    ws = torch.empty(daf.daf_window_attention_step_workspace_bytes(3, 16, kv, dim, far + rows, 500, 3), dtype=torch.uint8, device="cuda")
    results = []
    for cache, first in ((small, 0), (large, far)):
        k, v = cache[:, :kv], cache[:, kv:]
        out, lse, token = torch.zeros_like(q), torch.zeros(16, 300, device="cuda"), torch.zeros_like(q[:3])
        at = dict(k_starts=_int32(first + s for s in starts), k_lengths=_int32(lengths))
        daf.daf_window_attention(q, k, v, out, lse, q_starts=_int32([0, 10, 150, 300]), **at, **how)
        daf.daf_window_attention_step(q[:3], k, v, at["k_starts"], at["k_lengths"], token, ws, **how)
        results.append((out, lse, token))
    assert results[0][0].any() and all(torch.equal(a, b) for a, b in zip(*results))


def test_rows_beyond_32_bits():
    """Queries, keys, values and gradients 4.6 GB into one buffer, forward and backward: as in tensors of their own."""
    rows, heads, kv, dim, starts = 36000, 2, 1, 64, [0, 3, 34900, 35100, 35990]
    g = torch.Generator(device="cuda").manual_seed(5)
    counts = [heads, kv, kv, heads, heads, heads, kv, kv]               # q, k, v, out, grad_out and the gradients
    small = [torch.randn(rows, n, dim, generator=g, device="cuda").to(BF16) for n in counts]
    whole = torch.empty(rows, 1 << 16, dtype=BF16, device="cuda")
    large, at = [], 0
    for n, t in zip(counts, small):
        large.append(whole[:, at:at + n * dim].view(rows, n, dim))
        large[-1].copy_(t)
        at += n * dim
    results = []
    for q, k, v, out, grad, *grads in (small, large):
        lse = torch.zeros(heads, rows, device="cuda")
        ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(rows, heads, kv, dim, 4, 100, 2), dtype=torch.uint8, device="cuda")
        how = dict(q_starts=_int32(starts), window=100, sinks=2)
        daf.daf_window_attention(q, k, v, out, lse, **how)
        daf.daf_window_attention_backward(q, k, v, out, lse, grad, *grads, ws, **how)
        results.append([out, lse, *grads])
    assert all(torch.equal(a, b) for a, b in zip(*results)) and results[0][2][35500].any()


@pytest.mark.parametrize("heads,kv,dim,window,sinks", [(48, 48, 64, 100, 3), (44, 22, 128, 64, 33), (4, 2, 64, 100, 3)])
def test_sequences_that_overlap(heads, kv, dim, window, sinks):
    """Starts that decrease are no sequences, and what comes of their rows is not said: but nothing behind the workspace is read or written, nor any other row."""
    rows = 1300
    g = torch.Generator(device="cuda").manual_seed(6)
    r = lambda n: torch.randn(rows + 20, n, dim, generator=g, device="cuda").to(BF16)[:rows]
    q, k, v, grad = r(heads), r(kv), r(kv), r(heads)
    need = daf.daf_window_attention_backward_workspace_bytes(rows, heads, kv, dim, 3, window, sinks)
    behind = torch.full((need // 4 + (1 << 22),), 1e30, device="cuda")         # (a sum that is no number would be done again)
    ws = behind[:need // 4]
    ws.zero_()
    out, lse = torch.zeros_like(q), torch.zeros(heads, rows, device="cuda")
    grads = [torch.full((rows + 20, n, dim), 7.0, dtype=BF16, device="cuda") for n in (heads, kv, kv)]
    daf.daf_window_attention(q, k, v, out, lse, window=window, sinks=sinks, q_starts=_int32([0, rows]))
    daf.daf_window_attention_backward(q, k, v, out, lse, grad, *(t[:rows] for t in grads), ws, window=window, sinks=sinks, q_starts=_int32([0, rows, 0, rows]))
    torch.cuda.synchronize()
    assert all(t.abs().max() < 1e6 and (t[rows:] == 7.0).all() for t in grads) and (behind[need // 4:] == 1e30).all()


def test_one_workspace_for_smaller_calls():
    """Asked for once, for the most rows and sequences, and used for fewer: the same bits as with one of its own, and nothing behind it is touched."""
    heads, kv, dim, how = 4, 2, 128, dict(window=100, sinks=4)
    need = daf.daf_window_attention_backward_workspace_bytes(6000, heads, kv, dim, 64, 100, 4)
    step_need = daf.daf_window_attention_step_workspace_bytes(1200, heads, kv, dim, 6000, 0, 0)
    r = lambda n, h, g: torch.randn(n, h, dim, generator=g, device="cuda").to(BF16)
    for rows, starts in ((6000, list(range(0, 6001, 200)) + [6000]), (6000, [0, 5000, 6000]), (1500, [0, 1500]), (2000, [0, 700, 1400, 1990]), (40, [0, 40])):
        g = torch.Generator(device="cuda").manual_seed(rows)
        q, k, v, grad = r(rows, heads, g), r(rows, kv, g), r(rows, kv, g), r(rows, heads, g)
        out, lse = torch.zeros_like(q), torch.zeros(heads, rows, device="cuda")
        daf.daf_window_attention(q, k, v, out, lse, q_starts=_int32(starts), **how)
        own = daf.daf_window_attention_backward_workspace_bytes(rows, heads, kv, dim, len(starts) - 1, 100, 4)
        results = []
        for n in (own, need):
            ws = torch.full((n + 4096,), 90, dtype=torch.uint8, device="cuda")
            grads = [torch.zeros_like(t) for t in (q, k, v)]
            daf.daf_window_attention_backward(q, k, v, out, lse, grad, *grads, ws[:n], q_starts=_int32(starts), **how)
            assert (ws[n:] == 90).all() and own <= need, (rows, starts)
            results.append(grads)
        assert all(torch.equal(a, b) for a, b in zip(*results)) and all(t.any() for t in results[0])
    k, v = r(6000, kv, g), r(6000, kv, g)
    for sequences in (1, 5, 64, 300, 1200):
        q, starts, lengths = r(sequences, heads, g), [i % 50 for i in range(sequences)], [5900 - 4 * i for i in range(sequences)]
        own, results = daf.daf_window_attention_step_workspace_bytes(sequences, heads, kv, dim, 6000, 0, 0), []
        for n in (own, step_need):
            ws, out = torch.full((n + 4096,), 90, dtype=torch.uint8, device="cuda"), torch.zeros_like(q)
            daf.daf_window_attention_step(q, k, v, _int32(starts), _int32(lengths), out, ws[:n])
            assert (ws[n:] == 90).all() and own <= step_need, sequences
            results.append(out)
        assert torch.equal(*results) and results[0].any()


def test_step_without_a_workspace():
    """Where sequences are so many that none is cut a call needs none, though fewer would."""
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda n, h: torch.randn(n, h, 64, generator=g, device="cuda").to(BF16)
    k, v = r(2000, 8), r(2000, 8)
    for sequences, needs in ((6, True), (1200, False)):
        q, out, other = r(sequences, 16), *(torch.zeros(2, sequences, 16, 64, dtype=BF16, device="cuda"))
        starts, lengths = _int32(i % 40 for i in range(sequences)), _int32(1900 - i for i in range(sequences))
        ws = torch.zeros(daf.daf_window_attention_step_workspace_bytes(sequences, 16, 8, 64, 2000, 300), dtype=torch.uint8, device="cuda")
        daf.daf_window_attention_step(q, k, v, starts, lengths, out, ws, window=300)
        assert ws.numel() > 0 and out.any()
        if needs:
            with pytest.raises(ValueError, match="workspace"):
                daf.daf_window_attention_step(q, k, v, starts, lengths, other, window=300)
            assert not other.any()
        else:
            daf.daf_window_attention_step(q, k, v, starts, lengths, other, window=300)
            assert torch.equal(out, other)


@pytest.mark.parametrize("dtype,heads,kv,dim", [(BF16, 8, 2, 128), (F16, 130, 130, 64), (F16, 6, 3, 64), (BF16, 5, 1, 80)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_heads_of_their_own(dtype, heads, kv, dim, window, sinks):
    """Heads one after the other, [heads, rows, dim] each: the bits of heads beside each other, and nothing else is written."""
    print("case", dtype, heads, kv, dim, window, sinks, flush=True)
    rows, starts = 700, [2, 3, 400, 400, 690]
    g = torch.Generator(device="cuda").manual_seed(7)
    r = lambda n: torch.randn(rows, n, dim, generator=g, device="cuda").to(dtype)
    q, k, v, grad, token = r(heads), r(kv), r(kv), r(heads), r(heads)[:3]
    how = dict(window=window, sinks=sinks, q_starts=_int32(starts))
    k_starts, k_lengths = _int32([0, 100, 300]), _int32([700, 1, 333])
    ws = torch.zeros(daf.daf_window_attention_backward_workspace_bytes(rows, heads, kv, dim, 4, window, sinks), dtype=torch.uint8, device="cuda")
    ws2 = torch.zeros(max(16, daf.daf_window_attention_step_workspace_bytes(3, heads, kv, dim, rows, window, sinks)), dtype=torch.uint8, device="cuda")
    beside = lambda t: t.clone()
    after = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    results = []
    for lay in (beside, after):
        outs = [lay(torch.full_like(t, 7.0)) for t in (q, q, k, v, q, token)]
        out, gq, gk, gv, cached, step = outs
        lse, x = torch.full((heads, rows), 7.0, device="cuda"), [lay(t) for t in (q, k, v)]
        assert lay is beside or (x[0].stride(0) == dim and x[0].stride(1) == rows * dim)
        daf.daf_window_attention(*x, out, lse, **how)
        daf.daf_window_attention_backward(*x, out, lse, lay(grad), gq, gk, gv, ws, **how)
        daf.daf_window_attention(*x, cached, window=window, sinks=sinks, q_starts=_int32([0, 600, 601, 700]), k_starts=k_starts, k_lengths=k_lengths)
        daf.daf_window_attention_step(lay(token), *x[1:], k_starts, k_lengths, step, ws2, window=window, sinks=sinks)
        results.append([*outs, lse])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert all((t[:2] == 7.0).all() and (t[690:] == 7.0).all() and (t[2:690] != 7.0).any() for t in results[1][:4])


def test_a_thousand_sequences():
    """Documents of 0 to 80 rows, forward and backward, with far more sequences than tiles of 128 queries hold."""
    g = torch.Generator().manual_seed(13)
    lengths = torch.randint(0, 81, (1000,), generator=g).tolist()
    starts = [1]
    for n in lengths:
        starts.append(starts[-1] + n)
    _forward(BF16, 2, 1, 64, starts, 30, 2)
    _backward(BF16, 2, 1, 64, starts, 30, 2)
    _forward(F16, 1, 1, 128, starts, 0, 0)
    _backward(F16, 1, 1, 128, starts, 0, 0)
    _step(BF16, 1000, 4, 2, 64, lengths, 50, 1)

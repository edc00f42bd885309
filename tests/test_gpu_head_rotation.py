"""daf_head_rotation and its backward pass against the formulas in 64 bits.

Bounds: one rounding to the element's format, and binary32 arithmetic, of which every operation on the way may add 2^-24 of what it works on.  A value is
fewer than 64 such operations deep (a lane's 16 elements, the lanes of a head, the norm and the rotation); a weight's gradient adds up as many terms as
there are tokens and heads."""
import pytest
import torch

import paper_2507_07149_amd as daf
from tests import attention_reference as ref
from tests.block_reference import TINY, UNIT, assert_within

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
DEPTH = 64 * 2.0 ** -24
NAN = float("nan")
EPS = 1e-5


def _tables(positions, rotary):
    rate = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / max(rotary, 1))
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def _fused(tensors, dtype):
    whole = torch.cat(tensors, 1).to(dtype).cuda()
    at, views = 0, []
    for t in tensors:
        views.append(whole[:, at:at + t.shape[1]])
        at += t.shape[1]
    return views


def _case(dtype, tokens, heads, kv, dim, rotary, pairing, norm, weights, cache=0, in_place=False, seed=0):
    print("case", dtype, tokens, heads, kv, dim, rotary, pairing, norm, weights, cache, flush=True)
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    q, k, v, gq, gk = (r(tokens, n, dim).to(dtype).double() for n in (heads, kv, kv, heads, kv))
    w = {n: (1 + r(dim) / 4).to(dtype).double() if weights else None for n in "qk"}
    dw = {n: None if t is None else t.to(dtype).cuda() for n, t in w.items()}
    cos, sin = _tables(50, rotary)
    position = torch.randint(0, 50, (tokens,), generator=g)
    c, s = cos[position].double(), sin[position].double()
    away = torch.zeros(tokens, dtype=torch.bool)
    given = position.clone()
    if tokens > 2:
        given[1], given[2] = -1, 50                              # tokens that pad a batch
        away[1:3] = True
    dq, dk, dv = _fused([q, k, v], dtype)
    how = dict(q_weight=dw["q"], k_weight=dw["k"], norm=norm, eps=EPS, pairing=pairing)
    where = (given.to(torch.int32).cuda(), cos.cuda(), sin.cuda())
    nan = lambda *s: torch.full(s, NAN, dtype=dtype, device="cuda")
    rows = torch.arange(tokens)
    more = {}
    if cache:
        rows = torch.randperm(cache, generator=g)[:tokens]
        named = rows.clone()
        if tokens > 4:
            named[3], named[4] = -1, cache                       # no rows of the cache
        out_k, out_v = nan(cache, kv, dim), nan(cache, kv, dim)
        more = dict(v=dv, out_v=out_v, rows=named.to(torch.int32).cuda())
    else:
        out_k = nan(tokens, kv, dim)
    out_q = nan(tokens, heads, dim)
    if in_place:
        out_q, out_k = dq, dk
    daf.daf_head_rotation(dq, dk, *where, out_q, out_k, **how, **more)
    u = UNIT[dtype]
    for name, x, got in (("q", q, out_q), ("k", k, out_k)):
        want, size = ref.head_rotation(x, c, s, w[name], norm, EPS, pairing)
        want, size = want.masked_fill(away[:, None, None], 0.0), size.masked_fill(away[:, None, None], 0.0)
        if name == "k" and cache:
            keep = torch.ones(tokens, dtype=torch.bool)
            keep[3:5] = False
            whole, whole_size = torch.full((cache, kv, dim), NAN, dtype=torch.float64), torch.zeros(cache, kv, dim, dtype=torch.float64)
            whole[rows[keep]], whole_size[rows[keep]] = want[keep], size[keep]
            values = torch.full((cache, kv, dim), NAN, dtype=torch.float64)
            values[rows[keep]] = v[keep]
            assert_within(more["out_v"], values, torch.zeros(()), "v")
            want, size = whole, whole_size
        assert_within(got, want, u * torch.nan_to_num(want).abs() + DEPTH * size + TINY[dtype], name)
    if cache:
        return
    dq, dk, dv = _fused([q, k, v], dtype)
    dgq, dgk = gq.to(dtype).cuda(), gk.to(dtype).cuda()
    oq, ok, ov = _fused([torch.full_like(t, NAN) for t in (q, k, v)], dtype)
    if in_place:
        oq, ok = dgq, dgk
    vector = lambda: torch.full((dim,), NAN, device="cuda") if norm else None
    wq, wk = vector(), vector()
    ws = torch.full((max(16, daf.daf_head_rotation_backward_workspace_bytes(tokens, heads, kv, dim)),), 255, dtype=torch.uint8, device="cuda")
    x = (dq, dk) if norm else (None, None)
    daf.daf_head_rotation_backward(*x, *where, dgq, dgk, oq, ok, ws, out_grad_q_weight=wq, out_grad_k_weight=wk, **how)
    for name, x, grad, got, got_w in (("q", q, gq, oq, wq), ("k", k, gk, ok, wk)):
        grad = grad.masked_fill(away[:, None, None], 0.0)
        want, want_w, size, size_w = ref.head_rotation_backward(x, grad, c, s, w[name], norm, EPS, pairing)
        assert_within(got, want, u * want.abs() + DEPTH * size + TINY[dtype], "gradient of " + name)
        if norm:
            assert_within(got_w, want_w, (DEPTH + tokens * x.shape[1] * 2.0 ** -24) * size_w, "gradient of the weight of " + name)
    assert torch.isnan(ov).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("pairing", ["halves", "pairs"])
@pytest.mark.parametrize("heads,kv,dim,rotary", [(32, 8, 128, 128), (12, 12, 64, 32), (3, 1, 80, 80), (1, 1, 8, 0), (5, 5, 24, 16), (2, 1, 256, 128), (7, 1, 136, 16),
                                                 (9, 3, 200, 192), (4, 2, 48, 0), (2, 2, 40, 32)])
def test_heads(dtype, pairing, heads, kv, dim, rotary):
    for tokens in (1, 7):
        _case(dtype, tokens, heads, kv, dim, rotary, pairing, True, True)
    _case(dtype, 65, heads, kv, dim, rotary, pairing, True, False, in_place=True)
    _case(dtype, 5, heads, kv, dim, rotary, pairing, False, False)
    _case(dtype, 9, heads, kv, dim, rotary, pairing, True, True, cache=40)
    _case(dtype, 1, heads, kv, dim, rotary, pairing, False, False, cache=3)


def test_many_tokens():
    _case(BF16, 9001, 3, 1, 64, 64, "halves", True, True)
    _case(F32, 5000, 2, 2, 32, 32, "pairs", True, True)


def test_no_tokens():
    e = lambda *s: torch.zeros(*s, dtype=BF16, device="cuda")
    cos, sin = (t.cuda() for t in _tables(5, 32))
    w = [torch.full((64,), NAN, device="cuda") for _ in range(2)]
    position = torch.zeros(0, dtype=torch.int32, device="cuda")
    daf.daf_head_rotation(e(0, 4, 64), e(0, 2, 64), position, cos, sin, e(0, 4, 64), e(0, 2, 64))
    daf.daf_head_rotation_backward(e(0, 4, 64), e(0, 2, 64), position, cos, sin, e(0, 4, 64), e(0, 2, 64), e(0, 4, 64), e(0, 2, 64), None,
                                   out_grad_q_weight=w[0], out_grad_k_weight=w[1])
    assert not w[0].any() and not w[1].any()


def test_nan_in_one_head_stays_there():
    g = torch.Generator().manual_seed(2)
    q, k = (torch.randn(6, 3, 64, generator=g).to(BF16).cuda() for _ in range(2))
    cos, sin = (t.cuda() for t in _tables(9, 64))
    position = torch.tensor([0, 1, 9, 3, -5, 8], dtype=torch.int32, device="cuda")
    q[0, 1, 3], k[2, 0], q[3, 2, 0] = NAN, NAN, float("inf")
    oq, ok = torch.zeros_like(q), torch.zeros_like(k)
    daf.daf_head_rotation(q, k, position, cos, sin, oq, ok)
    bad = torch.isnan(oq).any(-1)
    want = torch.zeros(6, 3, dtype=torch.bool)
    want[0, 1] = want[3, 2] = True
    assert torch.equal(bad.cpu(), want) and not ok[2].any() and not ok[4].any()


@pytest.mark.parametrize("pairing", ["halves", "pairs"])
@pytest.mark.parametrize("norm", [True, False])
def test_tables_without_rows(pairing, norm):
    """No token has a position: zeros, zero gradients, rows of the cache written, values copied; nothing is read of tables that have no rows."""
    g = torch.Generator().manual_seed(6)
    q, k, v, gq = (torch.randn(9, n, 64, generator=g).to(BF16).cuda() for n in (4, 2, 2, 4))
    position = torch.tensor([0, 1, -1, 5, 0, 0, 2 ** 31 - 1, -2 ** 31, 0], dtype=torch.int32, device="cuda")
    cos, sin = (torch.zeros(0, 16, device="cuda") for _ in range(2))
    nan = lambda *s: torch.full(s, NAN, dtype=BF16, device="cuda")
    oq, ok, ov, dq, dk = nan(9, 4, 64), nan(12, 2, 64), nan(12, 2, 64), nan(9, 4, 64), nan(9, 2, 64)
    rows = torch.arange(11, 2, -1, dtype=torch.int32, device="cuda")
    how = dict(norm=norm, pairing=pairing)
    daf.daf_head_rotation(q, k, position, cos, sin, oq, ok, v=v, out_v=ov, rows=rows, **how)
    assert not oq.any() and not ok[3:].any() and ok[:3].isnan().all() and torch.equal(ov[3:].flip(0), v)
    wq = torch.full((64,), NAN, device="cuda") if norm else None
    ws = torch.zeros(daf.daf_head_rotation_backward_workspace_bytes(9, 4, 2, 64), dtype=torch.uint8, device="cuda")
    daf.daf_head_rotation_backward(q, k, position, cos, sin, gq, k, dq, dk, ws, out_grad_q_weight=wq, **how)
    assert not dq.any() and not dk.any() and (wq is None or not wq.any())


@pytest.mark.parametrize("dtype,size", [(F32, 1e-20), (F32, 3e-21), (BF16, 1e-20), (F32, 1e-12), (BF16, 1.0), (F16, 1.0)])
def test_no_eps(dtype, size):
    """eps of 0, also where mean squares lie among binary32's subnormal numbers, which are 2^-149 apart: 2 dim roundings of half of that in the sum of squares, one in
    the mean, half of what they are of the mean in the root, twice in a gradient (rstd itself, and the normalized elements)."""
    g = torch.Generator().manual_seed(7)
    tokens, heads, kv, dim = 9, 4, 2, 64
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    q, k = ((r(tokens, n, dim) * size).to(dtype).double() for n in (heads, kv))
    gq, gk = (r(tokens, n, dim).to(dtype).double() for n in (heads, kv))
    cos, sin = _tables(20, 32)
    position = torch.arange(tokens)
    c, s = cos[position].double(), sin[position].double()
    where, dev = (position.to(torch.int32).cuda(), cos.cuda(), sin.cuda()), lambda t: t.to(dtype).cuda()
    oq, ok, dq, dk = (torch.full(t.shape, NAN, dtype=dtype, device="cuda") for t in (q, k, q, k))
    wq, ws = torch.full((dim,), NAN, device="cuda"), torch.zeros(daf.daf_head_rotation_backward_workspace_bytes(tokens, heads, kv, dim), dtype=torch.uint8, device="cuda")
    daf.daf_head_rotation(dev(q), dev(k), *where, oq, ok, eps=0.0)
    daf.daf_head_rotation_backward(dev(q), dev(k), *where, dev(gq), dev(gk), dq, dk, ws, eps=0.0, out_grad_q_weight=wq)
    for name, x, grad, got, got_grad, got_w in (("q", q, gq, oq, dq, wq), ("k", k, gk, ok, dk, None)):
        mean = x.square().mean(-1, keepdim=True)
        off = (2 * dim + dim) * 2.0 ** -150 / (mean * dim) / 2
        want, large = ref.head_rotation(x, c, s, None, True, 0.0, "halves")
        assert_within(got, want, UNIT[dtype] * want.abs() + (DEPTH + 2 * off) * large + TINY[dtype], name)
        want, want_w, large, large_w = ref.head_rotation_backward(x, grad, c, s, None, True, 0.0, "halves")
        assert_within(got_grad, want, UNIT[dtype] * want.abs() + (DEPTH + 6 * off) * large + TINY[dtype], "gradient of " + name)
        if got_w is not None:
            assert_within(got_w, want_w, (DEPTH + tokens * heads * 2.0 ** -24 + 2 * off.max()) * large_w, "gradient of the weight")


def test_gradients_against_differences():
    """sum(out * grad) a step to each side of q and of its weight, in binary32: 2^-24 of every element's rounding over the step, and the third derivative."""
    g = torch.Generator().manual_seed(3)
    q, k = torch.randn(20, 4, 64, generator=g).cuda(), torch.randn(20, 2, 64, generator=g).cuda()
    grad, w = torch.randn(20, 4, 64, generator=g).cuda(), (1 + torch.randn(64, generator=g) / 4).cuda()
    cos, sin = (t.cuda() for t in _tables(20, 48))
    position = torch.arange(20, dtype=torch.int32, device="cuda")
    dq, dw, h = torch.randn(20, 4, 64, generator=g).cuda(), torch.randn(64, generator=g).cuda(), 2.0 ** -8
    side = []
    for sign in (h, -h):
        oq, ok = torch.zeros_like(q), torch.zeros_like(k)
        daf.daf_head_rotation(q + sign * dq, k, position, cos, sin, oq, ok, q_weight=w + sign * dw)
        side.append(oq.double())
    slope = ((side[0] - side[1]) * grad.double()).sum().item() / (2 * h)
    gq, gk, gw, ws = torch.zeros_like(q), torch.zeros_like(k), torch.zeros(64, device="cuda"), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    daf.daf_head_rotation_backward(q, k, position, cos, sin, grad, torch.zeros_like(k), gq, gk, ws, q_weight=w, out_grad_q_weight=gw)
    got = (gq.double() * dq.double()).sum().item() + (gw.double() * dw.double()).sum().item()
    size = (side[0].abs() * grad.abs()).sum().item()
    assert abs(slope - got) <= size * (64 * 2.0 ** -24 / h + 32 * h * h), (slope, got, size)


def test_captured_and_replayed():
    g = torch.Generator(device="cuda").manual_seed(1)
    qkv = torch.randn(70, 12, 64, generator=g, device="cuda").to(BF16)
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    cos, sin = (t.cuda() for t in _tables(80, 64))
    position, rows = torch.arange(70, dtype=torch.int32, device="cuda"), torch.arange(69, -1, -1, dtype=torch.int32, device="cuda")
    w = (torch.randn(64, generator=g, device="cuda")).to(BF16)
    oq, ok, ov, gq, gk = torch.zeros_like(q), torch.zeros(90, 2, 64, dtype=BF16, device="cuda"), torch.zeros(90, 2, 64, dtype=BF16, device="cuda"), torch.zeros_like(q), torch.zeros_like(k)
    gw = [torch.zeros(64, device="cuda") for _ in range(2)]
    ws = torch.zeros(daf.daf_head_rotation_backward_workspace_bytes(70, 8, 2, 64), dtype=torch.uint8, device="cuda")

    def calls():
        daf.daf_head_rotation(q, k, position, cos, sin, oq, ok, q_weight=w, k_weight=w, v=v, out_v=ov, rows=rows)
        daf.daf_head_rotation_backward(q, k, position, cos, sin, q, k, gq, gk, ws, q_weight=w, k_weight=w, out_grad_q_weight=gw[0], out_grad_k_weight=gw[1])
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    outs = [oq, ok, ov, gq, gk, *gw]
    for _ in range(3):
        qkv.mul_(-0.75)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a[:70], b[:70]) for a, b in zip(replayed, outs))


def test_a_cache_beyond_32_bits():
    """Rows 5 GB into a cache, those of the rows that are the token's own, and no others."""
    tokens, kv, dim, far = 50, 8, 128, 1300000
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(tokens, n, dim, generator=g, device="cuda").to(BF16) for n in (16, kv, kv))
    cos, sin = (t.cuda() for t in _tables(tokens, dim))
    position = torch.arange(tokens, dtype=torch.int32, device="cuda")
    want_k, want_v, out_q = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q)
    daf.daf_head_rotation(q, k, position, cos, sin, out_q, want_k, v=v, out_v=want_v)
    cache = torch.empty(far + 2 * tokens, 2 * kv, dim, dtype=BF16, device="cuda")
    cache[far:] = 7.0
    rows = far + 2 * torch.arange(tokens, dtype=torch.int32, device="cuda")
    rows[3], rows[5] = -1, far + 2 * tokens                              # (not there)
    daf.daf_head_rotation(q, k, position, cos, sin, out_q, cache[:, :kv], v=v, out_v=cache[:, kv:], rows=rows)
    got, there = cache[far:], torch.ones(tokens, dtype=torch.bool, device="cuda")
    there[3] = there[5] = False
    assert torch.equal(got[::2, :kv][there], want_k[there]) and torch.equal(got[::2, kv:][there], want_v[there])
    assert (got[1::2] == 7.0).all() and (got[::2][~there] == 7.0).all()


@pytest.mark.parametrize("dtype,heads,kv,dim,rotary,pairing", [(BF16, 8, 2, 128, 128, "halves"), (F32, 6, 3, 64, 32, "pairs"), (F16, 5, 5, 80, 80, "halves")])
def test_heads_of_their_own(dtype, heads, kv, dim, rotary, pairing):
    """Heads one after the other, [heads, tokens, dim] each, and a cache of such heads: the bits of heads beside each other."""
    g = torch.Generator(device="cuda").manual_seed(8)
    tokens, cache = 75, 200
    r = lambda n, h: torch.randn(n, h, dim, generator=g, device="cuda").to(dtype)
    q, k, v, gq, gk = r(tokens, heads), r(tokens, kv), r(tokens, kv), r(tokens, heads), r(tokens, kv)
    cos, sin = (t.cuda() for t in _tables(80, rotary))
    position, rows = torch.arange(tokens, dtype=torch.int32, device="cuda") + 4, torch.arange(tokens, dtype=torch.int32, device="cuda") * 2 + 1
    w, ws = torch.randn(dim, generator=g, device="cuda").to(dtype), torch.zeros(daf.daf_head_rotation_backward_workspace_bytes(tokens, heads, kv, dim), dtype=torch.uint8, device="cuda")
    results = []
    for lay in (lambda t: t.clone(), lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)):
        outs = [lay(torch.full((n, h, dim), 7.0, dtype=dtype, device="cuda")) for n, h in ((tokens, heads), (cache, kv), (cache, kv), (tokens, heads), (tokens, kv))]
        wq = torch.zeros(dim, device="cuda")
        daf.daf_head_rotation(lay(q), lay(k), position, cos, sin, *outs[:2], q_weight=w, pairing=pairing, v=lay(v), out_v=outs[2], rows=rows)
        daf.daf_head_rotation_backward(lay(q), lay(k), position, cos, sin, lay(gq), lay(gk), *outs[3:], ws, q_weight=w, pairing=pairing, out_grad_q_weight=wq)
        results.append([*outs, wq])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert torch.equal(results[1][2][1:2 * tokens:2], v) and all((t[0::2] == 7.0).all() and (t[2 * tokens:] == 7.0).all() for t in results[1][1:3])

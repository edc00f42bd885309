"""The operators of daf_block.h in 64 bits, from their formulas, for the tests; and what rounding may cost."""
import math

import torch

# Largest relative error of one rounding to the format, and its smallest step.
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def assert_within(got, want, bound, what):
    """|got - want| <= bound element by element; NaN and infinities in the same places."""
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu().expand(want.shape)
    assert got.shape == want.shape, what
    finite = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    same = finite | torch.isnan(want)
    assert torch.equal(got[~same], want[~same]), f"{what}: infinities"
    off = (got - want).abs()[finite]
    over = off > bound[finite]
    assert not over.any(), f"{what}: {int(over.sum())} of {over.numel()} off, the worst {float((off / bound[finite].clamp(min=1e-300)).max()):.3g} times its bound"


# ---- norms ----
def unit_of(v, layer, eps):
    n = v.shape[1]
    mean = v.sum(1, keepdim=True) / n if layer else torch.zeros_like(v[:, :1])
    rstd = 1 / torch.sqrt(((v - mean) ** 2).sum(1, keepdim=True) / n + eps)
    return (v - mean) * rstd, mean, rstd


def gate_rows(gate, rows, cols):
    if gate is None:
        return torch.ones(rows, cols, dtype=torch.float64)
    gate = gate.reshape(-1, cols)
    return gate.repeat_interleave(rows // gate.shape[0], 0) if rows else gate[:0]


def residual_norm(r, z, layer, eps, post, pre_w, pre_b, post_w, post_b, gate, scale):
    """s, y, stats and the largest |value| that a rounding of each row's s and y can come from."""
    rows, cols = r.shape
    one, zero = torch.ones(cols, dtype=torch.float64), torch.zeros(cols, dtype=torch.float64)
    pw, pb, qw, qb = (d if v is None else v for v, d in ((pre_w, one), (pre_b, zero), (post_w, one), (post_b, zero)))
    stats = torch.zeros(rows, 4, dtype=torch.float64)
    s, size = r.clone(), r.abs()
    if z is not None:
        p, size_p = z, z.abs()
        if post:
            p, mean, rstd = unit_of(z, layer, eps)
            stats[:, 0:1], stats[:, 1:2] = mean, rstd
            size_p = (z.abs() + mean.abs() + z.abs().amax(1, keepdim=True)) * rstd * qw.abs() + qb.abs()
            p = p * qw + qb
        g = scale * gate_rows(gate, rows, cols)
        s = r + g * p
        size = r.abs() + g.abs() * size_p
    u, mean, rstd = unit_of(s, layer, eps)
    stats[:, 2:3], stats[:, 3:4] = mean, rstd
    size_y = (size + size.amax(1, keepdim=True)) * rstd * pw.abs() + pb.abs()
    return s, u * pw + pb, stats, size, size_y


def residual_norm_backward(s, z, stats, dy, ds, layer, post, pre_w, post_w, post_b, gate, scale):
    """Gradients by name, and for each the sum of the sizes of what it is added up from."""
    like = s if s is not None else ds
    rows, cols = like.shape
    one, zero = torch.ones(cols, dtype=torch.float64), torch.zeros(cols, dtype=torch.float64)
    pw, qw, qb = (d if v is None else v for v, d in ((pre_w, one), (post_w, one), (post_b, zero)))
    pm, pr, m, rs = (stats[:, i:i + 1] for i in range(4))
    out, size = {}, {}
    total = torch.zeros_like(like) if ds is None else ds.clone()
    size_t = total.abs()
    if dy is not None:
        u, n = (s - m) * rs, dy * pw
        mean_n = n.mean(1, keepdim=True) if layer else torch.zeros_like(m)
        mean_nu = (n * u).mean(1, keepdim=True)
        total = total + rs * (n - mean_n - u * mean_nu)
        size_u = (s.abs() + m.abs()) * rs
        size_t = size_t + rs * (n.abs() + n.abs().mean(1, keepdim=True) + size_u * (n * size_u).abs().mean(1, keepdim=True))
        out["pre_weight"], size["pre_weight"] = (dy * u).sum(0), (dy.abs() * size_u).sum(0)
        out["pre_bias"], size["pre_bias"] = dy.sum(0), dy.abs().sum(0)
    out["residual"], size["residual"] = total, size_t
    if z is None:
        return out, size
    g = gate_rows(gate, rows, cols)
    d, size_d = scale * total, abs(scale) * size_t
    v, size_v = (z, z.abs()) if not post else ((z - pm) * pr, (z.abs() + pm.abs()) * pr)
    p, size_p = (v, size_v) if not post else (v * qw + qb, size_v * qw.abs() + qb.abs())
    groups = 1 if gate is None else gate.reshape(-1, cols).shape[0]
    by_group = lambda t: t.reshape(groups, rows // groups, cols).sum(1)
    out["gate"], size["gate"] = by_group(d * p), by_group(size_d * size_p)
    q, size_q = d * g, size_d * g.abs()
    if post:
        out["post_weight"], size["post_weight"] = (q * v).sum(0), (size_q * size_v).sum(0)
        out["post_bias"], size["post_bias"] = q.sum(0), size_q.sum(0)
        n, size_n = q * qw, size_q * qw.abs()
        mean_n = n.mean(1, keepdim=True) if layer else torch.zeros_like(pm)
        q = pr * (n - mean_n - v * (n * v).mean(1, keepdim=True))
        size_q = pr * (size_n + size_n.mean(1, keepdim=True) + size_v * (size_n * size_v).mean(1, keepdim=True))
    out["z"], size["z"] = q, size_q
    return out, size


# ---- gated product ----
def activation(a, act):
    """act(a) and its derivative."""
    if act == "relu":
        return torch.where(a > 0, a, torch.zeros_like(a)), (a > 0).double()
    if act == "silu":
        p = torch.sigmoid(a)
        return a * p, p + a * p * (1 - p)
    if act == "gelu":
        p = torch.erfc(-a / math.sqrt(2)) / 2
        return a * p, p + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    c = 2 * math.sqrt(2 / math.pi)
    p = torch.sigmoid(c * (a + 0.044715 * a ** 3))
    return a * p, p + a * p * (1 - p) * c * (1 + 3 * 0.044715 * a * a)

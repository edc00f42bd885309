"""daf_attention.h's formulas in 64 bits on the CPU, with the sizes that its tests' bounds are made of: the sums of the absolute values of what is added up."""
import math

import torch


def rotate(x, cos, sin, pairing, back=False):
    """x [tokens, heads, dim] by the tokens' cos and sin [tokens, rotary / 2]; with absolute values of everything where cos and sin are negative no more."""
    r = 2 * cos.shape[1]
    c, s = cos[:, None], (-sin if back else sin)[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if pairing == "pairs" else (x[..., :r // 2], x[..., r // 2:r])
    y = x.clone()
    if pairing == "pairs":
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, a * s + b * c
    else:
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, a * s + b * c
    return y


def rotate_size(x, cos, sin, pairing):
    r = 2 * cos.shape[1]
    c, s, x = cos.abs()[:, None], sin.abs()[:, None], x.abs()
    y = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if pairing == "pairs" else (slice(0, r // 2), slice(r // 2, r))
    y[..., first], y[..., second] = x[..., first] * c + x[..., second] * s, x[..., first] * s + x[..., second] * c
    return y


def head_rotation(x, cos, sin, weight, norm, eps, pairing):
    """The rotated heads and their size."""
    if norm:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * (1.0 if weight is None else weight)
    return rotate(x, cos, sin, pairing), rotate_size(x, cos, sin, pairing)


def head_rotation_backward(x, grad, cos, sin, weight, norm, eps, pairing):
    """Gradients of the heads and of the weight, and their sizes."""
    g, size = rotate(grad, cos, sin, pairing, back=True), rotate_size(grad, cos, sin, pairing)
    if not norm:
        return g, None, size, None
    w = torch.ones(x.shape[-1], dtype=torch.float64) if weight is None else weight
    rstd = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    u = x * rstd
    inner, inner_size = (g * w * u).mean(-1, keepdim=True), (size * w.abs() * u.abs()).mean(-1, keepdim=True)
    return (g * w - u * inner) * rstd, (g * u).sum((0, 1)), (size * w.abs() + u.abs() * inner_size) * rstd, (size * u.abs()).sum((0, 1))


def sequences(q_rows, q_starts=None, k_starts=None, k_lengths=None):
    """(first query, queries, first key, keys)."""
    q_starts = [0, q_rows] if q_starts is None else list(q_starts)
    for b, (begin, end) in enumerate(zip(q_starts, q_starts[1:])):
        yield (begin, end - begin, begin, end - begin) if k_starts is None else (begin, end - begin, k_starts[b], k_lengths[b])


def seen(queries, keys, window, sinks):
    p, j = (torch.arange(queries) + keys - queries)[:, None], torch.arange(keys)[None]
    return (j <= p) & ((p - j < window if window else j <= p) | (j < sinks))


def _heads(t, h, at, n):
    return t[at:at + n, h]


def attention(q, k, v, window, sinks, scale, seqs, out, lse):
    """Fills out and lse (64 bits), and returns the size of out: sum of p |v|, and the largest sum of |q| |k| scale."""
    size, score_size = torch.zeros_like(out), 0.0
    for begin, n, k_begin, keys in seqs:
        mask = seen(n, keys, window, sinks)
        some = mask.any(1)
        for h in range(q.shape[1]):
            g = h // (q.shape[1] // k.shape[1])
            x, y, z = _heads(q, h, begin, n), _heads(k, g, k_begin, keys), _heads(v, g, k_begin, keys)
            x, y, z = x[some], torch.where(mask.any(0)[:, None], y, 0.0), torch.where(mask.any(0)[:, None], z, 0.0)
            s = (x @ y.T * scale).masked_fill(~mask[some], -math.inf)
            if s.numel():
                score_size = max(score_size, (x.abs() @ y.abs().T).max().item() * abs(scale))
            log = torch.logsumexp(s, 1) if keys else torch.zeros(0, dtype=s.dtype)
            p = (s - log[:, None]).exp()
            for t, value in ((out, p @ z), (size, p @ z.abs())):
                t[begin:begin + n, h] = 0.0
                t[begin:begin + n, h][some] = value
            lse[h, begin:begin + n] = -math.inf
            lse[h, begin:begin + n][some] = log
    return size, score_size


def attention_backward(q, k, v, out, lse, grad, window, sinks, scale, seqs):
    """Gradients of q, k and v from lse as it is, and for each its bound's parts: the sum of |dS| (or P) times what it is multiplied by; the sum of P times
    that and what dP and delta are sums of; the same of what delta = sum(grad * out) is a sum of alone, for out's rounding."""
    grads = [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]
    sizes, inner, of_delta = ([torch.zeros_like(g) for g in grads] for _ in range(3))
    score_size = 0.0
    for begin, n, _, _ in seqs:
        mask = seen(n, n, window, sinks)
        for h in range(q.shape[1]):
            g = h // (q.shape[1] // k.shape[1])
            x, o, d = (_heads(t, h, begin, n) for t in (q, out, grad))
            y, z = _heads(k, g, begin, n), _heads(v, g, begin, n)
            if n == 0:
                continue
            score_size = max(score_size, (x.abs() @ y.abs().T).max().item() * abs(scale))
            p = torch.where(mask, (x @ y.T * scale - lse[h, begin:begin + n, None]).exp(), 0.0)
            dp = d @ z.T
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
            small = p * (d * o).abs().sum(1, keepdim=True) * abs(scale)
            parts = p * (d.abs() @ z.abs().T) * abs(scale) + small
            rows = slice(begin, begin + n)
            grads[0][rows, h] = ds @ y
            sizes[0][rows, h], inner[0][rows, h], of_delta[0][rows, h] = ds.abs() @ y.abs(), parts @ y.abs(), small @ y.abs()
            grads[1][rows, g] += ds.T @ x
            sizes[1][rows, g] += ds.abs().T @ x.abs()
            inner[1][rows, g] += parts.T @ x.abs()
            of_delta[1][rows, g] += small.T @ x.abs()
            grads[2][rows, g] += p.T @ d
            sizes[2][rows, g] += p.T @ d.abs()
    return grads, sizes, inner, of_delta, score_size

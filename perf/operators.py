"""The operators of a transformer block's training step around its feed-forward part, as cases that can be timed and compared.

Three operators, with the calls that a training (or serving) program makes of them through `paper_2507_07149_amd`:

  gated     h = act(x Wg^T) * (x Wu^T), the gated feed-forward product, daf_gated_linear; and its backward pass,
            daf_gated_linear_backward, which either reads the two pre-activations that the forward pass wrote or computes
            them again from x (nothing but x is then kept from the forward pass, and h comes out once more for the
            gradient of the projection behind it)
  norm      s = r + scale * gate * post_norm(z), y = pre_norm(s): the norm behind a block, its gate and residual scale, the
            residual sum and the norm in front of the next block, daf_residual_norm; and its backward pass,
            daf_residual_norm_backward
  clip      the norm of all gradients of a model and their scaling to a largest norm, daf_clip_grad_norm

Sizes are those of the repository's benchmark configurations (16 sequences of 2048 tokens with 11008 columns and 4096 inside, 32 x 1024
and 8 x 197 tokens of 768 columns) and generic odd ones; `draw` gives further ones of the same ranges.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
BYTES = {"float32": 4, "float16": 2, "bfloat16": 2}
EPS = 1e-5


def _gated(direction, dtype, rows, cols, inner, act, saved):
    """`saved`: the two pre-activations are written by the forward pass and read by the backward pass."""
    return {"op": "gated", "direction": direction, "dtype": dtype, "rows": rows, "cols": cols, "inner": inner, "act": act, "saved": saved}


def _norm(direction, dtype, rows, cols, kind, post, gate, scale):
    """`post`: the block's output is normalized too.  `gate`: 0 none, 1 one value per column, g one row of values for each of g runs of rows."""
    return {"op": "norm", "direction": direction, "dtype": dtype, "rows": rows, "cols": cols, "kind": kind, "post": post, "gate": gate, "scale": scale}


def _clip(dtype, sizes, vectors, max_norm):
    """`sizes`: elements of the tensors, as "count x elements" pieces; `vectors`: binary32 tensors of that many elements beside them (norm
    weights, kept in binary32), one for each tensor; 0: none."""
    return {"op": "clip", "dtype": dtype, "sizes": sizes, "vectors": vectors, "max_norm": max_norm}


def listed():
    named = {
        # the gated MLP of an LLM, 16 sequences of 2048 tokens: the forward pass of a training step that keeps x alone, or a long prompt
        "gated_llm_bf16": _gated("forward", "bfloat16", 16 * 2048, 11008, 4096, "silu", False),
        # the same for one token of a sequence that is being generated: the weights are read once for it
        "gated_token_bf16": _gated("forward", "bfloat16", 1, 11008, 4096, "silu", False),
        # a small ViT batch of 8 images of 197 tokens, pre-activations kept for the backward pass
        "gated_vit_f16": _gated("forward", "float16", 8 * 197, 2048, 768, "gelu", True),
        # backward pass of the LLM's MLP at 4 sequences, pre-activations computed again
        "gated_backward_llm_bf16": _gated("backward", "bfloat16", 4 * 2048, 11008, 4096, "silu", False),
        # backward pass of a ViT/BERT layer at 32 sequences of 1024 tokens, pre-activations kept
        "gated_backward_vit_f16": _gated("backward", "float16", 32 * 1024, 2048, 768, "gelu", True),
        # widths that are no multiple of a tile or of a load: what a pruned or searched model brings
        "gated_backward_odd_bf16": _gated("backward", "bfloat16", 3 * 577, 1365, 511, "gelu_tanh", False),
        # a pre-norm LLM block: residual sum and the next norm
        "norm_llm_bf16": _norm("forward", "bfloat16", 16 * 2048, 4096, "rms", False, 0, 1.0),
        # a ViT block with a norm behind it and a learned gate per column
        "norm_vit_f16": _norm("forward", "float16", 8 * 197, 768, "layer", True, 1, 1.0),
        # backward pass of a block with norms on both sides and gates per sequence
        "norm_backward_llm_bf16": _norm("backward", "bfloat16", 16 * 2048, 4096, "rms", True, 16, 1.0),
        # backward pass in binary32, odd rows and columns
        "norm_backward_odd_f32": _norm("backward", "float32", 7 * 577, 1001, "layer", True, 1, 0.5),
        # gradients of the adapters of 12 layers, two pairs of 768 x 8 each: launches count
        "clip_adapters_f32": _clip("float32", "48x6144", 0, 1.0),
        # gradients of the three MLP matrices of two LLM layers, with a norm weight beside each
        "clip_llm_bf16": _clip("bfloat16", "6x45088768", 4096, 1.0),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A number of columns: whole tiles, whole loads, or any."""
    n, step = _log_uniform(rng, lo, hi), rng.choice([64, 8, 1])
    return max(step, n // step * step)


def draw(rng):
    op = rng.choice(["gated", "gated", "norm", "norm", "clip"])
    if op == "gated":
        direction, saved = rng.choice(["forward", "backward"]), rng.random() < 0.5
        cols, inner = _width(rng, 64, 11008), _width(rng, 64, 4096)
        rows = min(_log_uniform(rng, 1, 16 * 2048), int(4.4e12 / (12 * cols * inner)))
        return _gated(direction, rng.choice(["bfloat16", "float16"]), rows, cols, inner, rng.choice(["silu", "gelu", "gelu_tanh", "relu"]), saved)
    if op == "norm":
        cols = _width(rng, 64, 11008)
        rows = min(_log_uniform(rng, 1, 16 * 2048), 32768 * 4096 // cols)
        sequences = rng.choice([s for s in (2, 3, 4, 7, 8, 16) if s <= rows] or [1])
        gate = rng.choice([0, 1, sequences])
        rows -= rows % gate if gate > 1 else 0
        return _norm(rng.choice(["forward", "backward"]), rng.choice(list(DTYPES)), rows, cols, rng.choice(["rms", "layer"]), rng.random() < 0.5, gate,
                     rng.choice([1.0, 0.5, 0.1]))
    pieces = ["%dx%d" % (rng.choice([1, 2, 12, 36, 48]), _log_uniform(rng, 1, 1 << 21)) for _ in range(rng.randint(1, 4))]
    return _clip(rng.choice(list(DTYPES)), "+".join(pieces), rng.choice([0, 768, 1001]), rng.choice([1.0, 0.1, 1e6]))


def _sizes(case):
    return [int(n) for p in case["sizes"].split("+") for n in [p.split("x")[1]] * int(p.split("x")[0])]


def _pitch(n):
    """Elements of a tensor in a gradient bucket, where every tensor starts at a multiple of 64 elements."""
    return -(-n // 64) * 64


def _bucket(sizes, dtype, scale, g):
    """One flat buffer of gradients and the tensors in it; the elements between them are zero."""
    at, flat = 0, torch.zeros(sum(_pitch(n) for n in sizes), dtype=dtype, device="cuda")
    views = []
    for n in sizes:
        views.append(flat[at:at + n])
        views[-1].copy_(torch.randn(n, generator=g, device="cuda") * scale)
        at += _pitch(n)
    return flat, views


def _same_views(flat, sizes):
    at, views = 0, []
    for n in sizes:
        views.append(flat[at:at + n])
        at += _pitch(n)
    return views


def _outlier_columns(x, g):
    """Some columns of a transformer's activations are an order of magnitude larger than the others."""
    big = torch.rand(x.shape[1], generator=g, device="cuda") < 0.01
    return x * torch.where(big, 8.0, 1.0)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    dt = DTYPES[case["dtype"]]
    empty = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="cuda")
    s = {"case": case}
    if case["op"] == "gated":
        m, n, k = case["rows"], case["cols"], case["inner"]
        s["x"] = _outlier_columns(randn(m, k), g).to(dt)
        s["w_gate"], s["w_up"] = ((randn(n, k) / math.sqrt(k)).to(dt) for _ in range(2))
        if case["direction"] == "forward":
            s["h"] = empty(m, n)
            s["gate"], s["up"] = (empty(m, n), empty(m, n)) if case["saved"] else (None, None)
        else:
            s["grad_h"] = (randn(m, n) * (0.01 if dt == torch.float16 else 0.001)).to(dt)
            s["gate"], s["up"] = ((s["x"].float() @ w.float().t()).to(dt) if case["saved"] else None for w in (s["w_gate"], s["w_up"]))
            s["h"] = None if case["saved"] else empty(m, n)
            s["grad_x"], s["grad_w_gate"], s["grad_w_up"] = empty(m, k), empty(n, k), empty(n, k)
    elif case["op"] == "norm":
        m, n, groups = case["rows"], case["cols"], case["gate"]
        s["z"] = _outlier_columns(randn(m, n), g).to(dt)
        s["residual"] = (randn(m, n) * 2 + 0.25).to(dt)
        weight = lambda: (1 + 0.1 * randn(n)).to(dt)
        bias = lambda: (0.1 * randn(n)).to(dt) if case["kind"] == "layer" else None
        s["pre_weight"], s["pre_bias"] = weight(), bias()
        s["post_weight"], s["post_bias"] = (weight(), bias()) if case["post"] else (None, None)
        s["gate"] = (0.5 + 0.2 * randn(groups, n)).to(dt).reshape(-1, n) if groups else None
        s["y"], s["sum"], s["stats"] = empty(m, n), empty(m, n), empty(m, 4, dtype=torch.float32)
        if case["direction"] == "backward":
            s["grad_y"], s["grad_sum"] = ((randn(m, n) * 0.01).to(dt) for _ in range(2))
            total, _, s["stats"] = _plain_norm(s)                  # what the forward pass left behind
            s["sum"] = total.to(dt)
            s["grad_residual"], s["grad_z"] = empty(m, n), empty(m, n)
            vector = lambda like: None if like is None else empty(*like.shape, dtype=torch.float32)
            for name in ("pre_weight", "pre_bias", "post_weight", "post_bias", "gate"):
                s["grad_" + name] = vector(s[name])
    else:
        sizes = _sizes(case)
        vectors = [case["vectors"]] * (len(sizes) if case["vectors"] else 0)
        s["sizes"], s["vector_sizes"] = sizes, vectors
        s["flat"], views = _bucket(sizes, dt, 0.02, g)
        s["flat_vectors"], vector_views = _bucket(vectors, torch.float32, 0.02, g)
        s["out"], s["out_vectors"] = torch.zeros_like(s["flat"]), torch.zeros_like(s["flat_vectors"])
        s["norm"] = empty(1, dtype=torch.float32)
        s["pairs"] = list(zip(views + vector_views, _same_views(s["out"], sizes) + _same_views(s["out_vectors"], vectors)))
    if own:
        _keep(s)
    return s


def _keep(s):
    """What a program that makes these calls allocates once: workspaces, and the list of its gradients."""
    import paper_2507_07149_amd as daf
    case = s["case"]
    sizes = (case.get("rows"), case.get("cols"), case.get("inner"), DTYPES[case["dtype"]])
    if case["op"] == "gated":
        need = daf.daf_gated_linear_workspace_bytes(*sizes) if case["direction"] == "forward" else daf.daf_gated_linear_backward_workspace_bytes(*sizes)
    elif case["op"] == "norm":
        need = daf.daf_residual_norm_backward_workspace_bytes(case["rows"], case["cols"], max(case["gate"], 1))
    else:
        need = daf.daf_grad_norm_workspace_bytes()
        s["items"] = daf.grad_items(s["pairs"])
    s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")


# ---- plain forms ----
def _act_and_slope(a, act):
    """act(a) and its derivative."""
    if act == "relu":
        return a.clamp(min=0), (a > 0).to(a.dtype)
    if act == "silu":
        p = torch.sigmoid(a)
        return a * p, p * (1 + a * (1 - p))
    if act == "gelu":
        p = 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))
        return a * p, p + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (a + 0.044715 * a * a * a))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * c * (1 + 3 * 0.044715 * a * a)


def _plain_gated(s, case):
    dt = s["x"].dtype
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    if case["direction"] == "forward":
        a, u = x @ wg.t(), x @ wu.t()
        h = _act_and_slope(a, case["act"])[0] * u
        return {"h": h.to(dt), "gate": a.to(dt), "up": u.to(dt)} if case["saved"] else {"h": h.to(dt)}
    a, u = (s["gate"].float(), s["up"].float()) if case["saved"] else (x @ wg.t(), x @ wu.t())
    f, df = _act_and_slope(a, case["act"])
    dh = s["grad_h"].float()
    da, du = dh * u * df, dh * f
    out = {"grad_x": (da @ wg + du @ wu).to(dt), "grad_w_gate": (da.t() @ x).to(dt), "grad_w_up": (du.t() @ x).to(dt)}
    if not case["saved"]:
        out["h"] = (f * u).to(dt)
    return out


def _normalized(v, kind):
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    rstd = torch.rsqrt((v - mean).square().mean(-1, keepdim=True) + EPS)
    return mean, rstd


def _affine(v, weight, bias):
    v = v if weight is None else v * weight.float()
    return v if bias is None else v + bias.float()


def _gate_rows(s, rows):
    """The gate of each row (or one row for all), with the residual scale."""
    gate = s["gate"]
    if gate is None:
        return s["case"]["scale"]
    return s["case"]["scale"] * gate.float().repeat_interleave(rows // gate.shape[0], 0)


def _plain_norm(s):
    """The residual sum, the normalized sum and the statistics, in 32 bits."""
    case, z = s["case"], s["z"].float()
    zeros = torch.zeros(z.shape[0], 1, device=z.device)
    post_mean, post_rstd = _normalized(z, case["kind"]) if case["post"] else (zeros, zeros)
    p = _affine((z - post_mean) * post_rstd, s["post_weight"], s["post_bias"]) if case["post"] else z
    total = s["residual"].float() + _gate_rows(s, z.shape[0]) * p
    mean, rstd = _normalized(total, case["kind"])
    y = _affine((total - mean) * rstd, s["pre_weight"], s["pre_bias"])
    return total, y, torch.cat([post_mean, post_rstd, mean, rstd], 1)


def _norm_gradient(grad, unit, rstd, kind):
    """Gradient of unit = (v - mean) * rstd with respect to v."""
    grad = grad - unit * (grad * unit).mean(-1, keepdim=True) - (grad.mean(-1, keepdim=True) if kind == "layer" else 0)
    return grad * rstd


def _plain_norm_backward(s):
    case, dt = s["case"], s["z"].dtype
    post_mean, post_rstd, mean, rstd = s["stats"].split(1, 1)
    dy, z = s["grad_y"].float(), s["z"].float()
    unit = (s["sum"].float() - mean) * rstd
    total = s["grad_sum"].float() + _norm_gradient(dy * s["pre_weight"].float(), unit, rstd, case["kind"])
    out = {"grad_residual": total.to(dt), "grad_pre_weight": (dy * unit).sum(0)}
    if case["kind"] == "layer":
        out["grad_pre_bias"] = dy.sum(0)
    q = total * _gate_rows(s, z.shape[0])
    post_unit = (z - post_mean) * post_rstd if case["post"] else z
    if s["gate"] is not None:
        p = _affine(post_unit, s["post_weight"], s["post_bias"])
        out["grad_gate"] = (total * p * case["scale"]).reshape(s["gate"].shape[0], -1, z.shape[1]).sum(1)
    if case["post"]:
        out["grad_post_weight"] = (q * post_unit).sum(0)
        if case["kind"] == "layer":
            out["grad_post_bias"] = q.sum(0)
        q = _norm_gradient(q * s["post_weight"].float(), post_unit, post_rstd, case["kind"])
    out["grad_z"] = q.to(dt)
    return out


def _plain_clip(s):
    flat, vectors = s["flat"].float(), s["flat_vectors"]
    norm = (flat.square().sum() + vectors.square().sum()).sqrt()
    factor = (s["case"]["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return {"norm": norm.reshape(1), "out": (flat * factor).to(s["flat"].dtype), "out_vectors": vectors * factor}


# ---- one pass ----
def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "gated":
            return _plain_gated(s, case)
        if case["op"] == "norm":
            if case["direction"] == "backward":
                return _plain_norm_backward(s)
            total, y, stats = _plain_norm(s)
            return {"sum": total.to(s["z"].dtype), "y": y.to(s["z"].dtype), "stats": stats}
        return _plain_clip(s)
    import paper_2507_07149_amd as daf
    if case["op"] == "gated":
        if case["direction"] == "forward":
            daf.daf_gated_linear(s["x"], s["w_gate"], s["w_up"], case["act"], s["h"], s["workspace"], out_gate=s["gate"], out_up=s["up"])
            return {"h": s["h"], "gate": s["gate"], "up": s["up"]} if case["saved"] else {"h": s["h"]}
        daf.daf_gated_linear_backward(s["x"], s["w_gate"], s["w_up"], s["grad_h"], case["act"], s["grad_x"], s["grad_w_gate"], s["grad_w_up"],
                                      s["workspace"], gate=s["gate"], up=s["up"], out_h=s["h"])
        out = {"grad_x": s["grad_x"], "grad_w_gate": s["grad_w_gate"], "grad_w_up": s["grad_w_up"]}
        return out if case["saved"] else dict(out, h=s["h"])
    if case["op"] == "norm":
        if case["direction"] == "forward":
            daf.daf_residual_norm(s["residual"], s["y"], s["stats"], kind=case["kind"], eps=EPS, z=s["z"], out_residual=s["sum"],
                                  pre_weight=s["pre_weight"], pre_bias=s["pre_bias"], post=case["post"], post_weight=s["post_weight"],
                                  post_bias=s["post_bias"], gate=s["gate"], scale=case["scale"])
            return {"sum": s["sum"], "y": s["y"], "stats": s["stats"]}
        daf.daf_residual_norm_backward(s["sum"], s["grad_y"], s["stats"], s["grad_residual"], s["workspace"], kind=case["kind"], z=s["z"],
                                       grad_residual=s["grad_sum"], out_grad_z=s["grad_z"], pre_weight=s["pre_weight"], post=case["post"],
                                       post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"], scale=case["scale"],
                                       out_grad_pre_weight=s["grad_pre_weight"], out_grad_pre_bias=s["grad_pre_bias"],
                                       out_grad_post_weight=s["grad_post_weight"], out_grad_post_bias=s["grad_post_bias"],
                                       out_grad_gate=s["grad_gate"])
        names = ("grad_residual", "grad_z", "grad_pre_weight", "grad_pre_bias", "grad_post_weight", "grad_post_bias", "grad_gate")
        return {name: s[name] for name in names if s[name] is not None}
    daf.daf_clip_grad_norm(s["items"], case["max_norm"], s["norm"], s["workspace"])
    return {"norm": s["norm"], "out": s["out"], "out_vectors": s["out_vectors"]}


# ---- what a pass cannot do without ----
def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "gated":
        m, n, k = case["rows"], case["cols"], case["inner"]
        inputs, product = m * k + 2 * n * k, 2 * m * n * k
        if case["direction"] == "forward":
            return {"bytes": e * (inputs + m * n * (3 if case["saved"] else 1)), "flops": 2 * product}
        # grad_h, and the kept pre-activations or h again; products: two for x's gradient, two for the weights', two computed again
        return {"bytes": e * (2 * inputs + m * n * (3 if case["saved"] else 2)), "flops": product * (4 if case["saved"] else 6)}
    if case["op"] == "norm":
        m, n = case["rows"], case["cols"]
        parameters = (1 + case["post"]) * (2 if case["kind"] == "layer" else 1) * n + case["gate"] * n
        if case["direction"] == "forward":
            return {"bytes": e * (4 * m * n + parameters) + 16 * m, "flops": m * n * (20 if case["post"] else 12)}
        return {"bytes": e * (6 * m * n + parameters) + 16 * m + 4 * parameters, "flops": m * n * (30 if case["post"] else 18)}
    sizes = _sizes(case)
    vectors = case["vectors"] * len(sizes)
    return {"bytes": 2 * (e * sum(sizes) + 4 * vectors) + 4, "flops": 3 * (sum(sizes) + vectors)}


# ---- the definitions in 64 bits ----
def _exact_act(a, act):
    if act == "relu":
        return torch.where(a > 0, a, torch.zeros_like(a))
    if act == "silu":
        return a / (1 + torch.exp(-a))
    if act == "gelu":
        return a * torch.erfc(-a / math.sqrt(2.0)) / 2
    return a / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)))


def _exact_slope(a, act):
    if act == "relu":
        return torch.where(a > 0, torch.ones_like(a), torch.zeros_like(a))
    if act == "silu":
        e = torch.exp(-a)
        return (1 + e + a * e) / (1 + e) ** 2
    if act == "gelu":
        return torch.erfc(-a / math.sqrt(2.0)) / 2 + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    c = 2 * math.sqrt(2 / math.pi)
    p = 1 / (1 + torch.exp(-c * (a + 0.044715 * a ** 3)))
    return p + a * p * (1 - p) * c * (1 + 0.134145 * a ** 2)


def _exact_unit(v, kind):
    """v normalized over its rows, with mean and 1 / standard deviation."""
    n = v.shape[1]
    mean = v.sum(1, keepdim=True) / n if kind == "layer" else torch.zeros(v.shape[0], 1, dtype=v.dtype, device=v.device)
    rstd = 1 / torch.sqrt(((v - mean) ** 2).sum(1, keepdim=True) / n + EPS)
    return (v - mean) * rstd, mean, rstd


def _exact_norm_gradient(g, unit, rstd, kind):
    n = g.shape[1]
    inner = unit * ((g * unit).sum(1, keepdim=True) / n)
    if kind == "layer":
        inner = inner + g.sum(1, keepdim=True) / n
    return rstd * (g - inner)


def exact(case, seed):
    s = prepare(case, seed)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] == "gated":
        act = case["act"]
        if case["direction"] == "backward" and case["saved"]:
            a, u = d["gate"], d["up"]
        else:
            a, u = torch.matmul(d["x"], d["w_gate"].T), torch.matmul(d["x"], d["w_up"].T)
        if case["direction"] == "forward":
            h = _exact_act(a, act) * u
            return {"h": h, "gate": a, "up": u} if case["saved"] else {"h": h}
        da, du = d["grad_h"] * u * _exact_slope(a, act), d["grad_h"] * _exact_act(a, act)
        out = {"grad_x": torch.matmul(da, d["w_gate"]) + torch.matmul(du, d["w_up"]), "grad_w_gate": torch.matmul(da.T, d["x"]),
               "grad_w_up": torch.matmul(du.T, d["x"])}
        return out if case["saved"] else dict(out, h=_exact_act(a, act) * u)
    if case["op"] == "norm":
        rows, kind = case["rows"], case["kind"]
        gate = case["scale"] * (d["gate"][torch.arange(rows, device="cuda") // (rows // case["gate"])] if case["gate"] else torch.ones(1, 1, device="cuda").double())
        weight, bias = d.get("post_weight"), d.get("post_bias", 0.0)
        if case["direction"] == "forward":
            zeros = torch.zeros(rows, 1, device="cuda").double()
            p, post_mean, post_rstd = _exact_unit(d["z"], kind) if case["post"] else (d["z"], zeros, zeros)
            total = d["residual"] + gate * (p * weight + bias if case["post"] else p)
            unit, mean, rstd = _exact_unit(total, kind)
            return {"sum": total, "y": unit * d["pre_weight"] + d.get("pre_bias", 0.0), "stats": torch.cat([post_mean, post_rstd, mean, rstd], 1)}
        post_mean, post_rstd, mean, rstd = (d["stats"][:, i:i + 1] for i in range(4))
        unit = (d["sum"] - mean) * rstd
        total = d["grad_sum"] + _exact_norm_gradient(d["grad_y"] * d["pre_weight"], unit, rstd, kind)
        p = (d["z"] - post_mean) * post_rstd if case["post"] else d["z"]
        q = total * gate
        out = {"grad_residual": total, "grad_pre_weight": torch.sum(d["grad_y"] * unit, 0)}
        if kind == "layer":
            out["grad_pre_bias"] = d["grad_y"].sum(0)
        if case["gate"]:
            whole = case["scale"] * total * (p * weight + bias if case["post"] else p)
            out["grad_gate"] = whole.view(case["gate"], rows // case["gate"], -1).sum(1)
        if case["post"]:
            out["grad_post_weight"] = torch.sum(q * p, 0)
            if kind == "layer":
                out["grad_post_bias"] = q.sum(0)
            q = _exact_norm_gradient(q * weight, p, post_rstd, kind)
        return dict(out, grad_z=q)
    norm = torch.sqrt(torch.sum(d["flat"] ** 2) + torch.sum(d["flat_vectors"] ** 2))
    factor = torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0)
    return {"norm": norm.reshape(1), "out": d["flat"] * factor, "out_vectors": d["flat_vectors"] * factor}

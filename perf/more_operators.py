"""The operators of a transformer block's attention half, as cases that can be timed and compared.

Two operators, with the calls that a training (or serving) program makes of them through `paper_2507_07149_amd`:

  rotation   the norm of every head of queries and keys and the rotation by position, in one pass over the projection's result,
             daf_head_rotation; with a cache, keys and values go straight to its rows; and its backward pass, daf_head_rotation_backward
  attention  causal attention with a window and a few first tokens that stay visible (sinks), over packed sequences or over a cache that
             holds a prompt's earlier part, daf_window_attention; its backward pass, daf_window_attention_backward; and its form for one
             token of each of many sequences, daf_window_attention_step

Sizes are those of the repository's benchmark configurations (16 sequences of 2048 tokens with 4096 columns, 32 x 1024 and 8 x 197 tokens of
768 columns) and generic odd ones; `draw` gives further ones of the same ranges.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
BYTES = {"float32": 4, "float16": 2, "bfloat16": 2}
EPS = 1e-6
POSITIONS = 4096                                                         # rows of the rotation's tables


def _rotation(direction, dtype, tokens, q_heads, kv_heads, dim, rotary, pairing, norm, cache):
    """`rotary`: elements of a head that rotate.  `cache`: rows of the cache that keys and values go to; 0: tensors of their own."""
    return {"op": "rotation", "direction": direction, "dtype": dtype, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "rotary": rotary, "pairing": pairing, "norm": norm, "cache": cache}


def _attention(direction, dtype, lengths, cached, q_heads, kv_heads, dim, window, sinks):
    """`lengths`: queries of the packed sequences, as "count x length" pieces.  `cached`: up to so many keys of each sequence come from earlier
    calls, and lie in a cache with the new ones; 0: the keys are the queries' tokens.  `window` 0: all tokens before."""
    return {"op": "attention", "direction": direction, "dtype": dtype, "lengths": lengths, "cached": cached, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "window": window, "sinks": sinks}


def _step(dtype, sequences, longest, q_heads, kv_heads, dim, window, sinks):
    """One token of each of `sequences` sequences, the longest of `longest` tokens, the shortest half as long."""
    return {"op": "step", "dtype": dtype, "sequences": sequences, "longest": longest, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "window": window, "sinks": sinks}


def listed():
    named = {
        # heads of an LLM block's projection, 16 sequences of 2048 tokens: forward pass of a training step, or long prompts
        "rotation_llm_bf16": _rotation("forward", "bfloat16", 16 * 2048, 32, 8, 128, 128, "halves", True, 0),
        # the same for one token of a sequence that is being generated, into its cache: the launch counts
        "rotation_token_bf16": _rotation("forward", "bfloat16", 1, 32, 8, 128, 128, "halves", True, 4096),
        # backward pass of the LLM's heads
        "rotation_backward_llm_bf16": _rotation("backward", "bfloat16", 16 * 2048, 32, 8, 128, 128, "halves", True, 0),
        # a small batch of 8 sequences of 197 tokens, 12 heads of 64 of which half the elements rotate, by neighbours
        "rotation_backward_vit_f16": _rotation("backward", "float16", 8 * 197, 12, 12, 64, 32, "pairs", True, 0),
        # an LLM's training step, forward: 16 sequences of 2048 tokens
        "attention_llm_bf16": _attention("forward", "bfloat16", "16x2048", 0, 32, 8, 128, 1024, 4),
        # one long document
        "attention_long_bf16": _attention("forward", "bfloat16", "1x32768", 0, 32, 8, 128, 4096, 4),
        # pieces of prompts of odd lengths over what the cache holds of them, heads of 80
        "attention_ragged_bf16": _attention("forward", "bfloat16", "1x1+2x197+1x511+3x1001+1x2047", 2900, 20, 4, 80, 1500, 1),
        # an LLM's training step, backward: 8 sequences of 2048 tokens
        "attention_backward_llm_bf16": _attention("backward", "bfloat16", "8x2048", 0, 32, 8, 128, 1024, 4),
        # documents of odd lengths packed into one row of 12 heads of 64, no window
        "attention_backward_ragged_f16": _attention("backward", "float16", "9x197+2x1024+1x577+5x33+1x1", 0, 12, 12, 64, 0, 0),
        # serving 64 sequences of 8192 ... 16384 tokens with a window
        "step_llm_bf16": _step("bfloat16", 64, 16384, 32, 8, 128, 4096, 4),
        # one sequence alone, every token before it visible
        "step_alone_bf16": _step("bfloat16", 1, 8191, 32, 8, 128, 0, 0),
        # a few sequences of 12 heads of 64 without shared keys
        "step_vit_f16": _step("float16", 8, 1025, 12, 12, 64, 512, 2),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most=40):
    kv = rng.choice([1, 2, 3, 4, 5, 8, 12])
    return kv * rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8, 12) if kv * g <= most]), kv


LARGEST = 2.2e12                                                         # operations of the largest case


def draw(rng):
    op = rng.choice(["rotation", "attention", "attention", "attention", "step"])
    dtype = rng.choice(["bfloat16", "float16"])
    (q_heads, kv_heads), dim = _heads(rng), rng.choice([128, 128, 64, 64, 96, 80, 8 * rng.randint(2, 16)])
    if op == "rotation":
        dtype = rng.choice(list(DTYPES))
        cache = rng.random() < 0.4
        tokens = _log_uniform(rng, 1, 2048 if cache else 16 * 2048)
        tokens = min(tokens, 160 * 1024 * 1024 // ((q_heads + 2 * kv_heads) * dim))
        rotary = dim // 16 * 16 if rng.random() < 0.6 else 16 * rng.randint(1, dim // 16)
        return _rotation("forward" if cache else rng.choice(["forward", "backward"]), dtype, tokens, q_heads, kv_heads, dim, rotary,
                         rng.choice(["halves", "pairs"]), rng.random() < 0.8, tokens + _log_uniform(rng, 1, 4096) if cache else 0)
    window = rng.choice([0, _log_uniform(rng, 1, 4096), _log_uniform(rng, 64, 4096)])
    sinks = rng.choice([0, 1, 4, rng.randint(2, 130)])
    if op == "step":
        sequences, longest = _log_uniform(rng, 1, 128), _log_uniform(rng, 1, 16384)
        longest = max(1, min(longest, (1 << 30) // (sequences * kv_heads * dim)))
        return _step(dtype, sequences, longest, q_heads, kv_heads, dim, window, sinks)
    direction = rng.choice(["forward", "backward"])
    pieces, tokens = [], 0
    for _ in range(rng.randint(1, 4)):
        count, length = rng.choice([1, 1, 2, 5, 16]), _log_uniform(rng, 1, 8192)
        if tokens + count * length <= 32768:
            pieces.append("%dx%d" % (count, length))
            tokens += count * length
    cached = _log_uniform(rng, 1, 4096) if direction == "forward" and rng.random() < 0.3 else 0
    case = _attention(direction, dtype, "+".join(pieces or ["1x300"]), cached, q_heads, kv_heads, dim, window, sinks)
    while work(case)["flops"] > LARGEST:
        case["lengths"] = "+".join(case["lengths"].split("+")[1:] or ["1x2049"])
    return case


# ---- inputs ----
def _lengths(case):
    return [int(n) for p in case["lengths"].split("+") for n in [p.split("x")[1]] * int(p.split("x")[0])]


def _sequences(case):
    """(queries, keys) of every sequence."""
    if case["op"] == "step":
        n, longest = case["sequences"], case["longest"]
        return [(1, longest - i * (longest // 2) // n) for i in range(n)]
    lengths = _lengths(case)
    return [(n, n + case["cached"] * (i + 1) // len(lengths)) for i, n in enumerate(lengths)]


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _tables(rotary):
    """cos and sin of position / 10000^(2 i / rotary), in 64 bits and rounded once."""
    rate = 10000.0 ** (-torch.arange(0, rotary, 2, device="cuda", dtype=torch.float64) / rotary)
    angle = torch.arange(POSITIONS, device="cuda", dtype=torch.float64)[:, None] * rate
    return angle.cos().float(), angle.sin().float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(dt)
    empty = lambda *shape, dtype=dt: torch.zeros(*shape, dtype=dtype, device="cuda")
    int32 = lambda values: torch.tensor(values, dtype=torch.int32, device="cuda")
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["dim"]
    s = {"case": case}
    if case["op"] == "rotation":
        n = case["tokens"]
        qkv = randn(n, hq + 2 * hkv, d) * 1.5
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]     # views of one projection's result
        s["cos"], s["sin"] = _tables(case["rotary"])
        weight = lambda: (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt) if case["norm"] else None
        s["q_weight"], s["k_weight"] = weight(), weight()
        if case["cache"]:
            s["position"] = torch.randint(POSITIONS, (n,), generator=g, device="cuda").to(torch.int32)
            s["rows"] = torch.randperm(case["cache"], generator=g, device="cuda")[:n].to(torch.int32)
            s["out_q"], s["out_k"], s["out_v"] = empty(n, hq, d), empty(case["cache"], hkv, d), empty(case["cache"], hkv, d)
        else:
            s["position"] = (torch.arange(n, device="cuda") % 2048).to(torch.int32)
            s["out_q"], s["out_k"] = empty(n, hq, d), empty(n, hkv, d)
        if case["direction"] == "backward":
            s["grad_q"], s["grad_k"] = randn(n, hq, d) * 0.01, randn(n, hkv, d) * 0.01
            grad = empty(n, hq + 2 * hkv, d)                              # the projection's gradient; attention writes that of v into it
            s["out_grad_q"], s["out_grad_k"] = grad[:, :hq], grad[:, hq:hq + hkv]
            s["out_grad_q_weight"], s["out_grad_k_weight"] = ((empty(d, dtype=torch.float32) if case["norm"] else None) for _ in range(2))
    elif case["op"] == "step":
        sequences = _sequences(case)
        pitch = case["longest"] + 1
        s["q"] = randn(len(sequences), hq, d)
        s["k"], s["v"] = randn(len(sequences) * pitch, hkv, d), randn(len(sequences) * pitch, hkv, d)
        s["starts"], s["lengths"] = [i * pitch for i in range(len(sequences))], [keys for _, keys in sequences]
        s["k_starts"], s["k_lengths"] = int32(s["starts"]), int32(s["lengths"])
        s["out"] = empty(len(sequences), hq, d)
    else:
        sequences = _sequences(case)
        s["starts"] = _starts([n for n, _ in sequences])
        tokens = s["starts"][-1]
        s["q_starts"] = int32(s["starts"])
        s["q"] = randn(tokens, hq, d)
        s["key_starts"], s["key_lengths"] = s["starts"][:-1], [keys for _, keys in sequences]
        s["k_starts"], s["k_lengths"] = None, None
        if case["cached"]:
            pitch = max(s["key_lengths"]) + 7                             # the cache has room for more
            s["key_starts"] = [i * pitch for i in range(len(sequences))]
            s["k_starts"], s["k_lengths"] = int32(s["key_starts"]), int32(s["key_lengths"])
            s["k"], s["v"] = randn(len(sequences) * pitch, hkv, d), randn(len(sequences) * pitch, hkv, d)
        else:
            s["k"] = randn(tokens, hkv, d)
            s["v"] = randn(tokens, hq + 2 * hkv, d)[:, hq + hkv:]         # v is read where the projection left it
        s["out"], s["lse"] = empty(tokens, hq, d), empty(hq, tokens, dtype=torch.float32)
        if case["direction"] == "backward":
            s["grad_out"] = randn(tokens, hq, d) * 0.05
            out, lse = _plain_attention(s)                                # what the forward pass left behind
            s["out"], s["lse"] = out.to(dt), lse
            s["grad_q"], s["grad_k"] = empty(tokens, hq, d), empty(tokens, hkv, d)
            s["grad_v"] = empty(tokens, hq + 2 * hkv, d)[:, hq + hkv:]
    if own:
        _keep(s)
    return s


def _keep(s):
    """What a program that makes these calls allocates once: workspaces."""
    import paper_2507_07149_amd as daf
    case, need = s["case"], 0
    if case["op"] == "rotation" and case["direction"] == "backward":
        need = daf.daf_head_rotation_backward_workspace_bytes(case["tokens"], case["q_heads"], case["kv_heads"], case["dim"])
    elif case["op"] == "attention" and case["direction"] == "backward":
        need = daf.daf_window_attention_backward_workspace_bytes(s["q"].shape[0], case["q_heads"], case["kv_heads"], case["dim"], len(s["starts"]) - 1,
                                                                 case["window"], case["sinks"])
    elif case["op"] == "step":
        need = daf.daf_window_attention_step_workspace_bytes(case["sequences"], case["q_heads"], case["kv_heads"], case["dim"], s["k"].shape[0],
                                                             case["window"], case["sinks"])
    s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")


# ---- plain forms ----
def _first_and_second(x, pairing):
    """The two members of every pair."""
    return (x[..., 0::2], x[..., 1::2]) if pairing == "pairs" else x.chunk(2, -1)


def _joined(a, b, pairing):
    return torch.stack([a, b], -1).flatten(-2) if pairing == "pairs" else torch.cat([a, b], -1)


def _turn(x, s, back=False):
    """Heads rotated by their tokens' angles (back: by minus them)."""
    case = s["case"]
    at = s["position"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    sin = -sin if back else sin
    a, b = _first_and_second(x[..., :case["rotary"]], case["pairing"])
    return torch.cat([_joined(a * cos - b * sin, a * sin + b * cos, case["pairing"]), x[..., case["rotary"]:]], -1)


def _plain_rotation(s):
    case, dt = s["case"], s["q"].dtype
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        if case["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * s[name + "_weight"].float()
        out[name] = _turn(x, s).to(dt)
    if case["cache"]:
        rows = s["rows"].long()
        s["out_k"][rows], s["out_v"][rows] = out["k"], s["v"]
        out["k"], out["v"] = s["out_k"], s["out_v"]
    return out


def _plain_rotation_backward(s):
    case, dt = s["case"], s["q"].dtype
    out = {}
    for name in ("q", "k"):
        grad = _turn(s["grad_" + name].float(), s, back=True)
        if case["norm"]:
            x = s[name].float()
            rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
            unit = x * rstd
            out[name + "_weight"] = (grad * unit).sum((0, 1))
            grad = grad * s[name + "_weight"].float()
            grad = (grad - unit * (grad * unit).mean(-1, keepdim=True)) * rstd
        out[name] = grad.to(dt)
    return out


ROWS = 1024                                                              # queries at a time in the plain form


def _blocks(s):
    """(slice of the queries, rows of their keys, mask of what each sees) for pieces of every sequence."""
    case = s["case"]
    window, sinks = case["window"], case["sinks"]
    for i, keys in enumerate(s["key_lengths"]):
        begin, end = s["starts"][i], s["starts"][i + 1]
        for at in range(begin, end, ROWS):
            stop = min(at + ROWS, end)
            first, last = keys - (end - at), keys - (end - stop) - 1      # positions of the piece's first and last query
            low = max(0, first - window + 1) if window else 0
            j = torch.cat([torch.arange(min(sinks, low), device="cuda"), torch.arange(low, last + 1, device="cuda")])
            p = torch.arange(first, last + 1, device="cuda")[:, None]
            seen = j <= p
            if window:
                seen = seen & ((p - j < window) | (j < sinks))
            yield slice(at, stop), s["key_starts"][i] + j, seen


def _grouped(x, kv_heads):
    """[rows, heads, dim] as [kv heads, heads of each x rows, dim]."""
    return x.float().transpose(0, 1).reshape(kv_heads, -1, x.shape[2])


def _probabilities(q, k, seen, scale):
    """Softmax over the visible keys and its logarithm's denominator; q [kv heads, heads x rows, dim], k [kv heads, keys, dim]."""
    score = torch.matmul(q, k.transpose(1, 2)) * scale
    score = score.view(score.shape[0], -1, *seen.shape).masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    return (p / total).flatten(1, 2), (top + torch.log(total))[..., 0]


def _plain_attention(s):
    hq, hkv, d = s["q"].shape[1], s["k"].shape[1], s["q"].shape[2]
    out = torch.empty(*s["q"].shape, device="cuda")
    lse = torch.empty(hq, s["q"].shape[0], device="cuda")
    for rows, keys, seen in _blocks(s):
        p, log = _probabilities(_grouped(s["q"][rows], hkv), _grouped(s["k"][keys], hkv), seen, 1 / math.sqrt(d))
        o = torch.matmul(p, _grouped(s["v"][keys], hkv))
        out[rows] = o.reshape(hq, -1, d).transpose(0, 1)
        lse[:, rows] = log.reshape(hq, -1)
    return out, lse


def _plain_attention_backward(s):
    hq, hkv, d, dt = s["q"].shape[1], s["k"].shape[1], s["q"].shape[2], s["q"].dtype
    scale = 1 / math.sqrt(d)
    grad_q = torch.empty(*s["q"].shape, device="cuda")
    grad_k, grad_v = (torch.zeros(hkv, s["k"].shape[0], d, device="cuda") for _ in range(2))
    for rows, keys, seen in _blocks(s):
        q, k, v, grad = (_grouped(t, hkv) for t in (s["q"][rows], s["k"][keys], s["v"][keys], s["grad_out"][rows]))
        p, _ = _probabilities(q, k, seen, scale)
        grad_p = torch.matmul(grad, v.transpose(1, 2))
        grad_s = p * (grad_p - (p * grad_p).sum(-1, keepdim=True)) * scale
        grad_q[rows] = torch.matmul(grad_s, k).reshape(hq, -1, d).transpose(0, 1)
        grad_k[:, keys] += torch.matmul(grad_s.transpose(1, 2), q)
        grad_v[:, keys] += torch.matmul(p.transpose(1, 2), grad)
    return {"grad_q": grad_q.to(dt), "grad_k": grad_k.transpose(0, 1).to(dt), "grad_v": grad_v.transpose(0, 1).to(dt)}


def _plain_step(s):
    hkv, d, dt = s["k"].shape[1], s["q"].shape[2], s["q"].dtype
    window, sinks = s["case"]["window"], s["case"]["sinks"]
    out = torch.empty(*s["q"].shape, device="cuda")
    for i, (start, keys) in enumerate(zip(s["starts"], s["lengths"])):
        low = max(0, keys - window) if window else 0
        pick = lambda t: torch.cat([t[start:start + min(sinks, low)], t[start + low:start + keys]])
        k, v = _grouped(pick(s["k"]), hkv), _grouped(pick(s["v"]), hkv)
        seen = torch.ones(1, k.shape[1], dtype=torch.bool, device="cuda")
        p, _ = _probabilities(_grouped(s["q"][i:i + 1], hkv), k, seen, 1 / math.sqrt(d))
        out[i] = torch.matmul(p, v).reshape(-1, d)
    return {"out": out.to(dt)}


# ---- one pass ----
def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "rotation":
            return _plain_rotation(s) if case["direction"] == "forward" else _plain_rotation_backward(s)
        if case["op"] == "step":
            return _plain_step(s)
        if case["direction"] == "backward":
            return _plain_attention_backward(s)
        out, lse = _plain_attention(s)
        return {"out": out.to(s["q"].dtype), "lse": lse}
    import paper_2507_07149_amd as daf
    if case["op"] == "rotation":
        how = {"q_weight": s["q_weight"], "k_weight": s["k_weight"], "norm": case["norm"], "eps": EPS, "pairing": case["pairing"]}
        if case["direction"] == "forward":
            if case["cache"]:
                how.update(v=s["v"], out_v=s["out_v"], rows=s["rows"])
            daf.daf_head_rotation(s["q"], s["k"], s["position"], s["cos"], s["sin"], s["out_q"], s["out_k"], **how)
            out = {"q": s["out_q"], "k": s["out_k"]}
            return dict(out, v=s["out_v"]) if case["cache"] else out
        daf.daf_head_rotation_backward(s["q"], s["k"], s["position"], s["cos"], s["sin"], s["grad_q"], s["grad_k"], s["out_grad_q"], s["out_grad_k"],
                                       s["workspace"], out_grad_q_weight=s["out_grad_q_weight"], out_grad_k_weight=s["out_grad_k_weight"], **how)
        if not case["norm"]:
            return {"q": s["out_grad_q"], "k": s["out_grad_k"]}
        return {"q_weight": s["out_grad_q_weight"], "q": s["out_grad_q"], "k_weight": s["out_grad_k_weight"], "k": s["out_grad_k"]}
    how = {"window": case["window"], "sinks": case["sinks"]}
    if case["op"] == "step":
        daf.daf_window_attention_step(s["q"], s["k"], s["v"], s["k_starts"], s["k_lengths"], s["out"], s["workspace"], **how)
        return {"out": s["out"]}
    if case["direction"] == "forward":
        daf.daf_window_attention(s["q"], s["k"], s["v"], s["out"], s["lse"], q_starts=s["q_starts"], k_starts=s["k_starts"], k_lengths=s["k_lengths"],
                                 **how)
        return {"out": s["out"], "lse": s["lse"]}
    daf.daf_window_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["grad_out"], s["grad_q"], s["grad_k"], s["grad_v"], s["workspace"],
                                      q_starts=s["q_starts"], **how)
    return {"grad_q": s["grad_q"], "grad_k": s["grad_k"], "grad_v": s["grad_v"]}


# ---- what a pass cannot do without ----
def _seen_of(keys, position, window, sinks):
    """Keys that the query at `position` sees."""
    if window == 0 or position < window:
        return position + 1
    return window + min(sinks, position + 1 - window)


def work(case):
    e, hq, hkv, d = BYTES[case["dtype"]], case["q_heads"], case["kv_heads"], case["dim"]
    if case["op"] == "rotation":
        n, heads = case["tokens"], hq + hkv
        beside = n * 4 + min(n, POSITIONS if case["cache"] else 2048) * case["rotary"] * 4 + 2 * d * e * case["norm"]
        if case["direction"] == "forward":
            return {"bytes": 2 * e * n * d * (heads + (hkv if case["cache"] else 0)) + beside + (4 * n if case["cache"] else 0),
                    "flops": n * heads * d * (7 if case["norm"] else 3)}
        return {"bytes": e * n * heads * d * (3 if case["norm"] else 2) + beside + 8 * d * case["norm"], "flops": n * heads * d * (14 if case["norm"] else 3)}
    window, sinks = case["window"], case["sinks"]
    pairs, touched, queries = 0, 0, 0
    for n, keys in _sequences(case):
        first = keys - n
        edge = min(max(first, window), keys) if window else keys           # positions from here on see a window and sinks
        pairs += (first + 1 + edge) * (edge - first) // 2
        pairs += sum(_seen_of(keys, p, window, sinks) for p in range(edge, keys)) if sinks and edge < keys else (keys - edge) * window
        low = max(0, first - window + 1) if window else 0
        touched += keys - low + min(sinks, low)
        queries += n
    reads = e * d * (queries * hq + 2 * touched * hkv)
    if case["op"] == "step" or case["direction"] == "forward":
        return {"bytes": reads + e * d * queries * hq + (0 if case["op"] == "step" else 4 * hq * queries), "flops": 4 * d * hq * pairs}
    # out, its gradient and lse beside q, k and v; the gradients of q, k and v; five products
    return {"bytes": reads + e * d * (3 * queries * hq + 2 * touched * hkv) + 4 * hq * queries, "flops": 10 * d * hq * pairs}


# ---- the definitions in 64 bits ----
def _exact_partner(x, rotary, pairing, sign):
    """The other member of every element's pair, with the sign that the rotation gives it."""
    i = torch.arange(rotary, device="cuda")
    if pairing == "pairs":
        other, first = i ^ 1, (i & 1) == 0
    else:
        other, first = (i + rotary // 2) % rotary, i < rotary // 2
    return x[..., other] * torch.where(first, -sign, sign).to(x.dtype)


def _exact_turn(x, s, sign):
    case = s["case"]
    r = case["rotary"]
    i = torch.arange(r, device="cuda")
    angle = i // 2 if case["pairing"] == "pairs" else i % (r // 2)
    at = s["position"].long()
    cos, sin = (s[t].double()[at][:, angle].unsqueeze(1) for t in ("cos", "sin"))
    y = x.clone()
    y[..., :r] = x[..., :r] * cos + _exact_partner(x[..., :r], r, case["pairing"], sign) * sin
    return y


def _exact_rotation(s):
    case, out = s["case"], {}
    backward = case["direction"] == "backward"
    for name in ("q", "k"):
        x = s[name].double()
        length = torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS)
        w = s[name + "_weight"].double() if case["norm"] else None
        if not backward:
            out[name] = _exact_turn(x / length * w if case["norm"] else x, s, 1.0)
            continue
        g = _exact_turn(s["grad_" + name].double(), s, -1.0)
        if case["norm"]:
            out[name + "_weight"] = torch.einsum("thd,thd->d", g, x / length)
            g = g * w
            g = g / length - x * torch.einsum("thd,thd->th", g, x)[..., None] / (case["dim"] * length ** 3)
        out[name] = g
    if not backward and case["cache"]:
        for name, rows in (("k", out["k"]), ("v", s["v"].double())):
            whole = torch.zeros(case["cache"], case["kv_heads"], case["dim"], dtype=torch.float64, device="cuda")
            whole.index_copy_(0, s["rows"].long(), rows)
            out[name] = whole
    return out


def _exact_attention(s, backward):
    """Sequence by sequence and a few heads at a time, with the whole mask."""
    case = s["case"]
    hq, d = case["q_heads"], case["dim"]
    group = hq // case["kv_heads"]
    step = case["op"] == "step"
    starts = list(range(case["sequences"] + 1)) if step else s["starts"]
    key_starts, key_lengths = (s["starts"], s["lengths"]) if step else (s["key_starts"], s["key_lengths"])
    zeros = lambda t: torch.zeros(*t.shape, dtype=torch.float64, device="cuda")
    out, lse = zeros(s["q"]), torch.zeros(hq, s["q"].shape[0], dtype=torch.float64, device="cuda")
    grad_q, grad_k, grad_v = (zeros(s["q"]), zeros(s["k"]), zeros(s["k"])) if backward else (None, None, None)
    for i, keys in enumerate(key_lengths):
        a, b, c = starts[i], starts[i + 1], key_starts[i]
        i_at = (torch.arange(b - a, device="cuda") + keys - (b - a))[:, None]
        j_at = torch.arange(keys, device="cuda")[None]
        near = i_at - j_at < case["window"] if case["window"] else torch.ones_like(i_at - j_at, dtype=torch.bool)
        hidden = (j_at > i_at) | ~(near | (j_at < case["sinks"]))
        many = max(1, int(2e8) // ((b - a) * keys))
        for h in range(0, hq, many):
            heads = list(range(h, min(h + many, hq)))
            kv = [x // group for x in heads]
            q, k, v = s["q"][a:b, heads].double(), s["k"][c:c + keys, kv].double(), s["v"][c:c + keys, kv].double()
            q, k, v = (t.permute(1, 0, 2).contiguous() for t in (q, k, v))
            score = torch.baddbmm(torch.zeros(1, 1, 1, dtype=torch.float64, device="cuda"), q, k.mT, alpha=d ** -0.5)
            score[:, hidden] = -math.inf
            log = torch.logsumexp(score, -1)
            p = torch.exp(score - log[..., None])
            lse[heads, a:b] = log
            out[a:b, heads] = torch.bmm(p, v).permute(1, 0, 2)
            if backward:
                g = s["grad_out"][a:b, heads].double().permute(1, 0, 2).contiguous()
                gp = torch.bmm(g, v.mT)
                gs = p * (gp - torch.sum(g * torch.bmm(p, v), -1, keepdim=True)) * d ** -0.5
                grad_q[a:b, heads] = torch.bmm(gs, k).permute(1, 0, 2)
                gk, gv = torch.bmm(gs.mT, q), torch.bmm(p.mT, g)
                for n, x in enumerate(kv):                                # heads that share keys add up
                    grad_k[c:c + keys, x] += gk[n]
                    grad_v[c:c + keys, x] += gv[n]
    if backward:
        return {"grad_q": grad_q, "grad_k": grad_k, "grad_v": grad_v}
    return {"out": out} if step else {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotation":
        return _exact_rotation(s)
    return _exact_attention(s, case.get("direction") == "backward")

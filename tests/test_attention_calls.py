"""The binding's two ways of making the calls of daf_attention.h, the native step and the general one: the same calls, and the native step leaves what is
not usual to the general checks without having done anything."""
import pytest
import torch

import paper_2507_07149_amd as daf
from paper_2507_07149_amd import attention, binding
from tests.test_block_calls import _Recorder, needs_the_module

BF16 = torch.bfloat16


def _calls(device):
    """{name: (function, arguments, keywords, outputs)}: every call with all that it can have."""
    g = torch.Generator().manual_seed(1)
    t = lambda *shape, dtype=BF16: torch.randn(*shape, generator=g).to(dtype).to(device)
    out = lambda *shape, dtype=BF16: torch.zeros(*shape, dtype=dtype, device=device)
    int32 = lambda *values: torch.tensor(values, dtype=torch.int32, device=device)
    n, heads, kv, dim = 12, 4, 2, 32
    qkv, grads, into = t(n, heads + 2 * kv, dim), t(n, heads + kv, dim), out(n, heads + 2 * kv, dim)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    gq, gk, gv = into[:, :heads], into[:, heads:heads + kv], into[:, heads + kv:]
    cos, sin, position, rows = t(20, 8, dtype=torch.float32), t(20, 8, dtype=torch.float32), int32(*range(n)), int32(*range(20, 20 - n, -1))
    w = dict(q_weight=t(dim), k_weight=t(dim), norm=True, eps=1e-5, pairing="pairs")
    oq, ok, ov = out(n, heads, dim), out(30, kv, dim), out(30, kv, dim)
    wq, wk = out(dim, dtype=torch.float32), out(dim, dtype=torch.float32)
    o, lse, token = out(n, heads, dim), out(heads, n, dtype=torch.float32), out(3, heads, dim)
    starts, k_starts, k_lengths = int32(0, 5, n), int32(0, 4), int32(5, 8)
    ws = out(1 << 20, dtype=torch.uint8)
    return {
        "head_rotation": (daf.daf_head_rotation, [q, k, position, cos, sin, oq, ok], dict(w, v=v, out_v=ov, rows=rows), [oq, ok, ov]),
        "head_rotation_backward": (daf.daf_head_rotation_backward, [q, k, position, cos, sin, grads[:, :heads], grads[:, heads:], gq, gk, ws],
                                   dict(w, out_grad_q_weight=wq, out_grad_k_weight=wk), [gq, gk, wq, wk]),
        "window_attention": (daf.daf_window_attention, [q, k, v, o, lse], dict(window=3, sinks=1, scale=0.25, q_starts=starts, k_starts=k_starts, k_lengths=k_lengths), [o, lse]),
        "window_attention_backward": (daf.daf_window_attention_backward, [q, k, v, grads[:, :heads], t(heads, n, dtype=torch.float32), t(n, heads, dim), gq, gk, gv, ws],
                                      dict(window=3, sinks=1, scale=0.25, q_starts=starts), [gq, gk, gv]),
        "window_attention_step": (daf.daf_window_attention_step, [t(3, heads, dim), k, v, int32(0, 2, 4), int32(5, 10, 8), token, ws], dict(window=4, sinks=2), [token]),
    }


NAMES = ("head_rotation", "head_rotation_backward", "window_attention", "window_attention_backward", "window_attention_step")


@needs_the_module
@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_both_ways(name, monkeypatch):
    attention._library()
    function, args, keywords, outs = _calls("cuda")[name]
    native = _Recorder()
    monkeypatch.setattr(attention, "_fast", native)
    function(*args, **keywords)
    assert native.answers == [0]
    want = [t.clone() for t in outs]
    assert all(t.any() for t in want)
    for t in outs:
        t.zero_()
    monkeypatch.setattr(attention, "_fast", binding._NoFastCalls())
    function(*args, **keywords)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@needs_the_module
@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_unusual_arguments_are_left_alone(name, monkeypatch):
    """One tensor at a time of another type, smaller, strided or on the host: the native step does nothing and the general checks say why."""
    attention._library()
    function, args, keywords, outs = _calls("cuda")[name]
    at = [("positional", i) for i, a in enumerate(args) if isinstance(a, torch.Tensor)] + [("keyword", k) for k, a in keywords.items() if isinstance(a, torch.Tensor)]
    for where, key in at:
        good = args[key] if where == "positional" else keywords[key]
        others = {"type": good.to(torch.float64), "size": good.reshape(-1)[:1].clone(), "host": good.cpu(), "strided": torch.stack([good, good], -1)[..., 0]}
        if good.dtype is torch.uint8:                                     # a workspace may be of any type; not all of them need bytes
            del others["type"]
            if name == "window_attention_step" and daf.daf_window_attention_step_workspace_bytes(3, 4, 2, 32, 12, 4, 2) == 0:
                del others["size"]
        for what, bad in others.items():
            a, k = list(args), dict(keywords)
            if where == "positional":
                a[key] = bad
            else:
                k[key] = bad
            native = _Recorder()
            monkeypatch.setattr(attention, "_fast", native)
            with pytest.raises(ValueError):
                function(*a, **k)
            assert native.answers == [None], (key, what)
    torch.cuda.synchronize()
    assert all(not t.any() for t in outs)


@needs_the_module
@pytest.mark.gpu
def test_without_norm_and_with_defaults(monkeypatch):
    attention._library()
    calls = _calls("cuda")
    native = _Recorder()
    monkeypatch.setattr(attention, "_fast", native)
    _, a, _, _ = calls["head_rotation"]
    daf.daf_head_rotation(*a[:6], torch.zeros(12, 2, 32, dtype=BF16, device="cuda"))
    _, a, _, _ = calls["head_rotation_backward"]
    daf.daf_head_rotation_backward(None, None, *a[2:9], norm=False)
    _, a, _, _ = calls["window_attention"]
    daf.daf_window_attention(*a[:4])
    _, a, _, _ = calls["window_attention_backward"]
    daf.daf_window_attention_backward(*a)
    _, a, _, _ = calls["window_attention_step"]
    daf.daf_window_attention_step(*a)
    assert native.answers == [0] * 5
    torch.cuda.synchronize()


@needs_the_module
@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_and_wrong_counts(name):
    attention._library()
    call = getattr(binding._fast_calls, name)
    assert call() is None and call(None) is None
    function, args, keywords, _ = _calls("cpu")[name]
    with pytest.raises(ValueError, match="device"):
        function(*args, **keywords)

"""The binding's two ways of making the calls of daf_block.h, the native step and the general one: the same calls, and the native step leaves what is not
usual to the general checks without having done anything."""
import pytest
import torch

import paper_2507_07149_amd as daf
from paper_2507_07149_amd import binding, block

BF16 = torch.bfloat16
needs_the_module = pytest.mark.skipif(binding._fast_calls is None, reason="the module does not compile here")


def _calls(device):
    """{name: (function, arguments, keywords, outputs)}: every call with all that it can have."""
    g = torch.Generator().manual_seed(1)
    t = lambda *shape, dtype=BF16: torch.randn(*shape, generator=g).to(dtype).to(device)
    out = lambda *shape, dtype=BF16: torch.zeros(*shape, dtype=dtype, device=device)
    rows, cols = 12, 40
    x, z, dy, ds = (t(rows, cols) for _ in range(4))
    vectors = {name: t(cols) for name in ("pre_weight", "pre_bias", "post_weight", "post_bias")}
    gate, stats = t(3, cols), t(rows, 4, dtype=torch.float32)
    grads = {"out_grad_" + name: out(cols, dtype=torch.float32) for name in vectors} | {"out_grad_gate": out(3, cols, dtype=torch.float32)}
    ws = out(1 << 20, dtype=torch.uint8)
    s, y, st, dr, dz = out(rows, cols), out(rows, cols), out(rows, 4, dtype=torch.float32), out(rows, cols), out(rows, cols)
    backward_vectors = {name: v for name, v in vectors.items() if name != "pre_bias"}
    wg, wu, gh, kept = t(24, cols), t(24, cols), t(rows, 24), (t(rows, 24), t(rows, 24))
    h, a, u, dx, dwg, dwu = out(rows, 24), out(rows, 24), out(rows, 24), out(rows, cols), out(24, cols), out(24, cols)
    norm, grad, clipped = out(1, dtype=torch.float32), t(1000), out(1000)
    return {
        "residual_norm": (daf.daf_residual_norm, [x, y, st], dict(kind="layer", eps=1e-5, z=z, out_residual=s, post=True, gate=gate, scale=0.5, **vectors), [s, y, st]),
        "residual_norm_backward": (daf.daf_residual_norm_backward, [x, dy, stats, dr, ws], dict(kind="layer", z=z, grad_residual=ds, out_grad_z=dz, post=True,
                                                                                              gate=gate, scale=0.5, **backward_vectors, **grads), [dr, dz, *grads.values()]),
        "gated_linear": (daf.daf_gated_linear, [x, wg, wu, "gelu", h, ws], dict(out_gate=a, out_up=u), [h, a, u]),
        "gated_linear_backward": (daf.daf_gated_linear_backward, [x, wg, wu, gh, "silu", dx, dwg, dwu, ws], dict(gate=kept[0], up=kept[1]), [dx, dwg, dwu]),
        "clip_grad_norm": (daf.daf_clip_grad_norm, [[(grad, clipped)] if device == "cpu" else daf.grad_items([(grad, clipped)]), 1.0, norm, ws], {}, [clipped, norm]),
    }


NAMES = ("residual_norm", "residual_norm_backward", "gated_linear", "gated_linear_backward", "clip_grad_norm")


class _Recorder:
    """The native step, and what it answered."""

    def __init__(self):
        self.answers = []

    def __getattr__(self, name):
        def call(*args):
            rc = getattr(binding._fast_calls, name)(*args)
            self.answers.append(rc)
            return rc
        return call


@needs_the_module
@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_both_ways(name, monkeypatch):
    block._library()
    function, args, keywords, outs = _calls("cuda")[name]
    native = _Recorder()
    monkeypatch.setattr(block, "_fast", native)
    function(*args, **keywords)
    assert native.answers == [0]
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    monkeypatch.setattr(block, "_fast", binding._NoFastCalls())
    function(*args, **keywords)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@needs_the_module
@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_unusual_arguments_are_left_alone(name, monkeypatch):
    """One tensor at a time of another type, smaller, strided or on the host: the native step does nothing and the general checks say why."""
    block._library()
    function, args, keywords, outs = _calls("cuda")[name]
    at = [("positional", i) for i, a in enumerate(args) if isinstance(a, torch.Tensor)] + [("keyword", k) for k, a in keywords.items() if isinstance(a, torch.Tensor)]
    for where, key in at:
        good = args[key] if where == "positional" else keywords[key]
        others = {"type": good.to(torch.float64), "size": good.reshape(-1)[:1].clone(), "host": good.cpu(), "strided": torch.stack([good, good], -1)[..., 0]}
        if good.dtype is torch.uint8:                                     # a workspace may be of any type
            del others["type"]
            if name == "gated_linear":                                    # (no bytes are needed for these sizes)
                del others["size"]
        if good.numel() == 1:
            del others["size"], others["strided"]
        for what, bad in others.items():
            a, k = list(args), dict(keywords)
            if where == "positional":
                a[key] = bad
            else:
                k[key] = bad
            native = _Recorder()
            monkeypatch.setattr(block, "_fast", native)
            with pytest.raises(ValueError):
                function(*a, **k)
            assert native.answers == [None], (key, what)
    torch.cuda.synchronize()
    assert all(not t.any() for t in outs)


@needs_the_module
@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_and_wrong_counts(name):
    block._library()
    call = getattr(binding._fast_calls, name)
    assert call() is None and call(None) is None
    function, args, keywords, _ = _calls("cpu")[name]
    with pytest.raises(ValueError, match="device"):
        function(*args, **keywords)

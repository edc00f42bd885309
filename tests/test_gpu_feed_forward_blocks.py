"""The example of a training step: norms, gated products, packed inputs and clipping together."""
import importlib.util
import os

import pytest
import torch

from paper_2507_07149_amd import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(build.CSRC)), "examples", "feed_forward_blocks.py")
    spec = importlib.util.spec_from_file_location("feed_forward_blocks", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _expected(net, x, grad_out):
    """Result and gradients in binary64, by automatic differentiation."""
    leaves = [{name: t.double().cpu().requires_grad_() for name, t in b.items()} for b in net.blocks]
    s, z = x.double().cpu().requires_grad_(), None
    first = s
    for b in leaves:
        s = s if z is None else s + net.scale * b["gate"] * z
        y = s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-5) * b["norm"]
        a = y @ b["w_gate"].t()
        z = (a * torch.sigmoid(a) * (y @ b["w_up"].t())) @ b["w_down"].t()
    out = s + net.scale * z
    out.backward(grad_out.double().cpu())
    return out.detach(), first.grad, leaves


@pytest.mark.parametrize("rows,width,inner", [(200, 96, 130), (33, 130, 75), (1, 64, 96)])
def test_gradients(example, rows, width, inner):
    """Nothing packed: every tensor of the two blocks is rounded to binary16 a few times on its way, at most 30 times in a row; all of one sign
    and none of it averaged out that is 30 units of 2^-11 of the norm."""
    net = example.Blocks(rows, width, inner, 2, bits=0, dtype=torch.float16)
    g = torch.Generator().manual_seed(7)
    x, grad_out = (torch.randn(rows, width, generator=g).half().cuda() for _ in range(2))
    out = net.forward(x)
    grad_x = net.backward(grad_out, 1e9)
    want, want_x, leaves = _expected(net, x, grad_out)
    pairs = [("out", out, want), ("x", grad_x, want_x)]
    pairs += [(f"{name} of {i}", net.grads[i][name], leaves[i][name].grad) for i in range(2) for name in leaves[i] if leaves[i][name].grad is not None]
    assert len(pairs) == 2 + 9
    for name, got, exact in pairs:
        off = (got.double().cpu() - exact).norm() / exact.norm()
        assert off <= 30 * 2.0 ** -11, (name, off.item())
    assert not net.grads[0]["gate"].any()
    total = torch.cat([t.double().cpu().flatten() for gr in net.grads for t in gr.values()]).norm()
    assert abs(net.norm.item() - total) <= 1e-6 * total


def test_clipped(example):
    net = example.Blocks(64, 64, 128, 2, bits=0)
    g = torch.Generator().manual_seed(8)
    x, grad_out = (torch.randn(64, 64, generator=g).bfloat16().cuda() for _ in range(2))
    net.forward(x)
    net.backward(grad_out, 0.125)
    assert net.norm.item() > 1.0
    total = torch.cat([t.double().cpu().flatten() for gr in net.grads for t in gr.values()]).norm()
    assert abs(total - 0.125) <= 2.0 ** -8 * 0.125                   # each gradient rounded once more


@pytest.mark.parametrize("bits", [8, 4])
def test_training_with_packed_inputs(example, bits):
    """The loss falls with packed inputs, close to how it falls without; the same seeds give the same bits."""
    def train(bits):
        net = example.Blocks(256, 128, 192, 3, bits=bits)
        g = torch.Generator().manual_seed(9)
        x, target = (torch.randn(256, 128, generator=g).bfloat16().cuda() for _ in range(2))
        losses = [net.step(x, target, 100.0, 1e-2, seed=3 * i)[0].item() for i in range(20)]
        return losses, net

    packed, net = train(bits)
    again, other = train(bits)
    plain, _ = train(0)
    assert packed == again and all(torch.equal(a[n], b[n]) for a, b in zip(net.blocks, other.blocks) for n in a)
    assert plain[-1] < 0.9 * plain[0] and packed[-1] < packed[0]
    assert abs((packed[0] - packed[-1]) / (plain[0] - plain[-1]) - 1) < 0.25


def test_a_token_alone(example):
    """One row through the same weights: the sums run in another order, nothing else."""
    net, one = example.Blocks(40, 128, 200, 2, bits=0), example.Blocks(1, 128, 200, 2, bits=0)
    one.blocks = net.blocks
    x = torch.randn(40, 128, generator=torch.Generator().manual_seed(10)).bfloat16().cuda()
    off = (one.forward(x[:1].clone()).double() - net.forward(x)[:1].double()).norm() / x[:1].double().norm()
    assert off <= 30 * 2.0 ** -9

"""Training steps of a stack of gated feed-forward blocks whose inputs are kept packed.

    block i:   s_i = s_(i-1) + scale * gate_i * z_(i-1),  y_i = rms(s_i) * weight_i          daf_residual_norm
               h = silu(y_i Wg^T) * (y_i Wu^T)                                               daf_gated_linear
               z_i = h Wd^T                                                                  a plain product

Of a block's activations the step keeps s_i and the statistics of its norm, and y_i as packed words (daf_quantize_pack); the two products and h, much the
largest tensors, are not kept at all: the backward pass computes them again from y_i (daf_gated_linear_backward without `gate` and `up`).  At
the end all gradients are clipped to a largest norm (daf_clip_grad_norm).  The same forward pass serves single tokens.

    python examples/feed_forward_blocks.py [--rows 4096] [--width 1024] [--inner 2816] [--blocks 4] [--bits 8] [--steps 10]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_07149_amd as daf  # noqa: E402


class Blocks:
    """Parameters, their gradients and the buffers that every step uses again."""

    VECTORS = ("norm", "gate")
    MATRICES = ("w_gate", "w_up", "w_down")

    def __init__(self, rows, width, inner, blocks, bits=8, dtype=torch.bfloat16, scale=0.5, device="cuda", seed=0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        randn = lambda *shape: torch.randn(*shape, generator=g)
        self.rows, self.width, self.inner, self.scale, self.dtype = rows, width, inner, scale, dtype
        self.blocks = []
        for _ in range(blocks):
            b = {"norm": torch.ones(width), "gate": 0.5 + 0.2 * randn(width), "w_gate": randn(inner, width) / width ** 0.5,
                 "w_up": randn(inner, width) / width ** 0.5, "w_down": randn(width, inner) / inner ** 0.5}
            self.blocks.append({name: t.to(device=device, dtype=dtype) for name, t in b.items()})
        empty = lambda *shape, kind=dtype: torch.empty(*shape, dtype=kind, device=device)
        # vectors' gradients come in binary32
        self.grads = [{name: empty(*t.shape, kind=torch.float32 if name in self.VECTORS else dtype) for name, t in b.items()} for b in self.blocks]
        self.plan = daf.daf_plan((rows, width), 64, bits) if bits else None
        words, groups = (self.plan.packed_words, self.plan.num_groups) if bits else (0, 0)
        self.kept = [{"sum": empty(rows, width), "stats": empty(rows, 4, kind=torch.float32), "z": empty(rows, width),
                      "y": empty(words, kind=torch.int32) if bits else empty(rows, width), "min": empty(groups, kind=torch.float32),
                      "scale": empty(groups, kind=torch.float32)} for _ in self.blocks]
        self.y, self.h, self.grad_h, self.grad_y = empty(rows, width), empty(rows, inner), empty(rows, inner), empty(rows, width)
        self.grad_sum, self.grad_z = [empty(rows, width) for _ in range(2)], [empty(rows, width) for _ in range(2)]
        need = max(daf.daf_gated_linear_backward_workspace_bytes(rows, inner, width, dtype), daf.daf_gated_linear_workspace_bytes(rows, inner, width, dtype),
                   daf.daf_residual_norm_backward_workspace_bytes(rows, width), daf.daf_grad_norm_workspace_bytes())
        self.workspace = empty(max(need, 16), kind=torch.uint8)
        self.norm = empty(1, kind=torch.float32)
        self.items = daf.grad_items([t for g in self.grads for t in g.values()])

    def forward(self, x, seed=0):
        """The last block's residual sum."""
        s, z = x, None
        for i, (b, k) in enumerate(zip(self.blocks, self.kept)):
            daf.daf_residual_norm(s, self.y, k["stats"], z=z, out_residual=k["sum"], pre_weight=b["norm"], gate=None if z is None else b["gate"],
                                  scale=self.scale)
            if self.plan is not None:
                daf.daf_quantize_pack(self.plan, self.y, seed + i, k["y"], k["min"], k["scale"])
            else:
                k["y"].copy_(self.y)
            daf.daf_gated_linear(self.y, b["w_gate"], b["w_up"], "silu", self.h, self.workspace)
            torch.mm(self.h, b["w_down"].t(), out=k["z"])
            s, z = k["sum"], k["z"]
        return s + self.scale * z

    def backward(self, grad_out, max_norm):
        """Gradients of all parameters, clipped, from that of forward's result.  Returns the gradient of x."""
        grad_sum = grad_out
        grad_z = self.scale * grad_out
        for i in reversed(range(len(self.blocks))):
            b, k, g = self.blocks[i], self.kept[i], self.grads[i]
            torch.mm(grad_z, b["w_down"], out=self.grad_h)
            if self.plan is not None:
                daf.daf_unpack_dequantize(self.plan, k["y"], k["min"], k["scale"], self.y)
            else:
                self.y.copy_(k["y"])
            daf.daf_gated_linear_backward(self.y, b["w_gate"], b["w_up"], self.grad_h, "silu", self.grad_y, g["w_gate"], g["w_up"], self.workspace, out_h=self.h)
            torch.mm(grad_z.t(), self.h, out=g["w_down"])
            next_sum, next_z = self.grad_sum[i % 2], self.grad_z[i % 2]
            before = self.kept[i - 1]["z"] if i else None
            daf.daf_residual_norm_backward(k["sum"], self.grad_y, k["stats"], next_sum, self.workspace, z=before, grad_residual=grad_sum,
                                           out_grad_z=next_z if i else None, pre_weight=b["norm"], gate=b["gate"] if i else None, scale=self.scale,
                                           out_grad_pre_weight=g["norm"], out_grad_gate=g["gate"] if i else None)
            if i == 0:
                g["gate"].zero_()                                # the first block has nothing in front of it to gate
            grad_sum, grad_z = next_sum, next_z
        daf.daf_clip_grad_norm(self.items, max_norm, self.norm, self.workspace)
        return grad_sum

    def update(self, rate):
        for b, g in zip(self.blocks, self.grads):
            for name, t in b.items():
                t.add_(g[name].to(t.dtype), alpha=-rate)

    def step(self, x, target, rate, max_norm, seed=0):
        """One step towards sum of squares of (result - target) / 2, over the elements.  Returns that and the gradients' norm, on the device."""
        off = self.forward(x, seed) - target
        self.backward(off / off.numel(), max_norm)
        self.update(rate)
        return off.float().square().mean() / 2, self.norm


def main():
    p = argparse.ArgumentParser()
    for name, value in (("rows", 4096), ("width", 1024), ("inner", 2816), ("blocks", 4), ("bits", 8), ("steps", 10)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    net = Blocks(a.rows, a.width, a.inner, a.blocks, a.bits)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, target = (torch.randn(a.rows, a.width, generator=g, device="cuda").to(net.dtype) for _ in range(2))
    kept = sum(t.numel() * t.element_size() for k in net.kept for t in k.values())
    print(f"{a.blocks} blocks keep {kept / 2 ** 20:.1f} MiB; the two products and h would be {a.blocks * 3 * a.rows * a.inner * 2 / 2 ** 20:.1f} MiB more")
    for i in range(a.steps):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        loss, norm = net.step(x, target, 200.0, 1e-2, seed=i * a.blocks)
        end.record()
        end.synchronize()
        print(f"step {i}: loss {loss.item():.5f}, norm of the gradients {norm.item():.3e}, {begin.elapsed_time(end):.2f} ms")
    token = Blocks(1, a.width, a.inner, a.blocks, bits=0)
    token.blocks = net.blocks
    token.forward(x[:1])
    print("one token alone:", (token.forward(x[:1]).float() - net.forward(x)[:1].float()).abs().max().item(), "off the batch's")


if __name__ == "__main__":
    main()

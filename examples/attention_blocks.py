"""Training steps of a stack of attention blocks over sequences of any lengths, and the same blocks answering token by token from a cache.

    block i:   s_i = s_(i-1) + scale * gate_i * z_(i-1),  y_i = rms(s_i) * weight_i          daf_residual_norm
               q, k, v = y_i Wqkv^T                                                          a plain product, [tokens, all heads, head_dim]
               every head of q and k normalized and rotated by its position                  daf_head_rotation
               a = attention of q over the window's keys and the sinks                       daf_window_attention, daf_window_attention_step
               z_i = a Wo^T                                                                  a plain product

Of a block's activations the step keeps s_i, the statistics of its norm, q, k, v as the product left them, a and its sums' logarithms, and y_i as
packed words (daf_quantize_pack); the rotated heads are computed again in the backward pass.  A server's keys and values go from the product straight to
their rows of the cache; a prompt may come in pieces, and then one token of each sequence at a time.

    python examples/attention_blocks.py [--length 2048] [--sequences 4] [--width 1024] [--heads 8] [--kv-heads 2] [--blocks 4] [--bits 8] [--steps 10]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2507_07149_amd as daf  # noqa: E402


def int32(values, device="cuda"):
    return torch.tensor(list(values), dtype=torch.int32, device=device)


def rotation_tables(positions, rotary, base=10000.0, device="cuda"):
    angles = torch.arange(positions, dtype=torch.float64)[:, None] / base ** (torch.arange(rotary // 2, dtype=torch.float64) * 2 / rotary)
    return angles.cos().float().to(device), angles.sin().float().to(device)


class Batch:
    """Where the tokens of a call stand: `lengths` new ones of each sequence behind `before` earlier ones, then rows that pad the batch up to `rows`."""

    def __init__(self, lengths, rows=None, before=None, first_rows=None):
        before = [0] * len(lengths) if before is None else before
        starts = [0]
        for n in lengths:
            starts.append(starts[-1] + n)
        self.rows = starts[-1] if rows is None else rows
        pad = self.rows - starts[-1]
        self.single = all(n == 1 for n in lengths) and not pad
        self.q_starts = int32(starts)
        self.position = int32([b + i for b, n in zip(before, lengths) for i in range(n)] + [-1] * pad)
        if first_rows is not None:                               # a cache holds the keys, each sequence's from a row of its own on
            self.cache_rows = int32([f + b + i for f, b, n in zip(first_rows, before, lengths) for i in range(n)] + [-1] * pad)
            self.k_starts, self.k_lengths = int32(first_rows), int32(b + n for b, n in zip(before, lengths))


class Blocks:
    """Parameters, their gradients and the buffers that every step of a batch of `rows` tokens uses again."""

    VECTORS = ("norm", "gate", "q_norm", "k_norm")

    def __init__(self, rows, width, heads, kv_heads, dim, blocks, window, sinks, positions, bits=8, dtype=torch.bfloat16, scale=0.5, seed=0, sequences=64):
        g = torch.Generator().manual_seed(seed)
        randn = lambda *shape: torch.randn(*shape, generator=g)
        self.rows, self.width, self.heads, self.kv_heads, self.dim = rows, width, heads, kv_heads, dim
        self.seen, self.scale, self.dtype = {"window": window, "sinks": sinks}, scale, dtype
        self.tables = rotation_tables(positions, dim // 16 * 16)
        all_heads = heads + 2 * kv_heads
        self.blocks = []
        for _ in range(blocks):
            b = {"norm": torch.ones(width), "gate": 0.5 + 0.2 * randn(width), "q_norm": 1 + 0.2 * randn(dim), "k_norm": 1 + 0.2 * randn(dim),
                 "w_qkv": randn(all_heads * dim, width) / width ** 0.5, "w_out": randn(width, heads * dim) / (heads * dim) ** 0.5}
            self.blocks.append({name: t.to("cuda", dtype) for name, t in b.items()})
        empty = lambda *shape, kind=dtype: torch.empty(*shape, dtype=kind, device="cuda")
        # vectors' gradients come in binary32
        self.grads = [{name: empty(*t.shape, kind=torch.float32 if name in self.VECTORS else dtype) for name, t in b.items()} for b in self.blocks]
        self.plan = daf.daf_plan((rows, width), 64, bits) if bits else None
        words, groups = (self.plan.packed_words, self.plan.num_groups) if bits else (0, 0)
        # rows that pad a batch are of no sequence: attention leaves them as they are, and they are zero from the beginning
        self.kept = [{"sum": empty(rows, width), "stats": empty(rows, 4, kind=torch.float32), "z": empty(rows, width), "qkv": empty(rows, all_heads, dim),
                      "out": empty(rows, heads, dim).zero_(), "lse": empty(heads, rows, kind=torch.float32),
                      "y": empty(words, kind=torch.int32) if bits else empty(rows, width), "min": empty(groups, kind=torch.float32),
                      "scale": empty(groups, kind=torch.float32)} for _ in self.blocks]
        self.y, self.grad_y, self.grad_out = empty(rows, width), empty(rows, width), empty(rows, heads, dim)
        self.rotated, self.grad_qkv = empty(rows, heads + kv_heads, dim), empty(rows, all_heads, dim).zero_()
        self.grad_sum, self.grad_z = [empty(rows, width) for _ in range(2)], [empty(rows, width) for _ in range(2)]
        self.sequences = sequences
        need = max(daf.daf_window_attention_backward_workspace_bytes(rows, heads, kv_heads, dim, sequences, window, sinks),
                   daf.daf_window_attention_step_workspace_bytes(min(rows, sequences), heads, kv_heads, dim, positions * sequences, window, sinks),
                   daf.daf_head_rotation_backward_workspace_bytes(rows, heads, kv_heads, dim),
                   daf.daf_residual_norm_backward_workspace_bytes(rows, width), daf.daf_grad_norm_workspace_bytes())
        self.workspace = empty(max(need, 16), kind=torch.uint8)
        self.norm = empty(1, kind=torch.float32)
        self.items = daf.grad_items([t for g in self.grads for t in g.values()])

    def _split(self, t):
        """Queries, keys and values: views of a product's result, or of a gradient's."""
        return t.split([self.heads, self.kv_heads, self.kv_heads], 1)

    def _rotate(self, b, k, batch, out_q, out_k, **cache):
        q, key, value = self._split(k["qkv"])
        if cache:
            cache["v"] = value
        daf.daf_head_rotation(q, key, batch.position, *self.tables, out_q, out_k, q_weight=b["q_norm"], k_weight=b["k_norm"], **cache)

    def new_cache(self, rows):
        """Keys and values of `rows` tokens, for every block."""
        return [torch.zeros(2, rows, self.kv_heads, self.dim, dtype=self.dtype, device="cuda") for _ in self.blocks]

    def forward(self, x, batch, cache=None, seed=0):
        """The last block's residual sum.  With a cache the batch's keys go to its rows, and its queries see what is there."""
        s, z = x, None
        for i, (b, k) in enumerate(zip(self.blocks, self.kept)):
            daf.daf_residual_norm(s, self.y, k["stats"], z=z, out_residual=k["sum"], pre_weight=b["norm"], gate=None if z is None else b["gate"],
                                  scale=self.scale)
            if cache is None and self.plan is not None:
                daf.daf_quantize_pack(self.plan, self.y, seed + i, k["y"], k["min"], k["scale"])
            elif cache is None:
                k["y"].copy_(self.y)
            torch.mm(self.y, b["w_qkv"].t(), out=k["qkv"].view(self.rows, -1))
            q = self.rotated[:, :self.heads]
            if cache is None:
                self._rotate(b, k, batch, q, self.rotated[:, self.heads:])
                daf.daf_window_attention(q, self.rotated[:, self.heads:], self._split(k["qkv"])[2], k["out"], k["lse"], q_starts=batch.q_starts, **self.seen)
            else:
                keys, values = cache[i]
                self._rotate(b, k, batch, q, keys, out_v=values, rows=batch.cache_rows)
                if batch.single:
                    daf.daf_window_attention_step(q, keys, values, batch.k_starts, batch.k_lengths, k["out"], self.workspace, **self.seen)
                else:
                    daf.daf_window_attention(q, keys, values, k["out"], q_starts=batch.q_starts, k_starts=batch.k_starts, k_lengths=batch.k_lengths, **self.seen)
            torch.mm(k["out"].view(self.rows, -1), b["w_out"].t(), out=k["z"])
            s, z = k["sum"], k["z"]
        return s + self.scale * z

    def backward(self, grad_out, batch, max_norm):
        """Gradients of all parameters, clipped, from that of forward's result.  Returns the gradient of x."""
        grad_sum = grad_out
        grad_z = self.scale * grad_out
        for i in reversed(range(len(self.blocks))):
            b, k, g = self.blocks[i], self.kept[i], self.grads[i]
            torch.mm(grad_z, b["w_out"], out=self.grad_out.view(self.rows, -1))
            torch.mm(grad_z.t(), k["out"].view(self.rows, -1), out=g["w_out"])
            rotated_q, rotated_k = self.rotated[:, :self.heads], self.rotated[:, self.heads:]
            self._rotate(b, k, batch, rotated_q, rotated_k)
            (q, key, value), (grad_q, grad_k, grad_v) = self._split(k["qkv"]), self._split(self.grad_qkv)
            daf.daf_window_attention_backward(rotated_q, rotated_k, value, k["out"], k["lse"], self.grad_out, grad_q, grad_k, grad_v, self.workspace,
                                              q_starts=batch.q_starts, **self.seen)
            daf.daf_head_rotation_backward(q, key, batch.position, *self.tables, grad_q, grad_k, grad_q, grad_k, self.workspace, q_weight=b["q_norm"],
                                           k_weight=b["k_norm"], out_grad_q_weight=g["q_norm"], out_grad_k_weight=g["k_norm"])
            if self.plan is not None:
                daf.daf_unpack_dequantize(self.plan, k["y"], k["min"], k["scale"], self.y)
            else:
                self.y.copy_(k["y"])
            torch.mm(self.grad_qkv.view(self.rows, -1), b["w_qkv"], out=self.grad_y)
            torch.mm(self.grad_qkv.view(self.rows, -1).t(), self.y, out=g["w_qkv"])
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

    def step(self, x, target, batch, rate, max_norm, seed=0):
        """One step towards sum of squares of (result - target) / 2, over the elements.  Returns that and the gradients' norm, on the device."""
        off = self.forward(x, batch, seed=seed) - target
        self.backward(off / off.numel(), batch, max_norm)
        for b, g in zip(self.blocks, self.grads):
            for name, t in b.items():
                t.add_(g[name].to(t.dtype), alpha=-rate)
        return off.float().square().mean() / 2, self.norm


def main():
    p = argparse.ArgumentParser()
    for name, value in (("length", 2048), ("sequences", 4), ("width", 1024), ("heads", 8), ("kv-heads", 2), ("dim", 128), ("blocks", 4), ("window", 1024),
                        ("sinks", 4), ("bits", 8), ("steps", 10)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    shape = (a.width, a.heads, a.kv_heads, a.dim, a.blocks, a.window, a.sinks, a.length)
    batch = Batch([a.length] * a.sequences)
    net = Blocks(batch.rows, *shape, bits=a.bits, sequences=a.sequences)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, target = (torch.randn(batch.rows, a.width, generator=g, device="cuda").to(net.dtype) for _ in range(2))
    for i in range(a.steps):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        loss, norm = net.step(x, target, batch, 200.0, 1e-2, seed=i * a.blocks)
        end.record()
        end.synchronize()
        print(f"step {i}: loss {loss.item():.5f}, norm of the gradients {norm.item():.3e}, {begin.elapsed_time(end):.2f} ms")
    # the last token of every sequence alone, over a cache that holds what is in front of it
    whole = net.forward(x, batch).view(a.sequences, a.length, -1)[:, -1]
    first = [i * a.length for i in range(a.sequences)]
    x = x.view(a.sequences, a.length, -1)
    prompt, token = (Blocks(n * a.sequences, *shape, bits=0, sequences=a.sequences) for n in (a.length - 1, 1))
    prompt.blocks = token.blocks = net.blocks
    cache = net.new_cache(batch.rows)
    prompt.forward(x[:, :-1].reshape(-1, a.width), Batch([a.length - 1] * a.sequences, first_rows=first), cache)
    alone = token.forward(x[:, -1].contiguous(), Batch([1] * a.sequences, before=[a.length - 1] * a.sequences, first_rows=first), cache)
    print("one token of each sequence from the cache:", (alone.float() - whole.float()).abs().max().item(), "off the whole sequences'")


if __name__ == "__main__":
    main()

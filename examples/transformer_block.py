"""One training step of a pre-norm transformer block with the operators of kt, from the input to the updated parameters.

    x -> a = x + proj(attention(qkv(norm1(x)))) -> a + down(gelu(up(norm2(a))))

What the forward pass keeps for the backward pass: the linear layers' and the norms' inputs as 8-bit checkpoints (1.03 bytes an
element), q, k, v and the attention's output as they are.  The backward pass writes every gradient where the plan's buckets
keep it, so nothing is packed; the buckets are then reduced over the peers and applied by the update.  The products with a weight
matrix that change no checkpoint are torch's.

    python examples/transformer_block.py [--dtype bf16|f32] [--batch 8] [--tokens 2048] [--width 2048] [--heads 16] [--kv-heads 16] [--steps 5]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_10183_amd as kt  # noqa: E402

EPS = 1e-5


class Checkpoint:
    """A matrix kept in 8 bits."""

    def __init__(self, rows, cols, device):
        q, e = kt.kt_act8_shapes(rows, cols)
        self.parts = torch.empty(q, dtype=torch.int8, device=device), torch.empty(e, dtype=torch.uint8, device=device)

    def save(self, x):
        kt.kt_act8_save(x, *self.parts)

    def restore(self, like):
        y = torch.empty_like(like)
        kt.kt_act8_restore(*self.parts, y)
        return y


class Block:
    def __init__(self, width, heads, kv_heads, mlp, dtype, device="cuda", seed=0):
        self.width, self.heads, self.kv_heads, self.dim = width, heads, kv_heads, width // heads
        self.dtype, self.device = dtype, device
        self.qkv_rows = (heads + 2 * kv_heads) * self.dim
        self.shapes = {"norm1": (width,), "norm1_bias": (width,), "qkv": (self.qkv_rows, width), "proj": (width, heads * self.dim),
                       "norm2": (width,), "norm2_bias": (width,), "up": (mlp, width), "down": (width, mlp)}
        g = torch.Generator(device=device).manual_seed(seed)
        self.master = {}
        for name, shape in self.shapes.items():
            if len(shape) == 2:
                self.master[name] = torch.randn(shape, generator=g, device=device) * shape[1] ** -0.5
            else:
                self.master[name] = torch.full(shape, 0.0 if name.endswith("bias") else 1.0, device=device)
        self.momenta = {n: torch.zeros_like(p) for n, p in self.master.items()}
        # what the passes read: in f32 the parameters themselves, in bf16 a copy that the update writes
        self.w = self.master if dtype == torch.float32 else {n: p.to(dtype) for n, p in self.master.items()}
        self.plan = kt.Plan([p.numel() for p in self.master.values()], "f32" if dtype == torch.float32 else "bf16", 25 << 20, 16)
        self.buckets = [torch.zeros(n, dtype=dtype, device=device) for n in self.plan.bucket_elems()]
        self.grads = {}
        for t, (name, shape) in enumerate(self.shapes.items()):
            b, at = self.plan.tensor_info(t)
            self.grads[name] = self.buckets[b][at:at + self.master[name].numel()].view(shape)
        self.kept = None
        self.stepped = False

    def _norm(self, x, which, y8):
        y = torch.empty_like(x)
        mean, rstd = (torch.empty(x.shape[0], device=self.device) for _ in range(2))
        kt.kt_layernorm_fwd(x, self.w[which], self.w[which + "_bias"], EPS, y, mean, rstd, y8=y8.parts)
        return y, mean, rstd

    def _heads(self, qkv, batch, tokens):
        """q, k and v as views of one product's output."""
        return qkv.view(batch, tokens, -1, self.dim).split([self.heads, self.kv_heads, self.kv_heads], dim=2)

    def forward(self, x, lens=None):
        """x [batch, tokens, width] -> the block's output; causal, with the keys of each sequence in `lens` (int32) or all."""
        batch, tokens, width = x.shape
        rows = batch * tokens
        x = x.reshape(rows, width)
        x8, y1_8, a8, y2_8 = (Checkpoint(rows, width, self.device) for _ in range(4))
        h8, z8 = (Checkpoint(rows, self.shapes["up"][0], self.device) for _ in range(2))
        x8.save(x)
        y1, mean1, rstd1 = self._norm(x, "norm1", y1_8)
        qkv = y1 @ self.w["qkv"].t()
        q, k, v = self._heads(qkv, batch, tokens)
        o = torch.empty(batch, tokens, self.heads, self.dim, dtype=self.dtype, device=self.device)
        lse = torch.empty(batch, self.heads, tokens, device=self.device)
        kt.kt_attention_fwd(q, k, v, o, lse, causal=True, k_lens=lens)
        a = x + o.view(rows, -1) @ self.w["proj"].t()
        a8.save(a)
        y2, mean2, rstd2 = self._norm(a, "norm2", y2_8)
        h = y2 @ self.w["up"].t()
        h8.save(h)
        z = torch.nn.functional.gelu(h)
        z8.save(z)
        self.kept = (x8, y1_8, mean1, rstd1, qkv, o, lse, lens, a8, y2_8, mean2, rstd2, h8, z8)
        return (a + z @ self.w["down"].t()).view(batch, tokens, width)

    def _norm_back(self, dy, x8, which, mean, rstd):
        kt.kt_layernorm_bwd(dy, x8.parts, self.w[which], mean, rstd, dy, self.grads[which], self.grads[which + "_bias"])
        return dy

    def backward(self, dout):
        """The gradient of x; those of the parameters go into the buckets."""
        x8, y1_8, mean1, rstd1, qkv, o, lse, lens, a8, y2_8, mean2, rstd2, h8, z8 = self.kept
        self.kept = None
        batch, tokens, width = dout.shape
        rows = batch * tokens
        dout = dout.reshape(rows, width)
        kt.kt_act8_weight_grad(dout, *z8.parts, self.grads["down"])
        dz = dout @ self.w["down"]
        dh = torch.ops.aten.gelu_backward(dz, h8.restore(dz))
        kt.kt_act8_weight_grad(dh, *y2_8.parts, self.grads["up"])
        da = self._norm_back(dh @ self.w["up"], a8, "norm2", mean2, rstd2).add_(dout)
        torch.mm(da.t(), o.view(rows, -1), out=self.grads["proj"])
        do = (da @ self.w["proj"]).view_as(o)
        dqkv = torch.empty_like(qkv)
        kt.kt_attention_bwd(do, *self._heads(qkv, batch, tokens), o, lse, *self._heads(dqkv, batch, tokens), causal=True, k_lens=lens)
        kt.kt_act8_weight_grad(dqkv, *y1_8.parts, self.grads["qkv"])
        dx = self._norm_back(dqkv @ self.w["qkv"], x8, "norm1", mean1, rstd1).add_(da)
        return dx.view(batch, tokens, width)

    def update(self, lr, momentum=0.9, peers=(), weights=(1.0,)):
        """The weighted sum of this process's buckets and those of its peers (lists of buckets), applied to the parameters."""
        if peers:
            copies = [self.buckets] + list(peers)
            flat = [copy[b] for b in range(len(self.buckets)) for copy in copies]
            self.plan.kt_weighted_reduce(-1, flat, len(copies), weights, self.buckets)
        master, momenta = list(self.master.values()), list(self.momenta.values())
        if self.dtype == torch.float32:
            self.plan.kt_bucket_unpack_sgd(-1, self.buckets, 1.0, master, momenta, lr, momentum, 0.0, not self.stepped)
        else:
            self.plan.kt_bucket_unpack_sgd_master(-1, self.buckets, 1.0, master, momenta, list(self.w.values()), lr, momentum, 0.0,
                                                  not self.stepped)
        self.stepped = True


def train(block, x, target, steps, lr, lens=None):
    """Steps towards `target` by the mean squared error; the losses, each from before its step."""
    losses = []
    for _ in range(steps):
        err = block.forward(x, lens) - target
        losses.append(err.float().square().mean())
        block.backward(err * (2.0 / err.numel()))
        block.update(lr)
    return torch.stack(losses).tolist()


def main():
    p = argparse.ArgumentParser(description="training steps of one transformer block")
    p.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--width", type=int, default=2048)
    p.add_argument("--heads", type=int, default=16)
    p.add_argument("--kv-heads", type=int, default=16)
    p.add_argument("--steps", type=int, default=5)
    p.add_argument("--lr", type=float, default=2.0)          # the loss is a mean over all elements
    a = p.parse_args()
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    block = Block(a.width, a.heads, a.kv_heads, 4 * a.width, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, target = (torch.randn(a.batch, a.tokens, a.width, generator=g, device="cuda").to(dtype) for _ in range(2))
    train(block, x, target, 2, a.lr)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    losses = train(block, x, target, a.steps, a.lr)
    end.record()
    end.synchronize()
    print("loss " + " ".join("%.4f" % v for v in losses))
    print("%.2f ms a step, %d tokens" % (start.elapsed_time(end) / a.steps, a.batch * a.tokens))


if __name__ == "__main__":
    main()

"""A training step of a small language model with the operators of kt, from token ids to the updated parameters: a table that is both the embedding and the
weight of the last layer, transformer blocks between them (transformer_block.py), and the cross entropy of the next token.

    ids -> scale * table[ids] -> blocks -> norm -> cross entropy of (norm table^T)

Neither the logits nor their gradient are ever kept.  The table's gradient is written where the bucket keeps it by the loss, and the embedding adds its own
to it.  Positions whose target is -1 (padding, prompts) take no part in the loss.

    python examples/language_model.py [--dtype bf16|f32] [--batch 8] [--tokens 2048] [--width 2048] [--heads 16] [--blocks 1] [--vocab 50304] [--steps 5]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2505_10183_amd as kt  # noqa: E402
from transformer_block import EPS, Block, Checkpoint  # noqa: E402


class LanguageModel:
    def __init__(self, vocab, width, heads, kv_heads, mlp, blocks, dtype, device="cuda", seed=0):
        self.vocab, self.width, self.dtype, self.device = vocab, width, dtype, device
        self.blocks = [Block(width, heads, kv_heads, mlp, dtype, device, seed=seed + 1 + i) for i in range(blocks)]
        g = torch.Generator(device=device).manual_seed(seed)
        self.shapes = {"table": (vocab, width), "norm": (width,), "norm_bias": (width,)}
        self.master = {"table": torch.randn(vocab, width, generator=g, device=device) * width ** -0.5,
                       "norm": torch.ones(width, device=device), "norm_bias": torch.zeros(width, device=device)}
        self.momenta = {n: torch.zeros_like(p) for n, p in self.master.items()}
        self.w = self.master if dtype == torch.float32 else {n: p.to(dtype) for n, p in self.master.items()}
        self.plan = kt.Plan([p.numel() for p in self.master.values()], "f32" if dtype == torch.float32 else "bf16", 25 << 20, 16)
        self.buckets = [torch.zeros(n, dtype=dtype, device=device) for n in self.plan.bucket_elems()]
        self.grads = {}
        for t, (name, shape) in enumerate(self.shapes.items()):
            b, at = self.plan.tensor_info(t)
            self.grads[name] = self.buckets[b][at:at + self.master[name].numel()].view(shape)
        self.scale = width ** 0.5
        self.kept = None
        self.stepped = False

    def forward(self, ids, targets, lens=None):
        """ids and targets [batch, tokens] -> the loss of each position (0 where the target is not in the vocabulary)."""
        batch, tokens = ids.shape
        x = torch.empty(batch, tokens, self.width, dtype=self.dtype, device=self.device)
        kt.kt_embedding_fwd(ids, self.w["table"], x, scale=self.scale)
        for block in self.blocks:
            x = block.forward(x, lens)
        rows = batch * tokens
        x = x.view(rows, self.width)
        x8 = Checkpoint(rows, self.width, self.device)
        x8.save(x)
        y = torch.empty_like(x)
        mean, rstd, loss, lse = (torch.empty(rows, device=self.device) for _ in range(4))
        kt.kt_layernorm_fwd(x, self.w["norm"], self.w["norm_bias"], EPS, y, mean, rstd)
        kt.kt_linear_xent_fwd(y, self.w["table"], targets.view(-1), loss, lse)
        self.kept = ids, targets, x8, y, mean, rstd, lse
        return loss.view(batch, tokens)

    def backward(self, dloss):
        """From the gradient of the losses to those of all parameters, in the buckets."""
        ids, targets, x8, y, mean, rstd, lse = self.kept
        self.kept = None
        dy = torch.empty_like(y)
        kt.kt_linear_xent_bwd(dloss.reshape(-1), y, self.w["table"], targets.view(-1), lse, dy, self.grads["table"])
        kt.kt_layernorm_bwd(dy, x8.parts, self.w["norm"], mean, rstd, dy, self.grads["norm"], self.grads["norm_bias"])
        dx = dy.view(*ids.shape, self.width)
        for block in reversed(self.blocks):
            dx = block.backward(dx)
        kt.kt_embedding_bwd(ids, dx.contiguous(), self.grads["table"], scale=self.scale, accumulate=True)

    def update(self, lr, momentum=0.9):
        for block in self.blocks:
            block.update(lr, momentum)
        master, momenta = list(self.master.values()), list(self.momenta.values())
        if self.dtype == torch.float32:
            self.plan.kt_bucket_unpack_sgd(-1, self.buckets, 1.0, master, momenta, lr, momentum, 0.0, not self.stepped)
        else:
            self.plan.kt_bucket_unpack_sgd_master(-1, self.buckets, 1.0, master, momenta, list(self.w.values()), lr, momentum, 0.0, not self.stepped)
        self.stepped = True


def train(model, ids, targets, steps, lr, lens=None):
    """Steps on one batch; the mean losses over the positions with a target, each from before its step."""
    live = (targets >= 0) & (targets < model.vocab)
    dloss = live.float() / live.sum().clamp(min=1)
    losses = []
    for _ in range(steps):
        losses.append((model.forward(ids, targets, lens) * dloss).sum())
        model.backward(dloss)
        model.update(lr)
    return torch.stack(losses).tolist()


def main():
    p = argparse.ArgumentParser(description="training steps of a small language model")
    p.add_argument("--dtype", choices=["bf16", "f32"], default="bf16")
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--tokens", type=int, default=2048)
    p.add_argument("--width", type=int, default=2048)
    p.add_argument("--heads", type=int, default=16)
    p.add_argument("--kv-heads", type=int, default=16)
    p.add_argument("--blocks", type=int, default=1)
    p.add_argument("--vocab", type=int, default=50304)
    p.add_argument("--steps", type=int, default=5)
    p.add_argument("--lr", type=float, default=0.1)
    a = p.parse_args()
    dtype = torch.bfloat16 if a.dtype == "bf16" else torch.float32
    model = LanguageModel(a.vocab, a.width, a.heads, a.kv_heads, 4 * a.width, a.blocks, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, a.vocab, (a.batch, a.tokens), generator=g, device="cuda")
    targets = torch.cat([ids[:, 1:], torch.full_like(ids[:, :1], -1)], 1)
    train(model, ids, targets, 2, a.lr)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    losses = train(model, ids, targets, a.steps, a.lr)
    end.record()
    end.synchronize()
    print("loss " + " ".join("%.4f" % v for v in losses))
    print("%.2f ms a step, %d tokens" % (start.elapsed_time(end) / a.steps, a.batch * a.tokens))


if __name__ == "__main__":
    main()

"""examples/language_model.py: the lookup, a block, the cross entropy and both gradients of a tied table in one step, against autograd in 64 bits.

Tolerances in norm, as the block's own test has them: checkpoints, up to five of them on a gradient's way, 1 % each; in bf16 half a step, 2^-8, of each of some
fifteen tensors besides.  The table's gradient is the sum of two that are each that near, rounded to bf16 once more."""
import importlib.util
import os
import sys

import pytest
import torch

from ops_util import DEV, DT, gen

pytestmark = pytest.mark.gpu

DIR = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("kt_example_language_model", os.path.join(DIR, "language_model.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def norm(t, gamma, beta):
    c = t - t.mean(-1, keepdim=True)
    return c / (c.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gamma + beta


def plain(model, ids, targets):
    """The losses in 64 bits by elementary operations, for autograd."""
    p = {n: t.double().detach().requires_grad_() for n, t in model.w.items()}
    inner = []
    x = p["table"][ids] * model.scale
    B, N = ids.shape
    for block in model.blocks:
        q = {n: t.double().detach().requires_grad_() for n, t in block.w.items()}
        inner.append(q)
        H, D = block.heads, block.dim
        qh, kh, vh = (norm(x, q["norm1"], q["norm1_bias"]) @ q["qkv"].t()).view(B, N, 3 * H, D).transpose(1, 2).split(H, dim=1)
        s = torch.matmul(qh, kh.transpose(2, 3)) * D ** -0.5
        s = s.masked_fill(~torch.ones(N, N, dtype=torch.bool, device=DEV).tril(), -1e30)
        x = x + torch.matmul(torch.softmax(s, 3), vh).transpose(1, 2).reshape(B, N, -1) @ q["proj"].t()
        x = x + torch.nn.functional.gelu(norm(x, q["norm2"], q["norm2_bias"]) @ q["up"].t()) @ q["down"].t()
    z = norm(x, p["norm"], p["norm_bias"]) @ p["table"].t()
    live = targets >= 0
    loss = torch.logsumexp(z, 2) - z.gather(2, targets.clamp(min=0)[:, :, None]).squeeze(2)
    return torch.where(live, loss, 0.0), p, inner


@pytest.mark.parametrize("dtype,vocab,tokens", [("f32", 503, 70), ("bf16", 503, 70), ("bf16", 1000, 300)])
def test_gradients(example, dtype, vocab, tokens):
    model = example.LanguageModel(vocab, 128, 2, 2, 512, 1, DT[dtype], seed=3)
    g = gen(4)
    ids = torch.randint(0, vocab, (3, tokens), generator=g, device=DEV)
    targets = torch.cat([ids[:, 1:], torch.full_like(ids[:, :1], -1)], 1)
    targets[1, tokens // 2:] = -1
    dloss = torch.rand(3, tokens, generator=g, device=DEV)
    loss = model.forward(ids, targets)
    model.backward(dloss)
    want, p, inner = plain(model, ids, targets)
    (want * dloss.double()).sum().backward()
    assert off(loss, want.detach()) <= (4e-4 if dtype == "f32" else 0.04)
    assert not loss[targets < 0].any()
    for name, grads, q in [(n, model.grads, p) for n in p] + [(n, model.blocks[0].grads, inner[0]) for n in inner[0]]:
        print(name, off(grads[name], q[name].grad), file=sys.stderr)
        assert off(grads[name], q[name].grad) <= (0.06 if dtype == "f32" else 0.11), name


def test_it_runs_with_its_own_arguments(example, capsys, monkeypatch):
    monkeypatch.setattr(sys, "argv", ["language_model.py", "--steps", "2"])
    example.main()
    line = capsys.readouterr().out.splitlines()[0].split()
    assert line[0] == "loss" and len(line) == 3 and all(torch.isfinite(torch.tensor(float(v))) for v in line[1:])

"""examples/transformer_block.py: the operators together, as a training step makes them, against autograd in 64 bits.

The forward pass uses no checkpoint: off by its sums of at most 1024 terms, 1024 u each of some six in a row, 4e-4 in norm (bf16:
half a step, 2^-8, of each of some ten tensors on the way: 4 %).
A checkpoint is off by at most half a step of its group's largest magnitude a, a / 128; of 32 normal members with a = 2.1 sigma and
an error spread over the step that is 1 % in norm.  A gradient passes up to four of them: 5 % (bf16: 9 %)."""
import importlib.util
import os
import sys

import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, HALF, U, gen, normal

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "transformer_block.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("kt_example_block", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def off(got, want):
    """Distance in norm, relative."""
    return float((got.double() - want).norm() / want.norm())


def plain(block, x, lens):
    """The block in 64 bits by elementary operations, for autograd."""
    p = {n: t.double().detach().requires_grad_() for n, t in block.w.items()}
    B, N, W = x.shape
    H, Hk, D = block.heads, block.kv_heads, block.dim

    def norm(t, which):
        c = t - t.mean(-1, keepdim=True)
        return c / (c.square().mean(-1, keepdim=True) + 1e-5).sqrt() * p[which] + p[which + "_bias"]

    q, k, v = (norm(x, "norm1") @ p["qkv"].t()).view(B, N, -1, D).split([H, Hk, Hk], dim=2)
    k, v = (t.repeat_interleave(H // Hk, 2) for t in (k, v))
    s = torch.einsum("bihd,bjhd->bhij", q, k) * D ** -0.5
    j, i = torch.arange(N, device=DEV), torch.arange(N, device=DEV)[:, None]
    seen = (j <= i).expand(B, N, N)
    if lens is not None:
        seen = seen & (j < lens[:, None, None])
    s = s.masked_fill(~seen[:, None], -1e30)
    w = torch.softmax(s, 3) * seen[:, None]
    a = x + torch.einsum("bhij,bjhd->bihd", w, v).reshape(B, N, -1) @ p["proj"].t()
    return a + torch.nn.functional.gelu(norm(a, "norm2") @ p["up"].t()) @ p["down"].t(), p


@pytest.mark.parametrize("lens", [None, [0, 77, 130]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (4, 2)])
def test_gradients(example, dtype, heads, kv_heads, lens):
    dt = DT[dtype]
    block = example.Block(256, heads, kv_heads, 1024, dt, seed=3)
    g = gen(4)
    x, dout = normal(g, 3, 130, 256, dtype=dt), normal(g, 3, 130, 256, dtype=dt)
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = block.forward(x, lens)
    dx = block.backward(dout)
    x64 = x.double().requires_grad_()
    want, p = plain(block, x64, lens)
    want.backward(dout.double())
    assert off(out, want.detach()) <= (4e-4 if dtype == "f32" else 0.04)
    for name, got, grad in [("x", dx, x64.grad)] + [(n, block.grads[n], p[n].grad) for n in p]:
        print(name, off(got, grad), file=sys.stderr)
        assert off(got, grad) <= (0.05 if dtype == "f32" else 0.09), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_update(example, dtype):
    """The weighted sum over the peers, rounded to the buckets' type, then lr times it: u for each of the steps."""
    dt = DT[dtype]
    block = example.Block(128, 2, 1, 512, dt, seed=5)
    g = gen(6)
    block.forward(normal(g, 2, 33, 128, dtype=dt))
    block.backward(normal(g, 2, 33, 128, dtype=dt))
    peers = [[normal(g, b.numel(), dtype=dt) for b in block.buckets] for _ in range(2)]
    _, weights = kt.kt_plan_shares([1.0, 0.6, 0.4], 64)
    before = {n: (block.master[n].clone(), block.grads[n].clone()) for n in block.master}
    lr = 0.25
    block.update(lr, peers=peers, weights=weights)
    for t, (name, (p, grad)) in enumerate(before.items()):
        b, at = block.plan.tensor_info(t)
        terms = [w * c.double().view_as(p) for w, c in zip(weights, [grad] + [q[b][at:at + p.numel()] for q in peers])]
        total, size = sum(terms), sum(c.abs() for c in terms)
        want = p.double() - lr * total
        tol = lr * (3 * U * size + (HALF[dt] if dtype == "bf16" else 0) * total.abs()) + 2 * U * (want.abs() + lr * size)
        assert bool(((block.master[name].double() - want).abs() <= tol).all()), name
        assert torch.equal(block.w[name], block.master[name].to(dt))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_it_learns(example, dtype):
    dt = DT[dtype]
    block = example.Block(128, 2, 2, 512, dt, seed=7)
    g = gen(8)
    x, target = normal(g, 4, 65, 128, dtype=dt), normal(g, 4, 65, 128, dtype=dt)
    losses = example.train(block, x, target, 12, 2.0)
    assert all(torch.isfinite(torch.tensor(losses))) and losses[-1] < 0.9 * losses[0], losses


def test_it_learns_with_its_own_arguments(example, capsys, monkeypatch):
    """As the command runs it: every loss is finite and below the first."""
    monkeypatch.setattr(sys, "argv", [PATH])
    example.main()
    line = capsys.readouterr().out.splitlines()[0].split()
    losses = [float(v) for v in line[1:]]
    assert line[0] == "loss" and len(losses) == 5
    assert all(v < losses[0] for v in losses[1:]) and losses[0] < 3.0, losses

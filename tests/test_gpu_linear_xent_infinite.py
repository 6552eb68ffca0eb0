"""Logits that are infinite mean the same whatever makes the products: one of -inf counts as exp(-inf) = 0, and the token's loss and gradients are those without that
class; one of +inf leaves a loss that is not finite, of its token alone.  Tolerances: test_gpu_linear_xent.py, from the columns that are not infinite."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, HALF, U, gen, within
from test_gpu_linear_xent import Case

pytestmark = pytest.mark.gpu

# few tokens, tiles, listed tokens, and (f32, from 80 tiles of 256 x 128 on) numbers in three parts, in one piece of the vocabulary and in several
WAYS = [("f32", 5, 300, 64), ("bf16", 5, 300, 64), ("bf16", 20, 700, 129), ("f32", 100, 200, 64), ("f32", 300, 701, 137), ("bf16", 300, 700, 136), ("bf16", 1500, 6200, 130),
        ("bf16", 15510, 6200, 520), ("f32", 1500, 6200, 130), ("f32", 700, 12301, 132), ("f32", 20000, 4099, 136), ("f32", 40000, 2200, 129)]


def without_first_column(dtype, tokens, vocab, width):
    c = Case(tokens, vocab, width, DT[dtype], gaps=tokens > 100)
    c.x.t[:, 0] = 0
    c.w.t[:, 0] = 0
    return c, c.exact()


def check(c, exact, z, tokens=slice(None)):
    """Against logits z that hold -inf; `exact`: of the same layer without the first column, which makes them."""
    x, w, _, ez, _, off = exact
    lse = torch.logsumexp(z, 1)
    n = torch.arange(len(z), device=DEV)
    hit = z[n, c.at]
    tol = off + 4 * U * lse.abs()
    within(c.lse[tokens], torch.where(c.live, lse, 0)[tokens], tol[tokens], "lse")
    within(c.loss[tokens], torch.where(c.live, lse - hit, 0)[tokens], (tol + ez[n, c.at] + 2 * U * (lse.abs() + hit.abs().nan_to_num(posinf=0)))[tokens], "loss")
    if isinstance(tokens, torch.Tensor):
        return
    up = torch.where(c.live & (c.dloss != 0), c.dloss.double(), 0)[:, None]
    p = torch.exp(z - lse[:, None])
    share = (ez.amax(1) + off)[:, None] + 4 * U * (z.abs().nan_to_num(posinf=0) + lse.abs()[:, None]) + 4 * U
    dz = p * up
    dz[n, c.at] -= up[:, 0]
    half = HALF[c.dt] if c.dt == torch.bfloat16 else U
    wrong = p * up.abs() * share + (half + 2 * U) * dz.abs()
    del p, share
    vocab, tokens = z.shape[1], z.shape[0]
    want, size = (dz @ w)[:, 1:], (dz.abs() @ w.abs())[:, 1:]
    within(c.dx.t[:, 1:], want, (wrong @ w.abs())[:, 1:] * (1 + half) + (vocab + 40) * U * size + HALF[c.dt] * want.abs(), "dx")
    dzt, wt = dz.t().contiguous(), wrong.t().contiguous()
    want, size = (dzt @ x)[:, 1:], (dzt.abs() @ x.abs())[:, 1:]
    within(c.dw.t[:, 1:], want, (wt @ x.abs())[:, 1:] * (1 + half) + (tokens + 40) * U * size + HALF[c.dt] * want.abs(), "dw")


@pytest.mark.parametrize("dtype,tokens,vocab,width", WAYS)
def test_one_logit_that_overflows(dtype, tokens, vocab, width):
    c, exact = without_first_column(dtype, tokens, vocab, width)
    t = int(c.live.nonzero()[0])
    v = (int(c.at[t]) + vocab // 2) % vocab
    c.w.t[v, 0] = 1.3 * 2.0 ** 100
    c.x.t[t, 0] = -1.1 * 2.0 ** 100
    z = exact[2].clone()
    z[t, v] = -float("inf")
    c.forward().backward()
    check(c, exact, z)
    assert bool(c.dx.t.isfinite().all()) and bool(c.dw.t.isfinite().all())
    c.x.t[t, 0] = 1.1 * 2.0 ** 100
    c.forward()
    assert not bool(c.loss[t].isfinite()) and not bool(c.lse[t].isfinite())
    check(c, exact, exact[2], torch.arange(tokens, device=DEV) != t)


@pytest.mark.parametrize("dtype,tokens,vocab,width", WAYS)
def test_a_class_of_infinite_weight(dtype, tokens, vocab, width):
    """Its logits are -inf for all tokens: no token's loss knows of it but that of the one whose target it is."""
    c, exact = without_first_column(dtype, tokens, vocab, width)
    v, t = vocab - 2, int(c.live.nonzero()[-1])
    c.at = torch.where(c.at == v, 0, c.at)
    c.at[t] = v
    c.targets.copy_(torch.where(c.live, c.at, c.targets))
    c.x.t[:, 0] = 1 + torch.rand(tokens, generator=gen(1), device=DEV)
    c.w.t[v, 0] = -float("inf")
    z = exact[2].clone()
    z[:, v] = -float("inf")
    c.forward().backward()
    assert float(c.loss[t]) == float("inf") and bool(c.lse.isfinite().all())
    check(c, exact, z)


@pytest.mark.parametrize("tokens,vocab,width", [(600, 12301, 200), (6200, 1100, 257), (30001, 2400, 130)])
def test_numbers_of_many_sizes_in_three_parts(tokens, vocab, width):
    """Columns from 2^-35 to 2^35, which parts can hold; and to 2^60, whose products are those of the numbers themselves."""
    for most in (35, 60):
        c = Case(tokens, vocab, width, torch.float32)
        power = torch.exp2(torch.randint(-most, most + 1, (width,), generator=gen(3), device=DEV).float())
        power[0] = 2.0 ** most
        c.x.put(c.x.t * power)
        c.w.put(c.w.t / power)
        c.forward().check_forward(most)
        c.backward().check_backward(most)


@pytest.mark.parametrize("dtype,tokens,vocab,width", [("f32", 1500, 6200, 130), ("f32", 20000, 4099, 136)])
def test_a_large_number_leaves_nothing_behind(dtype, tokens, vocab, width):
    """A call with infinite weights in a workspace, then one without: its bits are those of the first call of all."""
    c = Case(tokens, vocab, width, DT[dtype])
    c.forward().backward()
    outs = (c.loss, c.lse, c.dx.t, c.dw.t)
    want = [t.clone() for t in outs]
    ws = torch.empty(max(f(c.dt, tokens, vocab, width) for f in (kt.kt_linear_xent_fwd_workspace, kt.kt_linear_xent_bwd_workspace)), dtype=torch.uint8, device=DEV)
    row = c.w.t[vocab - 1].clone()
    for _ in range(2):
        c.w.t[vocab - 1] = float("inf")
        c.forward(workspace=ws).backward(workspace=ws)
        c.w.t[vocab - 1] = row
        c.forward(workspace=ws).backward(workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


@pytest.mark.parametrize("dtype,tokens,vocab,width", WAYS)
def test_only_logits_of_minus_infinity(dtype, tokens, vocab, width):
    """Nothing is left to divide by: the loss of each token with a target is not finite, the others' is 0."""
    c, _ = without_first_column(dtype, tokens, vocab, width)
    c.x.t[:, 0] = 1
    c.w.t[:, 0] = -float("inf")
    c.forward()
    assert not bool(c.loss[c.live].isfinite().any()) and not c.loss[~c.live].any() and not c.lse[~c.live].any()

"""bf16 gradients stand no further from their definition than rounding them once leaves them, and the roundings of the elements of dz that are no target's.

A bf16 number of 8 bits is off by half a step at most, 2^-8 of its power of two, evenly spread: by 2^-8 / sqrt(3) of that power, which is below 2^-8 / sqrt(3) of the number and, over
a power of two, 0.83 * 2^-9 of it in the root of the mean square.  dz of a token (unit dloss) is the target's element and others of norm r of it; the directions of w's rows (and x's) are
random, so that a gradient's relative error is at most sqrt(e^2 + (2^-9 r)^2), e that of rounding it once.  A tenth more for the spread of some thousands of numbers about it."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV
from test_gpu_linear_xent import Case

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def check(c):
    tokens, vocab, width = c.shape
    x, w, z, _, lse, _ = c.exact()
    dz = torch.exp(z - lse[:, None])
    n = torch.arange(tokens, device=DEV)
    dz[n, c.at] -= 1
    dz *= torch.where(c.live, c.dloss.double(), 0)[:, None]
    others = dz.clone()
    others[n, c.at] = 0
    bound = 2.0 ** -9 * float(others.norm() / dz.norm())
    for got, want in ((c.dx.t, dz @ w), (c.dw.t, dz.t().contiguous() @ x)):
        once = off(want.to(BF16), want)
        assert off(got, want) <= 1.1 * (once ** 2 + bound ** 2) ** 0.5, (off(got, want), once, bound)


# tokens in registers and in tiles of every size, sums of pieces of the tokens and of the vocabulary, several pieces of the vocabulary with carried sums and without, and more
# rows to a tile than a list has
@pytest.mark.parametrize("tokens,vocab,width,gap,off_", [(1, 5003, 2048, 0, 0), (5, 300, 1000, 0, 0), (16, 1000, 1001, 3, 1), (33, 1000, 768, 0, 0), (105, 1000, 2048, 0, 0),
                                                         (256, 5003, 1024, 0, 0), (257, 5003, 1003, 1, 1), (810, 1000, 1024, 8, 8), (3000, 4200, 136, 0, 0),
                                                         (15329, 300, 1024, 0, 0), (9000, 70, 512, 0, 0), (300001, 33, 24, 0, 0), (20000, 7003, 72, 0, 0), (65536, 4200, 128, 0, 0)])
def test_gradients(tokens, vocab, width, gap, off_):
    c = Case(tokens, vocab, width, BF16, gap, off_, gaps=tokens > 100)
    c.dloss.fill_(1 / tokens)
    c.forward().backward()
    check(c)


@pytest.mark.parametrize("tokens,vocab,width", [(40, 700, 520), (700, 700, 520), (5000, 900, 264)])
def test_targets_that_many_tokens_share(tokens, vocab, width):
    """Half of the tokens one target, dloss of either sign, some 0; and each gradient alone."""
    c = Case(tokens, vocab, width, BF16, gaps=False)
    c.targets[::2] = 7
    c.at = c.targets.long()
    c.dloss[1::5] = 0
    c.forward().backward()
    check(c)
    for which, want in (("dx", c.dx.t), ("dw", c.dw.t)):
        got = torch.empty_like(want)
        kt.kt_linear_xent_bwd(c.dloss, c.x.t, c.w.t, c.targets, c.lse, **{which: got})
        assert torch.equal(got, want)

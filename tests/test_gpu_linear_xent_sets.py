"""f32 logits are as near as sums in sets of 128 products, not as one sum of thousands, whatever makes them.

The model, u = 2^-24: an addition rounds its sum s by up to u 2^e, 2^e <= |s|, evenly spread, a deviation of at most u |s| / sqrt(3).  The sums s are computed in 64 bits:
each product within its set and each set's.  (Instructions that add several products at once round less often, and parts of 8 bits are exact.)  The loss rounds three times more, the
difference with the largest logit, the logarithm and their sum, each at the size of what it makes.  The log-sum-exp has the logits' errors in proportion to p.  Over the tokens
the root of the mean square stays within 1.5 times that: of 40 tokens on it spreads by an eighth about its own mean."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, U, gen, normal

pytestmark = pytest.mark.gpu

SET = 128


def deviation(prods):
    """Of sums along the last dimension (a multiple of 128): products one after another in a set, then sets."""
    sets = prods.unflatten(-1, (-1, SET))
    within, total = sets.cumsum(-1), sets.sum(-1).cumsum(-1)
    return ((within ** 2).sum((-1, -2)) + (total ** 2).sum(-1)).mul(U * U / 3).sqrt()


# up to 16 tokens in registers; tiles of 64 and of 128; numbers in three parts, from 80 tiles of 256 x 128 on
@pytest.mark.parametrize("tokens,vocab,width", [(16, 700, 8192), (200, 300, 8192), (90, 1153, 1024), (2000, 1600, 4096), (1200, 2304, 4096), (300, 7000, 4096)])
def test_loss(tokens, vocab, width):
    off, rows, model = 0.0, 0, 0.0
    for seed in range(4 if tokens < 100 else 1):
        g = gen(seed)
        w, x = normal(g, vocab, width, scale=width ** -0.5), normal(g, tokens, width)
        t = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
        loss, lse = torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV)
        kt.kt_linear_xent_fwd(x, w, t, loss, lse)
        z = x.double() @ w.double().t().contiguous()
        n = torch.arange(tokens, device=DEV)
        want = torch.logsumexp(z, 1) - z[n, t]
        hit = deviation(x.double() * w[t].double())
        p2 = torch.softmax(z, 1).square().sum(1)
        top = z.amax(1)
        rounds = (U * U / 3) * ((top - z[n, t]) ** 2 + (torch.logsumexp(z, 1) - top) ** 2 + want ** 2)
        off += float(((loss.double() - want) ** 2).sum())
        model += float((hit ** 2 * (1 + p2) + rounds).sum())
        rows += tokens
    assert (off / rows) ** 0.5 <= 1.5 * (model / rows) ** 0.5, ((off / rows) ** 0.5, (model / rows) ** 0.5)


@pytest.mark.parametrize("tokens,vocab,width", [(100, 300, 8192), (600, 700, 4096)])
def test_one_sum_after_another_would_be_rounded_away(tokens, vocab, width):
    """Products of 1 and a little, whose little is less than half a step of a sum of thousands of them: off by (128 + width / 128 + 2) u of the sum at most."""
    x = torch.full((tokens, width), 1.0, device=DEV)
    w = torch.full((vocab, width), 1.0 + 0.4 * 2.0 ** -11, device=DEV)
    t = torch.zeros(tokens, dtype=torch.int64, device=DEV)
    loss, lse = torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV)
    kt.kt_linear_xent_fwd(x, w, t, loss, lse)
    z = float(w[0, 0]) * width
    want = z + float(torch.log(torch.tensor(vocab, dtype=torch.float64)))
    assert float((lse.double() - want).abs().max()) <= (SET + width / SET + 2) * U * z + 8 * U * want

"""Gradients of likely targets where the vocabulary is taken in pieces, with an lse that has none of the kernels' roundings: as near their definition as in one
piece (tolerances: test_targets_that_are_likely, whose check this is)."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, gen
from test_gpu_linear_xent import Case
from test_gpu_linear_xent import test_targets_that_are_likely as check_likely

pytestmark = pytest.mark.gpu

# more dz than 2^27 elements, 2^26 in three parts; more of a weight at odd addresses than is copied at a time: few tokens, tiles
SHAPES = [(20000, 6657, 40), (30001, 2400, 130), (16500, 4100, 264), (70, 9500, 8191), (5, 9001, 16383), (130, 5001, 8191)]


@pytest.mark.parametrize("tokens,vocab,width", SHAPES)
def test_in_several_pieces(tokens, vocab, width):
    check_likely(tokens, vocab, width)


@pytest.mark.parametrize("tokens,vocab,width", [(30001, 2400, 130), (70, 9500, 8191)])
def test_one_gradient_only_and_the_same_bits_every_time(tokens, vocab, width):
    """With repeated targets, tokens that take no part, whatever the workspace held, and rows at odd places."""
    c = Case(tokens, vocab, width, torch.float32, 3, 1, lean=16.0)
    c.targets[::3] = 7
    c.forward()
    c.dloss[torch.rand(tokens, generator=gen(2), device=DEV) < 0.1] = 0
    c.backward()
    dx, dw = c.dx.t.clone(), c.dw.t.clone()
    assert c.dx.intact() and c.dw.intact()
    ws = torch.empty(kt.kt_linear_xent_bwd_workspace(torch.float32, tokens, vocab, width), dtype=torch.uint8, device=DEV)
    for fill in (255, 0, 126):
        ws.fill_(fill)
        c.dx.t.fill_(7.0)
        c.dw.t.fill_(7.0)
        c.backward(workspace=ws)
        assert torch.equal(c.dx.t, dx) and torch.equal(c.dw.t, dw)
    for which, want in (("dx", dx), ("dw", dw)):
        got = torch.empty_like(want)
        kt.kt_linear_xent_bwd(c.dloss, c.x.t, c.w.t, c.targets, c.lse, **{which: got})
        assert torch.equal(got, want)

"""Ways of the cross entropy that only large calls take, against their definitions in 64 bits (tolerances: test_gpu_linear_xent.py), and what a workspace held
before a call, whatever way it takes.  Shapes follow from the rules that choose a way; each test names the rule."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, gen
from test_gpu_linear_xent import Case

pytestmark = pytest.mark.gpu


def with_others(tokens, vocab, width, dt, **more):
    """A case with tokens that take no part, whole tiles of them and single ones, and NaN in their rows."""
    c = Case(tokens, vocab, width, dt, **more)
    none = torch.zeros(tokens, dtype=torch.bool, device=DEV)
    none[tokens // 3:tokens // 3 + 300] = none[-3:] = True
    c.targets[none] = -100
    c.live = c.live & ~none
    c.at = torch.where(c.live, c.targets, 0).long()
    c.x.t[~c.live] = float("nan")
    return c


# the forward pass lists the tokens that take part from tokens * vocab * width of 5e10 on in bf16, an eighth of it in f32; f32 numbers are not taken in parts
# below a width of 128 or 256 tokens
@pytest.mark.parametrize("dtype,vocab,width,gap,off", [("bf16", 6200, 520, 0, 0), ("bf16", 6201, 519, 3, 1), ("f32", 10100, 126, 0, 0), ("f32", 10101, 124, 0, 0)])
def test_long_forward_passes_list_their_tokens(dtype, vocab, width, gap, off):
    tokens = int(5e10 / (8 if dtype == "f32" else 1) / vocab / width) + 1
    with_others(tokens, vocab, width, DT[dtype], gap=gap, off=off).forward().check_forward()


def test_a_long_forward_pass_of_few_tokens():
    with_others(255, 50304, 512, torch.float32).forward().check_forward()


# more dz than 2^27 elements (2^26 in three parts) is made in pieces of the vocabulary; so many tokens that a product over such a piece is not cut again, so that dx
# goes on from carried sums to its result at once; and fewer, where it is cut
@pytest.mark.parametrize("dtype,tokens,vocab,width", [("bf16", 65536, 4200, 128), ("f32", 65536, 4200, 128), ("f32", 140000, 1100, 36), ("bf16", 40000, 4201, 131),
                                                      ("f32", 30001, 2400, 130)])
def test_pieces_of_the_vocabulary_with_others(dtype, tokens, vocab, width):
    assert tokens * vocab > 1 << 26
    c = with_others(tokens, vocab, width, DT[dtype]).forward()
    c.dloss[torch.rand(tokens, generator=gen(1), device=DEV) < 0.1] = 0
    c.check_forward()
    c.backward().check_backward()


SEVERAL = [("bf16", 20000, 7003, 72), ("bf16", 65536, 4200, 128), ("f32", 20000, 6657, 40), ("f32", 20000, 4099, 136), ("f32", 70, 9500, 8191), ("bf16", 5, 9001, 16383)]


@pytest.mark.parametrize("dtype,tokens,vocab,width", SEVERAL)
def test_one_gradient_only_of_several_pieces(dtype, tokens, vocab, width):
    c = Case(tokens, vocab, width, DT[dtype]).forward().backward()
    dx, dw = torch.empty_like(c.dx.t), torch.empty_like(c.dw.t)
    kt.kt_linear_xent_bwd(c.dloss, c.x.t, c.w.t, c.targets, c.lse, dx=dx)
    kt.kt_linear_xent_bwd(c.dloss, c.x.t, c.w.t, c.targets, c.lse, dw=dw)
    assert torch.equal(dx, c.dx.t) and torch.equal(dw, c.dw.t)


# few tokens; tiles of every size; numbers in three parts; rows at odd places; several pieces of the vocabulary
@pytest.mark.parametrize("dtype,tokens,vocab,width,gap,off", [(*s, 0, 0) for s in SEVERAL] + [
    ("f32", 20, 700, 136, 0, 0), ("bf16", 7, 300, 129, 3, 1), ("f32", 300, 700, 132, 0, 0), ("f32", 300, 701, 131, 3, 1), ("bf16", 300, 700, 131, 1, 1),
    ("f32", 1500, 6200, 130, 0, 0), ("bf16", 3000, 4200, 136, 0, 0), ("f32", 1500, 2100, 100, 0, 0)])
def test_what_a_workspace_held_before_reaches_nothing(dtype, tokens, vocab, width, gap, off):
    """All of it NaN, zeros, or large numbers: the same bits every time, and nothing behind its end."""
    c = with_others(tokens, vocab, width, DT[dtype], gap=gap, off=off) if tokens > 900 else Case(tokens, vocab, width, DT[dtype], gap, off)
    c.forward().backward()
    outs = (c.loss, c.lse, c.dx.t, c.dw.t)
    first = [t.clone() for t in outs]
    needs = [f(c.dt, tokens, vocab, width) for f in (kt.kt_linear_xent_fwd_workspace, kt.kt_linear_xent_bwd_workspace)]
    ws = torch.empty(max(needs) + 64, dtype=torch.uint8, device=DEV)
    for fill in (255, 0, 126):
        for t in outs:
            t.fill_(7.0)
        for need, call in zip(needs, (c.forward, c.backward)):
            ws.fill_(fill)
            call(workspace=ws[:need])
            assert bool((ws[need:] == fill).all())
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
        assert c.dx.intact() and c.dw.intact()


@pytest.mark.parametrize("dtype,tokens,vocab,width", [("bf16", 12, 300, 72), ("bf16", 500, 700, 136), ("bf16", 20000, 7003, 72), ("f32", 500, 700, 136), ("f32", 1500, 6200, 130)])
def test_dloss_of_many_sizes(dtype, tokens, vocab, width):
    """Each token's row of dx is as near as with equal ones, though dz in bf16 is kept in units of the largest (2^-90 of it times a probability is above 2^-126)."""
    c = Case(tokens, vocab, width, DT[dtype]).forward()
    c.dloss.copy_(torch.exp2(torch.randint(-60, 31, (tokens,), generator=gen(4), device=DEV).float()) * torch.where(c.dloss < 0, -1, 1))
    c.backward().check_backward()

"""Cross entropy of a linear layer and its gradients against their definitions in 64 bits.

Tolerances, u = 2^-24.  A logit is a sum of `width` products: off by ez = (width + 2) u sum|x w|.  The log-sum-exp is off by the largest of
them, by its exponentials (of arguments below 128 in magnitude: 200 u) and their sum, fewer than 100 + vocab / 16 additions one after another, and by the logarithm and the sum with
the largest logit, 4 u |lse|.  An exponential p of the backward pass is off by a share of ez + that + 4 u (|z| + |lse|) + 4 u.  dz is rounded to the
operands' type, HALF of it in bf16 and u in f32; the products are sums of as many terms as the vocabulary or the tokens have, some 20 more for pieces, and rounded once."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, HALF, U, Placed, gen, normal, within

pytestmark = pytest.mark.gpu

IT = {32: torch.int32, 64: torch.int64}


def targets_of(g, n, vocab, gaps=True, it=64):
    t = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    if gaps:
        other = torch.tensor([-1, -100, vocab, vocab + 7, -2 ** 31, 2 ** 31 - 1], device=DEV)
        t = torch.where(torch.rand(n, generator=g, device=DEV) < 0.3, other[torch.randint(0, 6, (n,), generator=g, device=DEV)], t)
    return t.to(IT[it])


class Case:
    """x, w, targets and dloss, and what the definitions say of them."""

    def __init__(self, tokens, vocab, width, dt, gap=0, off=0, seed=0, gaps=True, it=64, lean=4.0):
        g = gen(seed + 3 * tokens + vocab + width)
        self.shape, self.dt = (tokens, vocab, width), dt
        self.targets = targets_of(g, tokens, vocab, gaps, it)
        w = normal(g, vocab, width, scale=width ** -0.5)
        self.live = (self.targets >= 0) & (self.targets < vocab)
        self.at = torch.where(self.live, self.targets, 0).long()
        self.w = Placed(vocab, width, dt, gap, off).put(w)
        self.x = Placed(tokens, width, dt, gap, off).put(normal(g, tokens, width) + lean * w[self.at])
        self.dloss = torch.rand(tokens, generator=g, device=DEV) - 0.3
        self.loss, self.lse = torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV)
        self.dx, self.dw = Placed(tokens, width, dt, gap + 1 if gap else 0, off), Placed(vocab, width, dt, gap + 2 if gap else 0, off)

    def forward(self, **more):
        kt.kt_linear_xent_fwd(self.x.t, self.w.t, self.targets, self.loss, self.lse, **more)
        return self

    def backward(self, **more):
        kt.kt_linear_xent_bwd(self.dloss, self.x.t, self.w.t, self.targets, self.lse, self.dx.t, self.dw.t, **more)
        return self

    def exact(self):
        tokens, vocab, width = self.shape
        x, w = self.x.t.double(), self.w.t.double()
        x = torch.where(self.live[:, None], x, 0)
        z = x @ w.t().contiguous()
        ez = (width + 2) * U * (x.abs() @ w.abs().t().contiguous()) if tokens * vocab < 1 << 25 else \
            (width + 2) * U * (x.norm(dim=1)[:, None] * w.norm(dim=1).max()).expand(tokens, vocab)
        lse = torch.logsumexp(z, 1)
        off = ez.amax(1) + (300 + vocab / 16) * U + 4 * U * lse.abs()
        return x, w, z, ez, lse, off

    def check_forward(self, what=""):
        _, _, z, ez, lse, off = self.exact()
        n = torch.arange(len(z), device=DEV)
        hit = z[n, self.at]
        within(self.lse, torch.where(self.live, lse, 0), torch.where(self.live, off, 0), what)
        tol = off + ez[n, self.at] + 2 * U * (lse.abs() + hit.abs())
        within(self.loss, torch.where(self.live, lse - hit, 0), torch.where(self.live, tol, 0), what)

    def check_backward(self, what="", dx=True, dw=True):
        tokens, vocab, _ = self.shape
        x, w, z, ez, lse, off = self.exact()
        up = torch.where(self.live & (self.dloss != 0), self.dloss.double(), 0)[:, None]
        p = torch.exp(z - lse[:, None])
        share = (ez.amax(1) + off)[:, None] + 4 * U * (z.abs() + lse.abs()[:, None]) + 4 * U
        dz = p * up
        dz[torch.arange(tokens, device=DEV), self.at] -= up[:, 0]
        half = HALF[self.dt] if self.dt == torch.bfloat16 else U
        wrong = p * up.abs() * share + (half + 2 * U) * dz.abs()        # of dz
        del p, z, share
        if dx:
            size = dz.abs() @ w.abs()
            want = dz @ w
            within(self.dx.t, want, wrong @ w.abs() * (1 + half) + (vocab + 40) * U * size + HALF[self.dt] * want.abs(), (what, "dx"))
            assert self.dx.intact()
        if dw:
            dzt, wt = dz.t().contiguous(), wrong.t().contiguous()
            size = dzt.abs() @ x.abs()
            want = dzt @ x
            within(self.dw.t, want, wt @ x.abs() * (1 + half) + (tokens + 40) * U * size + HALF[self.dt] * want.abs(), (what, "dw"))
            assert self.dw.intact()


SHAPES = [(1, 1, 1), (1, 7, 8), (2, 300, 64), (3, 1000, 100), (63, 65, 63), (64, 64, 64), (65, 129, 1001), (130, 500, 257), (257, 1023, 768),
          (300, 5003, 200), (1, 50304, 256), (33, 4099, 2048), (16, 4099, 72), (17, 4099, 72), (30, 17000, 2048), (30, 4099, 1001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,width", SHAPES)
def test_against_64_bits(tokens, vocab, width, dtype):
    for gap, off, it in ((0, 0, 64), (3, 1, 32), (8, 8, 64)):       # rows at multiples of 16 bytes where the width is one, and not
        c = Case(tokens, vocab, width, DT[dtype], gap, off, gaps=tokens > 1, it=it).forward()
        c.check_forward((gap, off))
        c.backward().check_backward((gap, off))


# tiles of 128 and 256 in each of the three products, with ends that fill no tile and no step; pieces of the tokens and of the vocabulary
@pytest.mark.parametrize("dtype,tokens,vocab,width", [
    ("bf16", 3000, 4200, 136), ("f32", 1500, 2100, 132), ("bf16", 1500, 2100, 136), ("bf16", 6200, 700, 2056), ("bf16", 700, 6200, 2056),
    ("f32", 3100, 300, 1028), ("f32", 300, 3100, 1028), ("bf16", 3100, 300, 1032), ("bf16", 300, 3100, 1032), ("bf16", 1024, 1000, 768), ("f32", 1024, 1000, 768)])
def test_tiles_and_pieces(dtype, tokens, vocab, width):
    Case(tokens, vocab, width, DT[dtype]).forward().backward().check_backward()
    c = Case(tokens, vocab, width, DT[dtype], seed=1).forward()
    c.check_forward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [8192, 8193, 300001])
def test_many_tokens(tokens, dtype):
    """Listed by workgroups that count for themselves, and in two launches."""
    c = Case(tokens, 33, 24, DT[dtype], it=32).forward()
    c.check_forward()
    c.backward().check_backward()


# f32 numbers in three parts: widths that fill no group of 32 and tiles that fill no 256 x 128, rows at odd places, pieces of the tokens and of the vocabulary
@pytest.mark.parametrize("tokens,vocab,width,gap,off", [(512, 12288, 128, 0, 0), (700, 12301, 132, 0, 0), (513, 12289, 129, 3, 1), (6200, 1100, 257, 8, 8),
                                                        (20000, 4099, 136, 1, 3), (1100, 5003, 1001, 0, 0)])
def test_numbers_in_three_parts(tokens, vocab, width, gap, off):
    c = Case(tokens, vocab, width, torch.float32, gap, off).forward()
    c.check_forward()
    c.backward().check_backward()


def test_numbers_in_three_parts_of_every_size():
    """From 2^-100 to 2^100, and the type's largest, whose nearest number of 8 bits is infinity: 100 columns that both sides have, products of 1 about."""
    g = gen(3)
    c = Case(600, 12301, 200, torch.float32, gaps=False)
    power = torch.exp2(torch.randint(-100, 101, (200,), generator=g, device=DEV).float())
    c.x.put(c.x.t * power)
    c.w.put(c.w.t / power)
    c.x.t[:, 0], c.w.t[:, 0] = torch.finfo(torch.float32).max, 2.0 ** -126
    c.forward().check_forward()
    c.backward().check_backward()


# more vocabulary than a piece of dz takes; more of a weight at odd addresses than is copied at a time
@pytest.mark.parametrize("dtype,tokens,vocab,width", [("bf16", 20000, 7003, 72), ("f32", 20000, 6657, 40), ("f32", 70, 9500, 8191), ("bf16", 5, 9001, 16383)])
def test_pieces_of_the_vocabulary(dtype, tokens, vocab, width):
    c = Case(tokens, vocab, width, DT[dtype]).forward()
    c.check_forward()
    c.backward().check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,width", [(700, 300, 100), (130, 90, 64), (3000, 4200, 136), (1500, 6200, 130)])
def test_tokens_that_take_no_part(dtype, tokens, vocab, width):
    """Whole tiles and steps of them, at the start, in between and at the end; what their rows hold reaches nothing."""
    c = Case(tokens, vocab, width, DT[dtype])
    none = torch.zeros(tokens, dtype=torch.bool, device=DEV)
    none[:tokens // 3] = none[tokens // 2:tokens // 2 + 70] = none[-5:] = True
    c.targets[none] = -100
    c.live = c.live & ~none
    c.at = torch.where(c.live, c.targets, 0).long()
    zero = torch.rand(tokens, generator=gen(9), device=DEV) < 0.2
    c.dloss[zero] = 0
    c.forward().check_forward()
    c.backward().check_backward()
    dx, dw = c.dx.t.clone(), c.dw.t.clone()
    for bad in (float("nan"), float("inf")):
        c.x.t[~c.live | zero] = bad
        c.dloss[~c.live] = bad
        c.lse[~c.live | zero] = bad
        c.backward()
        assert torch.equal(c.dx.t, dx) and torch.equal(c.dw.t, dw)
        assert not c.dx.t[~c.live | zero].any()
    c.forward()
    assert not c.loss[~c.live].any() and not c.lse[~c.live].any() and bool(c.loss[c.live & ~zero].isfinite().all())
    c.targets.fill_(-1)
    c.forward().backward()
    assert not c.loss.any() and not c.lse.any() and not c.dx.t.any() and not c.dw.t.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens(dtype):
    c = Case(5, 70, 90, DT[dtype])
    n = torch.empty(0, device=DEV)
    kt.kt_linear_xent_fwd(c.x.t[:0], c.w.t, c.targets[:0], n, n)
    c.dw.put(torch.ones(70, 90, device=DEV))
    kt.kt_linear_xent_bwd(n, c.x.t[:0], c.w.t, c.targets[:0], n, c.dx.t[:0], c.dw.t)
    assert not c.dw.t.any() and c.dw.intact()
    kt.kt_linear_xent_bwd(n, c.x.t[:0], c.w.t, c.targets[:0], n, c.dx.t[:0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_gradient_only_and_no_lse(dtype):
    c = Case(200, 300, 72, DT[dtype]).forward().backward()
    loss = torch.empty_like(c.loss)
    kt.kt_linear_xent_fwd(c.x.t, c.w.t, c.targets, loss)
    assert torch.equal(loss, c.loss)
    dx, dw = torch.empty_like(c.dx.t), torch.empty_like(c.dw.t)
    kt.kt_linear_xent_bwd(c.dloss, c.x.t, c.w.t, c.targets, c.lse, dx=dx)
    kt.kt_linear_xent_bwd(c.dloss, c.x.t, c.w.t, c.targets, c.lse, dw=dw)
    assert torch.equal(dx, c.dx.t) and torch.equal(dw, c.dw.t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(dtype):
    """Logits of a few thousand: nothing overflows, and one token's certainty leaves a gradient of 0 for the others."""
    c = Case(100, 200, 64, DT[dtype], gaps=False, lean=2000.0)
    c.forward()
    c.check_forward()
    assert bool(c.loss.isfinite().all())
    c.backward()
    assert bool(c.dx.t.isfinite().all()) and bool(c.dw.t.isfinite().all())


@pytest.mark.parametrize("tokens,vocab,width", [(100, 200, 64), (1500, 6200, 130)])
def test_logits_that_are_not_finite(tokens, vocab, width):
    c = Case(tokens, vocab, width, torch.float32, gaps=False)
    c.forward()
    want = c.loss.clone()
    c.x.t[7] = float("nan")
    c.x.t[9] = float("inf")
    c.forward()
    assert not bool(c.loss[7].isfinite()) and not bool(c.loss[9].isfinite())
    keep = torch.ones(tokens, dtype=torch.bool, device=DEV)
    keep[[7, 9]] = False
    assert torch.equal(c.loss[keep], want[keep])


@pytest.mark.parametrize("tokens,vocab,width", [(4, 1000, 4096), (30, 900, 520), (300, 700, 136), (700, 12301, 132)])
def test_targets_that_are_likely(tokens, vocab, width):
    """With an lse that has none of the kernels' roundings a target of probability p lacks as much of 1 as the others have: off by a share of 1 - p, not of p."""
    c = Case(tokens, vocab, width, torch.float32, gaps=False, lean=16.0)
    x, w = c.x.t.double(), c.w.t.double()
    z = x @ w.t().contiguous()
    ez = (width + 2) * U * (x.abs() @ w.abs().t().contiguous())
    lse = torch.logsumexp(z, 1)
    c.lse.copy_(lse)
    c.dloss.abs_()
    c.backward()
    n = torch.arange(tokens, device=DEV)
    p, share = torch.exp(z - lse[:, None]), ez + 5 * U * lse[:, None] + 4 * U * (z.abs() + 1)
    dz, wrong = p.clone(), p * share
    dz[n, c.at] = 0
    others, off = dz.sum(1), wrong.sum(1) - wrong[n, c.at]
    dz[n, c.at] = -others
    wrong[n, c.at] = torch.where(others < 0.49, off + (300 + vocab / 16) * U * others, wrong[n, c.at] + off)
    assert bool((others < 0.49).any())
    up = c.dloss.double()[:, None]
    dz, wrong = dz * up, wrong * up + 3 * U * dz.abs() * up
    want, size = dz @ w, dz.abs() @ w.abs()
    within(c.dx.t, want, wrong @ w.abs() * (1 + U) + (vocab + 40) * U * size + U * want.abs(), "dx")
    dzt, wt = dz.t().contiguous(), wrong.t().contiguous()
    want, size = dzt @ x, dzt.abs() @ x.abs()
    within(c.dw.t, want, wt @ x.abs() * (1 + U) + (tokens + 40) * U * size + U * want.abs(), "dw")


@pytest.mark.parametrize("tokens,vocab,width", [(3, 500, 264), (200, 300, 72), (3000, 300, 72)])
def test_a_common_dloss_is_not_rounded_to_bf16(tokens, vocab, width):
    """dz is rounded in units of the largest dloss: gradients of equal ones are in proportion but for their own two roundings."""
    c = Case(tokens, vocab, width, torch.bfloat16).forward()
    c.dloss.fill_(1.0)
    c.backward()
    dx, dw = c.dx.t.double(), c.dw.t.double()
    for up in (1 / 3, 0.7, 1e-20, 3e4):
        c.dloss.fill_(up)
        c.backward()
        up = float(c.dloss[0])
        for got, one in ((c.dx.t, dx), (c.dw.t, dw)):
            within(got, up * one, 2.01 * HALF[torch.bfloat16] * (up * one).abs(), up)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_dloss_that_is_not_finite(dtype):
    c = Case(200, 300, 72, DT[dtype], gaps=False).forward().backward()
    dx, largest = c.dx.t.clone(), int(c.dloss.abs().argmax())
    t = (largest + 1) % 200
    for bad in (float("inf"), float("nan")):
        c.dloss[t] = bad
        c.backward()
        others = torch.arange(200, device=DEV) != t
        assert torch.equal(c.dx.t[others], dx[others]) and not bool(c.dx.t[t].isfinite().all()) and not bool(c.dw.t.isfinite().all())


def test_gradient_against_differences():
    """Of the sum of dloss * loss: central differences with steps of h are off by h^2 of the third derivative (below 1 for logits' steps of h) and
    by twice the losses' own error over 2 h."""
    c = Case(90, 130, 40, torch.float32).forward().backward()
    h = 2.0 ** -6

    def value():
        c.forward()
        return float((c.loss.double() * c.dloss.double())[c.live].sum())

    for t, row, col, got in ((c.x.t, 5, 3, c.dx.t), (c.x.t, 77, 39, c.dx.t), (c.w.t, 0, 0, c.dw.t), (c.w.t, 129, 20, c.dw.t)):
        at = t[row, col].clone()
        got = float(got[row, col])
        t[row, col] = at + h
        up = value()
        step = float(t[row, col].double())
        t[row, col] = at - h
        down = value()
        step -= float(t[row, col].double())
        t[row, col] = at
        curve = float(c.x.t.double().abs().pow(3).sum(0).max() + 1) * h * h
        noise = 90 * 2 * (42 * U * 40 + 400 * U) / step
        assert abs((up - down) / step - got) <= curve + noise, (row, col)


def test_the_same_bits_every_time_and_with_a_workspace_of_the_callers():
    c = Case(1024, 1000, 136, torch.bfloat16).forward().backward()
    first = [t.clone() for t in (c.loss, c.lse, c.dx.t, c.dw.t)]
    needs = [f(torch.bfloat16, 1024, 1000, 136) for f in (kt.kt_linear_xent_fwd_workspace, kt.kt_linear_xent_bwd_workspace)]
    ws = torch.empty(max(needs) + 64, dtype=torch.uint8, device=DEV)
    for fill in (255, 0, 127):
        ws.fill_(fill)
        for t in (c.loss, c.lse, c.dx.t, c.dw.t):
            t.fill_(7.0)
        c.forward(workspace=ws[:needs[0]])
        assert bool((ws[needs[0]:] == fill).all())
        c.backward(workspace=ws[:needs[1]])
        assert bool((ws[max(needs):] == fill).all())
        assert all(torch.equal(a, b) for a, b in zip(first, (c.loss, c.lse, c.dx.t, c.dw.t)))


@pytest.mark.parametrize("dtype,tokens,vocab,width", [("bf16", 300, 700, 136), ("f32", 300, 700, 129), ("bf16", 3000, 4200, 136), ("f32", 1500, 6200, 130), ("f32", 20, 700, 136)])
def test_in_graphs_and_on_another_stream(dtype, tokens, vocab, width):
    """Two recorded calls share a workspace; their replays follow each other."""
    c = Case(tokens, vocab, width, DT[dtype]).forward().backward()
    outs = (c.loss, c.lse, c.dx.t, c.dw.t)
    want = [t.clone() for t in outs]
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        for t in outs:
            t.zero_()
        s.wait_stream(torch.cuda.current_stream())
        c.forward(stream=stream).backward(stream=stream)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
    ws = torch.empty(max(f(c.dt, tokens, vocab, width) for f in (kt.kt_linear_xent_fwd_workspace, kt.kt_linear_xent_bwd_workspace)), dtype=torch.uint8,
                     device=DEV)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        c.forward(workspace=ws)
    with torch.cuda.graph(graphs[1]):
        c.backward(workspace=ws)
    for seed in (1, 2, 3):
        c.x.put(normal(gen(seed), tokens, width))
        c.targets.copy_(targets_of(gen(seed), tokens, vocab))
        c.forward().backward()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


@pytest.mark.parametrize("dtype,width,off", [("bf16", 33, 0), ("bf16", 64, 0), ("f32", 64, 0)])
def test_written_into_a_bucket(dtype, width, off):
    plan = kt.Plan([7, 90 * width, 5], dtype, 0, 16)
    bucket = [torch.full((n,), 3.0, dtype=DT[dtype], device=DEV) for n in plan.bucket_elems()]
    b, at = plan.tensor_info(1)
    c = Case(200, 90, width, DT[dtype]).forward().backward()
    view = bucket[b][at:at + 90 * width].view(90, width)
    kt.kt_linear_xent_bwd(c.dloss, c.x.t, c.w.t, c.targets, c.lse, dw=view)
    assert torch.equal(view, c.dw.t)
    view.fill_(3.0)
    assert all(bool((x == 3.0).all()) for x in bucket)

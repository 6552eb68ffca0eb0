"""Layer norm forward and backward against the formulas in 64 bits.

Tolerances.  u = 2^-24.  A sum over a row adds at most 32 terms in a lane and at most 10 levels across lanes and wavefronts: 42
roundings, with those of the terms themselves K = 48.  Results are rounded once to the type: half a step, HALF.
  mean: K u mean|x|;  variance: relative (2 K + 4) u + (error of the mean)^2 / variance;  rstd: half of that and 3 u.
  y: |g| rstd (error of the mean + u |x - mean|) + |xh g| (error of rstd + 2 u) + 2 u |y| + HALF |y|
  dx: rstd (4 u |t| + (K + 4) u mean|t| + |xh| (K + 10) u mean|t xh|) + 6 u |dx| + HALF |dx|
  dgamma, dbeta: a chain of L additions, L = rows of a wavefront + 4 + parts / 16 + 16 + 6: L u sum|terms| + HALF |sum|
"""
import math

import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, HALF, U, Placed, gen, normal, saved64, stands_for, within

pytestmark = pytest.mark.gpu

K = 48
EPS = 1e-5
SHAPES = [(1, 1), (2, 2), (5, 7), (197, 768), (3, 1001), (64, 1024), (33, 1025), (130, 2048), (9, 2049), (17, 4096), (6, 8192),
          (5, 8200), (3, 16384), (4, 16383), (20000, 40), (9000, 768)]


def inputs(rows, cols, dt, pdt, seed, gap=0, off=0):
    g = gen(seed)
    x = Placed(rows, cols, dt, gap, off).put(normal(g, rows, cols) * 1.7 + normal(g, rows, 1))
    gamma = (1 + 0.3 * normal(g, cols)).to(pdt)
    beta = (0.2 * normal(g, cols)).to(pdt)
    return g, x, gamma, beta


def forward64(x, gamma, beta):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = 1 / (var + EPS).sqrt()
    xh = (x - mean) * rstd
    y = xh * gamma.double() + (0 if beta is None else beta.double())
    e_mean = K * U * x.abs().mean(1, keepdim=True)
    e_rstd = ((K + 2) * U + 0.5 * e_mean.square() / (var + EPS) + 3 * U)                  # relative
    tol = gamma.double().abs() * rstd * (e_mean + U * (x - mean).abs()) + (xh * gamma.double()).abs() * (e_rstd + 2 * U) + 2 * U * y.abs()
    return y, mean, rstd, tol, e_mean, e_rstd * rstd


def backward64(dy, x, gamma, mean, rstd, out_type):
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xh, t = (x - mean) * rstd, dy * gamma.double()
    m = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    dx = rstd * (t - m(t) - xh * m(t * xh))
    tol = rstd * (4 * U * t.abs() + (K + 4) * U * m(t.abs()) + xh.abs() * (K + 10) * U * m((t * xh).abs())) + (6 * U + HALF[out_type]) * dx.abs()
    rows = dy.shape[0]
    L = math.ceil(rows / 4) if rows < 8192 else math.ceil(rows / 512)
    L = L + 4 + 32 + 16 + 6
    return dx, tol, ((dy * xh).sum(0), L * U * (dy * xh).abs().sum(0)), (dy.sum(0), L * U * dy.abs().sum(0))


@pytest.mark.parametrize("pdtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rows, cols, dtype, pdtype):
    gap, off = (0, 0) if cols % 2 == 0 else (5, 3)
    dt, pdt = DT[dtype], DT[pdtype]
    _, x, gamma, beta = inputs(rows, cols, dt, pdt, rows + cols, gap, off)
    y = Placed(rows, cols, dt, gap, off)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    q, e = [torch.full(s, 99, dtype=d, device=DEV) for s, d in zip(kt.kt_act8_shapes(rows, cols), (torch.int8, torch.uint8))]
    kt.kt_layernorm_fwd(x.t, gamma, beta, EPS, y.t, mean, rstd, y8=(q, e))
    want, m, r, tol, tm, tr = forward64(x.t, gamma, beta)
    within(mean[:, None], m, tm, "mean")
    within(rstd[:, None], r, tr, "rstd")
    within(y.t, want, tol + HALF[dt] * want.abs(), "y")
    assert y.intact()
    qw, ew = saved64(y.t)                   # of the y that was stored
    assert torch.equal(e, ew) and torch.equal(q, qw)
    # without a checkpoint, bias and statistics; over x itself
    y2 = Placed(rows, cols, dt, gap, off).put(x.t)
    kt.kt_layernorm_fwd(y2.t, gamma, None, EPS, y2.t)
    want, _, _, tol, _, _ = forward64(x.t, gamma, None)
    within(y2.t, want, tol + HALF[dt] * want.abs(), "y without bias")
    assert y2.intact()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("pdtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_backward(rows, cols, dtype, pdtype, eight):
    gap, off = (0, 0) if cols % 2 == 0 else (5, 3)
    dt, pdt = DT[dtype], DT[pdtype]
    g, x, gamma, _ = inputs(rows, cols, dt, pdt, rows + cols, gap, off)
    dy = Placed(rows, cols, dt, gap + 1, off).put(normal(g, rows, cols))
    _, m, r, _, _, _ = forward64(x.t, gamma, None)
    mean, rstd = m[:, 0].float(), r[:, 0].float()
    given, used = x.t, x.t
    if eight:
        given = saved64(x.t)
        used = stands_for(*given, cols)
    dx = Placed(rows, cols, dt, gap, off)
    bucket = torch.full((2 * cols + 7,), 5.0, device=DEV).to(pdt)               # the gradients lie in a bucket, side by side
    dgamma, dbeta = bucket[3:3 + cols], bucket[3 + cols:3 + 2 * cols]
    kt.kt_layernorm_bwd(dy.t, given, gamma, mean, rstd, dx.t, dgamma, dbeta)
    want, tol, (dg, tg), (db, tb) = backward64(dy.t, used, gamma, mean, rstd, dt)
    within(dx.t, want, tol, "dx")
    within(dgamma, dg, tg + HALF[pdt] * dg.abs(), "dgamma")
    within(dbeta, db, tb + HALF[pdt] * db.abs(), "dbeta")
    assert dx.intact() and bool((bucket[:3] == 5).all()) and bool((bucket[3 + 2 * cols:] == 5).all())
    # over dy itself, without dbeta, with a workspace that the caller keeps: the same bits
    ws = torch.full((kt.kt_layernorm_bwd_workspace(rows, cols) + 256,), 255, dtype=torch.uint8, device=DEV)
    dg2 = torch.empty(cols, dtype=pdt, device=DEV)
    kt.kt_layernorm_bwd(dy.t, given, gamma, mean, rstd, dy.t, dg2, workspace=ws[:-256])
    assert torch.equal(dy.t, dx.t) and torch.equal(dg2, dgamma) and bool((ws[-256:] == 255).all())


def test_gradient_by_differences():
    """The backward pass is the derivative of the forward pass: f(x + h d) - f(x - h d) = 2 h <grad, d> + O(h^3).  f32 with
    values of order 1: the difference carries 2 * 24 roundings of y each, <|y|, |w|> 60 u, over 2 h; the cubic term is
    taken out by Richardson's step."""
    rows, cols = 6, 37
    g = gen(5)
    x, w, gamma, beta = normal(g, rows, cols), normal(g, rows, cols), 1 + 0.3 * normal(g, cols), normal(g, cols)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)

    def f(x, gamma, beta):
        kt.kt_layernorm_fwd(x, gamma, beta, EPS, y, mean, rstd)
        return float((y.double() * w.double()).sum())

    f(x, gamma, beta)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    kt.kt_layernorm_bwd(w, x, gamma, mean.clone(), rstd.clone(), dx, dg, db)
    size = float((y.double().abs() * w.double().abs()).sum()) + float(w.abs().sum()) * 4
    for which, grad in ((0, dx), (1, dg), (2, db)):
        d = normal(g, *grad.shape)
        at = [x, gamma, beta]

        def slope(h):
            v = []
            for sign in (1, -1):
                moved = list(at)
                moved[which] = at[which] + sign * h * d
                v.append(f(*moved))
            return (v[0] - v[1]) / (2 * h)

        h = 2.0 ** -5
        got = (4 * slope(h / 2) - slope(h)) / 3
        want = float((grad.double() * d.double()).sum())
        assert abs(got - want) <= 3 * 60 * U * size / h + 60 * h ** 4 * size, (which, got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_rows(dtype):
    dt = DT[dtype]
    x = torch.empty(0, 768, dtype=dt, device=DEV)
    gamma = torch.ones(768, dtype=dt, device=DEV)
    none = torch.empty(0, device=DEV)
    kt.kt_layernorm_fwd(x, gamma, gamma, EPS, torch.empty_like(x), none, torch.empty(0, device=DEV))
    dg, db = torch.full_like(gamma, 3), torch.full_like(gamma, 3)
    kt.kt_layernorm_bwd(x, torch.empty_like(x), gamma, none, none, torch.empty_like(x), dg, db)
    assert not dg.any() and not db.any()


def test_a_row_that_is_not_finite_stays_alone():
    x = normal(gen(6), 40, 768)
    clean = x.clone()
    x[7, 100] = float("nan")
    x[20, 3] = float("inf")
    gamma = torch.ones(768, device=DEV)
    out = []
    for v in (x, clean):
        y, mean, rstd = torch.empty_like(v), torch.empty(40, device=DEV), torch.empty(40, device=DEV)
        dx, dg = torch.empty_like(v), torch.empty_like(gamma)
        kt.kt_layernorm_fwd(v, gamma, None, EPS, y, mean, rstd)
        kt.kt_layernorm_bwd(clean, v, gamma, mean, rstd, dx, dg)
        out.append((y, dx, mean, rstd))
    rest = [i for i in range(40) if i not in (7, 20)]
    for a, b in zip(*out):
        assert torch.equal(a[rest], b[rest])
        assert a[[7, 20]].isnan().any()


def test_constant_rows_and_far_means():
    """A row of one value has variance 0; a mean far from 0 does not cost the variance its digits."""
    x = torch.full((4, 512), 3.25, device=DEV)
    x[1] = 0
    x[2] = 4096 + torch.arange(512, device=DEV) % 2                 # exact sums
    gamma = torch.ones(512, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    kt.kt_layernorm_fwd(x, gamma, None, EPS, y, mean, rstd)
    want = (x.double() - x.double().mean(1, keepdim=True)) / (x.double().var(1, correction=0, keepdim=True) + EPS).sqrt()
    within(y, want, 8 * U * want.abs())


def test_in_a_graph_and_on_another_stream():
    rows, cols = 700, 2048
    g = gen(8)
    x, dy, gamma = normal(g, rows, cols, dtype=torch.bfloat16), normal(g, rows, cols, dtype=torch.bfloat16), normal(g, cols, dtype=torch.bfloat16)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    y, dx, dg, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)

    def step(stream=None):
        kt.kt_layernorm_fwd(x, gamma, gamma, EPS, y, mean, rstd, stream=stream)
        kt.kt_layernorm_bwd(dy, x, gamma, mean, rstd, dx, dg, db, stream=stream)

    step()
    want = [t.clone() for t in (y, dx, dg, db)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for stream in (s, s.cuda_stream):
        for t in (y, dx, dg, db):
            t.zero_()
        s.wait_stream(torch.cuda.current_stream())
        step(stream)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dg, db), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3):
        x.copy_(normal(gen(seed), rows, cols))
        step()
        want = [t.clone() for t in (y, dx, dg, db)]
        for t in (y, dx, dg, db):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dg, db), want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [41, 47, 82, 768, 1001, 2998, 8198])
def test_a_constant_gradient_has_no_effect_through_the_mean(cols, dtype):
    """t = 1 in every column and xh = 0: dx = 1 - mean(t) with the exact sum `cols`, whose division is exact."""
    dt = DT[dtype]
    x, dy = torch.zeros(5, cols, dtype=dt, device=DEV), torch.ones(5, cols, dtype=dt, device=DEV)
    gamma = torch.ones(cols, device=DEV)
    mean, rstd = torch.zeros(5, device=DEV), torch.ones(5, device=DEV)
    dx, dgamma = torch.full_like(x, 5.0), torch.empty_like(gamma)
    kt.kt_layernorm_bwd(dy, x, gamma, mean, rstd, dx, dgamma)
    assert not dx.any()


@pytest.mark.parametrize("pdtype", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_three_chunks_a_lane_of_four_wavefronts(dtype, pdtype):
    """5 000 columns of bf16, 2 500 of f32."""
    cols = 5000 if dtype == "bf16" else 2500
    test_forward(7, cols, dtype, pdtype)
    for eight in (False, True):
        test_backward(7, cols, dtype, pdtype, eight)

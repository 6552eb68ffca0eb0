"""The embedding lookup and its gradient against their definitions in 64 bits.

Tolerances: the lookup is one product in binary32, u |want|, and the rounding to the output's type.  A row of the gradient is a sum of n_v
terms, at most n_v + 16 additions one after another (the pieces' own zeros and the join), the product with the scale and, where it is added to what is
there, one more: (n_v + 18) u sum|terms| + HALF |want|."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, HALF, U, Placed, gen, normal, within

pytestmark = pytest.mark.gpu

IT = {32: torch.int32, 64: torch.int64}
WIDTHS = [1, 7, 8, 64, 255, 513, 1001, 2048, 4100]


def tokens_of(g, n, vocab, kind="text", it=64):
    """Token ids; a tenth of them name no token where the kind is `gaps`."""
    if kind == "one":
        t = torch.full((n,), vocab // 2, device=DEV)
    elif kind == "none":
        t = torch.full((n,), -1, device=DEV)
    elif kind == "even":
        t = torch.randint(0, vocab, (n,), generator=g, device=DEV)
    else:
        t = (torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * torch.log(torch.tensor(vocab + 1.0))).exp().long().sub(1).clamp(0, vocab - 1)
    if kind == "gaps":
        other = torch.tensor([-1, -100, vocab, vocab + 7, -2 ** 31, 2 ** 31 - 1], device=DEV)
        t = torch.where(torch.rand(n, generator=g, device=DEV) < 0.3, other[torch.randint(0, 6, (n,), generator=g, device=DEV)], t)
    return t.to(IT[it])


def alive(ids, vocab):
    return (ids >= 0) & (ids < vocab)


def looked_up(ids, w, scale):
    at = torch.where(alive(ids, w.shape[0]), ids, w.shape[0]).long()
    return torch.cat([w.double(), torch.zeros(1, w.shape[1], dtype=torch.float64, device=DEV)])[at] * scale


def collected(ids, dy, vocab, scale):
    """(sum, sum of magnitudes, terms) for every row of the table."""
    keep = alive(ids, vocab)
    at, rows = ids[keep].long(), dy[keep].double() * scale
    zero = torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device=DEV)
    return zero.clone().index_add_(0, at, rows), zero.index_add_(0, at, rows.abs()), torch.bincount(at, minlength=vocab)


def check(dw, ids, dy, scale, before=None, what=""):
    want, size, n = collected(ids, dy, dw.shape[0], scale)
    if before is not None:
        want, size = want + before.double(), size + before.double().abs()
        assert torch.equal(dw[n == 0], before[n == 0])
    else:
        assert not dw[n == 0].any()
    within(dw, want, (n[:, None] + 18) * U * size + HALF[dw.dtype] * want.abs(), what)


@pytest.mark.parametrize("dtype,table", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("width", WIDTHS)
def test_lookup(width, dtype, table):
    for n, vocab, it, gap, off in ((1, 1, 32, 0, 0), (1, 50, 64, 0, 0), (67, 300, 64, 3, 1), (1000, 40, 32, 8, 0)):
        g = gen(width + n)
        w = Placed(vocab, width, DT[table], gap, off).put(normal(g, vocab, width))
        y = Placed(n, width, DT[dtype], gap + 1 if gap else 0, off)
        ids = tokens_of(g, n, vocab, "gaps" if n > 1 else "even", it)
        kt.kt_embedding_fwd(ids, w.t, y.t, scale=width ** 0.5)
        want = looked_up(ids, w.t, float(torch.tensor(width ** 0.5)))
        within(y.t, want, (U + HALF[DT[dtype]]) * want.abs(), (n, vocab))
        assert y.intact()


def test_lookup_of_a_batch_and_without_tokens():
    g = gen(1)
    w, ids = normal(g, 90, 130), tokens_of(g, 24, 90).view(2, 3, 4)
    y = torch.empty(2, 3, 4, 130, device=DEV)
    kt.kt_embedding_fwd(ids, w, y)
    assert torch.equal(y, w[ids])
    kt.kt_embedding_fwd(ids[:0].reshape(0), w, torch.empty(0, 130, device=DEV))
    dw = normal(g, 90, 130)
    before = dw.clone()
    kt.kt_embedding_bwd(ids[:0].reshape(0), torch.empty(0, 130, device=DEV), dw, accumulate=True)
    assert torch.equal(dw, before)
    kt.kt_embedding_bwd(ids[:0].reshape(0), torch.empty(0, 130, device=DEV), dw)
    assert not dw.any()


def test_what_is_not_finite_stays_in_its_row():
    """A row of the table reaches its own tokens only; a row of dy its own token's, and none where there is no token."""
    g = gen(2)
    w, ids = normal(g, 50, 96), tokens_of(g, 400, 50, "gaps")
    w[7], w[9] = float("nan"), float("inf")
    y = torch.empty(400, 96, device=DEV)
    kt.kt_embedding_fwd(ids, w, y, scale=0.0)
    assert bool(y[(ids == 7) | (ids == 9)].isnan().all()) and not y[(ids != 7) & (ids != 9)].any()
    dy = normal(g, 400, 96)
    dy[~alive(ids, 50)] = float("nan")
    dy[ids == 3] = float("inf")
    dw = torch.empty(50, 96, device=DEV)
    kt.kt_embedding_bwd(ids, dy, dw)
    assert bool((dw[3] == float("inf")).all()) and bool(dw[:3].isfinite().all()) and bool(dw[4:].isfinite().all())


# up to 256 tokens are not sorted, up to 4 096 by one workgroup; digits of 8 or 9 bits: one, two or three of them
@pytest.mark.parametrize("kind", ["text", "even", "one", "none", "gaps"])
@pytest.mark.parametrize("n,vocab", [(1, 1), (2, 3), (7, 2), (8, 9), (9, 1), (63, 100), (197, 1000), (256, 90), (257, 90), (1025, 40), (4096, 5003), (4097, 5003), (6000, 1),
                                     (9001, 1023), (9001, 1024), (20000, 70000), (35000, 300), (4100, 1 << 20)])
def test_gradient(n, vocab, kind):
    width = 40 if vocab > 60000 else 100
    for dtype, table, it in (("f32", "f32", 32), ("bf16", "bf16", 64)):
        g = gen(n + vocab)
        ids, dy = tokens_of(g, n, vocab, kind, it), normal(g, n, width, dtype=DT[dtype])
        dw = Placed(vocab, width, DT[table])
        kt.kt_embedding_bwd(ids, dy, dw.t, scale=3.25)
        check(dw.t, ids, dy, 3.25, None, (dtype, table))
        assert dw.intact()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,table", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("width", WIDTHS)
def test_gradient_of_any_width(width, dtype, table, accumulate):
    for n, vocab, gap, off in ((200, 37, 0, 0), (200, 37, 3, 1), (300, 37, 0, 0), (300, 37, 3, 1), (5000, 900, 8, 0)):
        g = gen(width + n)
        ids = tokens_of(g, n, vocab, "gaps")
        dy = Placed(n, width, DT[dtype], gap, off).put(normal(g, n, width))
        dw = Placed(vocab, width, DT[table], gap + 1 if gap else 0, off).put(normal(g, vocab, width))
        before = dw.t.clone()
        kt.kt_embedding_bwd(ids, dy.t, dw.t, scale=-0.5, accumulate=accumulate)
        check(dw.t, ids, dy.t, -0.5, before if accumulate else None, (n, gap))
        assert dw.intact()


def test_gradient_against_differences():
    """The lookup is linear in the table: with a step of a power of two the difference of two values is exact but for their rounding."""
    g = gen(5)
    n, vocab, width = 700, 60, 33
    w, ids, dy = normal(g, vocab, width), tokens_of(g, n, vocab, "gaps"), normal(g, n, width)
    dw = torch.empty(vocab, width, device=DEV)
    kt.kt_embedding_bwd(ids, dy, dw, scale=1.5)

    def value(table):
        y = torch.empty(n, width, device=DEV)
        kt.kt_embedding_fwd(ids, table, y, scale=1.5)
        return (y.double() * dy.double()).sum(), (y.double().abs() * dy.double().abs()).sum()

    for v, c in ((0, 0), (1, 32), (7, 5), (59, 20)):
        up, down = w.clone(), w.clone()
        up[v, c] += 1
        down[v, c] -= 1
        (a, size), (b, _) = value(up), value(down)
        step = float(up[v, c].double() - down[v, c].double())
        assert abs(float(a - b) / step - float(dw[v, c])) <= 2 * U * float(size) / step + (n + 18) * U * float(dy[ids == v].abs().sum() * 1.5)


def test_the_same_bits_every_time_and_with_a_workspace_of_the_callers():
    g = gen(6)
    ids, dy = tokens_of(g, 9000, 500), normal(g, 9000, 264, dtype=torch.bfloat16)
    dw = torch.empty(500, 264, dtype=torch.bfloat16, device=DEV)
    need = kt.kt_embedding_bwd_workspace(9000, 500, 264)
    assert need > 0 and kt.kt_embedding_bwd_workspace(0, 500, 264) == 0
    kt.kt_embedding_bwd(ids, dy, dw)
    first = dw.clone()
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    for _ in range(5):
        dw.fill_(7.0)
        kt.kt_embedding_bwd(ids, dy, dw, workspace=ws[:need])
        assert torch.equal(dw, first) and bool((ws[need:] == 255).all())


@pytest.mark.parametrize("n", [200, 300, 9000])
def test_in_graphs_and_on_another_stream(n):
    """Two recorded calls share a workspace; their replays follow each other."""
    g = gen(7)
    vocab, width = 700, 200
    ids, dy, w = tokens_of(g, n, vocab, "gaps"), normal(g, n, width), normal(g, vocab, width)
    dw, other, y = torch.empty(vocab, width, device=DEV), torch.empty(vocab, width, device=DEV), torch.empty(n, width, device=DEV)
    kt.kt_embedding_bwd(ids, dy, dw)
    want = dw.clone()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        dw.zero_()
        s.wait_stream(torch.cuda.current_stream())
        kt.kt_embedding_bwd(ids, dy, dw, stream=stream)
        kt.kt_embedding_fwd(ids, dw, y, stream=stream)
        s.synchronize()
        assert torch.equal(dw, want) and torch.equal(y, torch.where(alive(ids, vocab)[:, None], want[ids.clamp(0, vocab - 1)], 0))
    ws = torch.empty(max(kt.kt_embedding_bwd_workspace(n, vocab, width), 16), dtype=torch.uint8, device=DEV)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        kt.kt_embedding_fwd(ids, w, y)
        kt.kt_embedding_bwd(ids, dy, dw, workspace=ws)
    with torch.cuda.graph(graphs[1]):
        kt.kt_embedding_bwd(ids, y, other, workspace=ws, accumulate=True)
    for seed in (1, 2, 3):
        dy.copy_(normal(gen(seed), n, width))
        ids.copy_(tokens_of(gen(seed), n, vocab, "gaps"))
        other.fill_(1.0)
        eager, eager2, y2 = torch.empty_like(dw), torch.ones_like(other), torch.empty_like(y)
        kt.kt_embedding_fwd(ids, w, y2)
        kt.kt_embedding_bwd(ids, dy, eager)
        kt.kt_embedding_bwd(ids, y2, eager2, accumulate=True)
        y.zero_()
        dw.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(dw, eager) and torch.equal(other, eager2)


def test_written_into_a_bucket():
    """The table's gradient where the plan keeps it: the bucket equals the one that packing makes."""
    plan = kt.Plan([7, 90 * 33, 5], "bf16", 0, 16)
    packed, direct = [[torch.zeros(n, dtype=torch.bfloat16, device=DEV) for n in plan.bucket_elems()] for _ in range(2)]
    g = gen(8)
    ids, dy = tokens_of(g, 500, 90, "gaps"), normal(g, 500, 33, dtype=torch.bfloat16)
    own = [torch.full((7,), 2.5, dtype=torch.bfloat16, device=DEV), torch.empty(90, 33, dtype=torch.bfloat16, device=DEV),
           torch.full((5,), -1.5, dtype=torch.bfloat16, device=DEV)]
    kt.kt_embedding_bwd(ids, dy, own[1])
    for t, x in enumerate(own):
        b, at = plan.tensor_info(t)
        view = direct[b][at:at + x.numel()].view(x.shape)
        if t == 1:
            kt.kt_embedding_bwd(ids, dy, view)
        else:
            view.copy_(x)
    plan.kt_bucket_pack(-1, own, packed)
    assert all(torch.equal(a, b) for a, b in zip(packed, direct))

"""The weight gradient from an 8-bit checkpoint against the product in 64 bits.

Tolerance: products of bf16 pairs are exact, those of f32 carry one rounding; the sum over t is a chain of at most `tokens`
additions and 16 pieces: (tokens + 20) u sum|terms| + HALF |sum|, u = 2^-24."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, HALF, U, Placed, gen, normal, saved64, stands_for, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 1), (1, 64, 33), (3, 5, 7), (15, 64, 64), (16, 65, 100), (33, 130, 257), (197, 768, 768), (257, 100, 2304),
          (2100, 96, 130), (700, 1001, 1001), (300, 1793, 1800), (200, 3600, 3700)]


def case(tokens, out, inn, dt, gdt, gap=0, off=0, seed=0):
    g = gen(seed + tokens + out + inn)
    x = normal(g, tokens, inn, dtype=dt) * (1 + 3 * torch.rand(tokens, 1, generator=g, device=DEV)).to(dt)
    q, e = saved64(x)
    dy = Placed(tokens, out, dt, gap, off).put(normal(g, tokens, out))
    return dy, q, e, Placed(out, inn, gdt, gap + 1 if gap else 0, off)


def check(dy, q, e, dw, inn, what=""):
    x, d = stands_for(q, e, inn), dy.double()
    want, size = d.t().contiguous() @ x, d.abs().t().contiguous() @ x.abs()
    within(dw, want, (dy.shape[0] + 20) * U * size + HALF[dw.dtype] * want.abs(), what)


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("tokens,out,inn", SHAPES)
def test_against_64_bits(tokens, out, inn, dtype, grad):
    for gap, off in ((0, 0), (3, 1)):
        dy, q, e, dw = case(tokens, out, inn, DT[dtype], DT[grad], gap, off)
        kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
        check(dy.t, q, e, dw.t, inn)
        assert dw.intact()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens(dtype):
    dy, q, e, dw = case(0, 70, 90, DT[dtype], DT[dtype])
    kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
    assert not dw.t.any()


def test_the_same_bits_every_time_and_with_a_workspace_of_the_callers():
    dy, q, e, dw = case(2100, 96, 130, torch.bfloat16, torch.bfloat16)
    need = kt.kt_act8_weight_grad_workspace(torch.bfloat16, 2100, 96, 130)
    assert need > 0
    kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
    first = dw.t.clone()
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)
    kt.kt_act8_weight_grad(dy.t, q, e, dw.t, workspace=ws[:need])
    assert torch.equal(dw.t, first) and bool((ws[need:] == 255).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_group_that_is_not_finite_reaches_its_columns_only(dtype):
    dy, q, e, dw = case(300, 200, 260, DT[dtype], DT[dtype])
    kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
    want = dw.t.clone()
    e[123, 2] = 255
    q[123, 64:96] = 0
    kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
    assert bool(dw.t[:, 64:96].isnan().all())
    assert torch.equal(dw.t[:, :64], want[:, :64]) and torch.equal(dw.t[:, 96:], want[:, 96:])


def test_in_a_graph_and_on_another_stream():
    dy, q, e, dw = case(2100, 96, 130, torch.bfloat16, torch.float32)
    kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
    want = dw.t.clone()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        dw.t.zero_()
        s.wait_stream(torch.cuda.current_stream())
        kt.kt_act8_weight_grad(dy.t, q, e, dw.t, stream=stream)
        s.synchronize()
        assert torch.equal(dw.t, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
    for seed in (1, 2, 3):
        dy.put(normal(gen(seed), 2100, 96))
        kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
        want = dw.t.clone()
        dw.t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw.t, want)


def test_written_into_a_bucket():
    """The gradient goes straight to where the plan keeps it: the bucket equals the one that packing makes."""
    shapes = [(96, 130), (7,), (70, 33)]
    plan = kt.Plan([96 * 130, 7, 70 * 33], "bf16", 0, 16)
    made = []
    packed, direct = [[torch.zeros(n, dtype=torch.bfloat16, device=DEV) for n in plan.bucket_elems()] for _ in range(2)]
    for t, shape in enumerate(shapes):
        b, at = plan.tensor_info(t)
        view = direct[b][at:at + plan.numels[t]].view(shape)
        if len(shape) == 1:
            view.fill_(2.5)
            made.append(view.clone())
            continue
        dy, q, e, dw = case(500, shape[0], shape[1], torch.bfloat16, torch.bfloat16)
        kt.kt_act8_weight_grad(dy.t, q, e, view)
        kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
        made.append(dw.t.contiguous())
    plan.kt_bucket_pack(-1, made, packed)
    assert all(torch.equal(a, b) for a, b in zip(packed, direct))


# Tiles of 128 and 256 and their pieces: 192 to 255 tiles and 512 tokens or more are cut in two, no whole step at their ends.
@pytest.mark.parametrize("dtype,grad,pieces,tokens,out,inn", [
    ("bf16", "bf16", 1, 300, 1792, 1800), ("bf16", "f32", 2, 1111, 1792, 1800), ("f32", "f32", 1, 300, 1792, 1800), ("f32", "bf16", 2, 1111, 1792, 1800),
    ("bf16", "bf16", 1, 300, 3600, 3700), ("bf16", "bf16", 2, 1111, 3600, 3700), ("bf16", "f32", 2, 1111, 3592, 3490)])
def test_tiles_and_pieces(dtype, grad, pieces, tokens, out, inn):
    need = kt.kt_act8_weight_grad_workspace(DT[dtype], tokens, out, inn)
    assert need == (0 if pieces == 1 else pieces * out * ((inn + 3) // 4 * 4) * 4)
    for gap, off in ((0, 0), (3, 1)):               # rows of dy at multiples of 16 bytes, and not
        dy, q, e, dw = case(tokens, out, inn, DT[dtype], DT[grad], gap, off)
        kt.kt_act8_weight_grad(dy.t, q, e, dw.t)
        check(dy.t, q, e, dw.t, inn, (gap, off))
        assert dw.intact()

"""Activation checkpoints in 8 bits: bytes and scales equal those of the definition in 64 bits, bit for bit."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, Placed, gen, normal, saved64, stands_for, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (7, 64), (5, 100), (197, 768), (129, 1001), (1, 5000), (4099, 40), (300, 2048)]


def checkpoint(rows, cols):
    qs, es = kt.kt_act8_shapes(rows, cols)
    return torch.full(qs, 77, dtype=torch.int8, device=DEV), torch.full(es, 77, dtype=torch.uint8, device=DEV)


def values(g, rows, cols, dtype):
    """Groups of many magnitudes, from 2^-126 to 2^120, zeros among them."""
    x = torch.randn(rows, cols, generator=g, device=DEV)
    groups = (cols + 31) // 32
    power = torch.randint(-126, 121, (rows, groups), generator=g, device=DEV).double()
    x = (x.double() * torch.exp2(power).repeat_interleave(32, 1)[:, :cols]).float()
    x[torch.rand(rows, cols, generator=g, device=DEV) < 0.05] = 0.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("gap,off", [(0, 0), (3, 1), (16, 5)])
def test_bytes_and_values(rows, cols, dtype, gap, off):
    g = gen(rows * 31 + cols)
    x = Placed(rows, cols, DT[dtype], gap, off).put(values(g, rows, cols, DT[dtype]))
    q, e = checkpoint(rows, cols)
    kt.kt_act8_save(x.t, q, e)
    qw, ew = saved64(x.t)
    assert torch.equal(e, ew) and torch.equal(q, qw)
    y = Placed(rows, cols, DT[dtype], gap, off)
    kt.kt_act8_restore(q, e, y.t)
    assert torch.equal(y.t.double(), stands_for(q, e, cols))       # every value is exact in either type
    assert y.intact()
    # half a step of the group's scale, one step where the member is clamped
    step = torch.exp2(e.double() - 127).repeat_interleave(32, 1)[:, :cols]
    within(y.t, x.t, torch.where(x.t.double().abs() > 127.5 * step, step, step / 2), "restored")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_values(dtype):
    dt = DT[dtype]
    x = torch.zeros(12, 64, dtype=dt, device=DEV)
    x[1, 3] = float("inf")
    x[2, 40] = float("nan")
    x[2, 41] = float("inf")
    x[3, 0] = float("-inf")
    x[4, 5] = torch.finfo(dt).max
    x[5, 6] = -torch.finfo(dt).max
    x[6, 7] = torch.finfo(dt).tiny
    x[7, :] = -0.0
    x[8, :32] = torch.arange(32, device=DEV).to(dt) + 0.5             # ties
    x[8, 0] = 127.0
    x[9, :32] = 1.0 - 2.0 ** -8                                       # 127.5 steps of 2^-7: clamped
    x[10, 33] = 2.0 ** -133                                           # below the smallest normal number
    x[11, 34] = 2.0 ** -120
    q, e = checkpoint(12, 64)
    kt.kt_act8_save(x, q, e)
    qw, ew = saved64(x)
    assert torch.equal(e, ew) and torch.equal(q, qw)
    y = torch.empty_like(x)
    kt.kt_act8_restore(q, e, y)
    nan = torch.zeros(12, 64, dtype=torch.bool, device=DEV)
    nan[1, :32] = nan[2, 32:] = nan[3, :32] = True
    assert torch.equal(y.isnan(), nan)
    assert torch.equal(y.double().nan_to_num(), stands_for(q, e, 64).nan_to_num())


def test_no_rows_and_leading_dimensions():
    q, e = checkpoint(0, 64)
    kt.kt_act8_save(torch.empty(0, 64, device=DEV), q, e)
    kt.kt_act8_restore(q, e, torch.empty(0, 64, device=DEV))
    x = normal(gen(1), 3, 5, 96)
    q, e = checkpoint(15, 96)
    kt.kt_act8_save(x, q, e)
    assert torch.equal(q, saved64(x.view(15, 96))[0])


def test_on_another_stream_and_in_a_graph():
    x = normal(gen(2), 513, 1001, dtype=torch.bfloat16)
    q, e = checkpoint(513, 1001)
    y = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    kt.kt_act8_save(x, q, e, stream=s)
    kt.kt_act8_restore(q, e, y, stream=s.cuda_stream)
    s.synchronize()
    want = stands_for(*saved64(x), 1001)
    assert torch.equal(y.double(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kt.kt_act8_save(x, q, e)
        kt.kt_act8_restore(q, e, y)
    for seed in (3, 4, 5):
        x.copy_(normal(gen(seed), 513, 1001, dtype=torch.bfloat16))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.double(), stands_for(*saved64(x), 1001))

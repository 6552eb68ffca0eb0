"""Rows and tokens far apart: offsets of more than 2^31 elements and 2^32 bytes.  The results are those of the same kernels on rows that
lie close, bit for bit."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, gen, normal

pytestmark = pytest.mark.gpu

ROWS = 600


class Row:
    """Matrices side by side in rows `ld` elements apart; each starts `off` elements past a multiple of 64."""

    def __init__(self, ld, off, dtype):
        self.buf, self.ld, self.at, self.off = torch.empty((ROWS - 1) * ld + 20000, dtype=dtype, device=DEV), ld, 0, off

    def window(self, cols, value=None):
        t = self.buf.as_strided((ROWS, cols), (self.ld, 1), self.at + self.off)
        self.at += (cols + 127) // 64 * 64
        assert self.at < 20000 and self.at <= self.ld
        t.copy_(value) if value is not None else t.fill_(7.0)
        return t


def far_and_near(far, off, dtype, run):
    """Outputs of `run` on rows far apart and on rows that lie close, both at multiples of 16 bytes or both not."""
    out = []
    for ld in (far, 20000 + off):
        out.append([t.clone() for t in run(Row(ld, off, dtype))])
        torch.cuda.synchronize()
    assert len(out[0]) == len(out[1]) and all(torch.equal(a, b) for a, b in zip(*out))
    assert all(bool(t.any()) for t in out[0])


@pytest.mark.parametrize("dtype,far,off", [("bf16", 1 << 22, 0), ("bf16", (1 << 22) + 1, 1), ("f32", 1 << 22, 0), ("f32", (1 << 22) + 1, 3)])
def test_layernorm_and_checkpoints(dtype, far, off):
    dt, g = DT[dtype], gen(1)
    x, dy, gamma = normal(g, ROWS, 1000, dtype=dt), normal(g, ROWS, 1000, dtype=dt), normal(g, 1000, dtype=dt)

    def run(row):
        a, d, y, dx, z = row.window(1000, x), row.window(1000, dy), row.window(1000), row.window(1000), row.window(1000)
        mean, rstd = torch.empty(ROWS, device=DEV), torch.empty(ROWS, device=DEV)
        q, e = (torch.empty(s, dtype=t, device=DEV) for s, t in zip(kt.kt_act8_shapes(ROWS, 1000), (torch.int8, torch.uint8)))
        dg, db = torch.empty_like(gamma), torch.empty_like(gamma)
        kt.kt_layernorm_fwd(a, gamma, gamma, 1e-5, y, mean, rstd)
        kt.kt_layernorm_bwd(d, a, gamma, mean, rstd, dx, dg, db)
        kt.kt_act8_save(a, q, e)
        kt.kt_act8_restore(q, e, z)
        return y, mean, rstd, dx, dg, db, q, e, z

    far_and_near(far, off, dt, run)


# bf16 rows 2^23 apart are past what the loads into LDS address within a tile
@pytest.mark.parametrize("dtype,far,off", [("bf16", 1 << 22, 0), ("bf16", (1 << 22) + 1, 1), ("bf16", (1 << 23) + 1, 1), ("f32", (1 << 22) - 4, 0)])
def test_weight_gradient(dtype, far, off):
    dt, g = DT[dtype], gen(2)
    dy = normal(g, ROWS, 264, dtype=dt)
    q = torch.randint(-127, 128, (ROWS, 320), generator=g, device=DEV, dtype=torch.int8)
    e = torch.randint(118, 123, (ROWS, 10), generator=g, device=DEV, dtype=torch.uint8)

    def run(row):
        d, dw = row.window(264, dy), row.window(300)[:264]
        kt.kt_act8_weight_grad(d, q, e, dw)
        return (dw,)

    far_and_near(far, off, dt, run)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,far,off", [("bf16", 1 << 22, 0), ("bf16", (1 << 22) + 1, 1), ("bf16", (1 << 23) + 1, 1), ("f32", (1 << 22) - 4, 0),
                                           ("f32", (1 << 22) + 1, 1)])
def test_attention(dtype, far, off, causal):
    dt, g = DT[dtype], gen(3)
    values = [normal(g, ROWS, h * 128, dtype=dt) for h in (2, 1, 1, 2)]

    def run(row):
        q, k, v, do, o, dq, dk, dv = (t.unflatten(1, (-1, 128))[None] for t in [row.window(v.shape[1], v) for v in values] +
                                      [row.window(h * 128) for h in (2, 2, 1, 1)])
        lse = torch.empty(1, 2, ROWS, device=DEV)
        kt.kt_attention_fwd(q, k, v, o, lse, causal=causal)
        kt.kt_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, causal=causal)
        return o, lse, dq, dk, dv

    far_and_near(far, off, dt, run)

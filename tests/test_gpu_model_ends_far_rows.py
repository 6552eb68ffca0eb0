"""The embedding and the cross entropy on rows far apart: offsets of more than 2^31 elements and 2^32 bytes.  The results are those of the same kernels on
rows that lie close, bit for bit."""
import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, gen, normal
from test_gpu_ops_far_rows import ROWS, far_and_near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,far,off", [("bf16", 1 << 22, 0), ("bf16", (1 << 22) + 1, 1), ("f32", 1 << 22, 0), ("f32", (1 << 22) + 1, 3)])
@pytest.mark.parametrize("tokens", [ROWS, 200])
def test_embedding(dtype, far, off, tokens):
    dt, g = DT[dtype], gen(1)
    table, dy = normal(g, ROWS, 1000, dtype=dt), normal(g, ROWS, 1000, dtype=dt)
    ids = torch.randint(-1, ROWS, (tokens,), generator=g, device=DEV)
    ids[:5] = ROWS - 1

    def run(row):
        w, d, y, dw, add = row.window(1000, table), row.window(1000, dy), row.window(1000), row.window(1000), row.window(1000, dy)
        kt.kt_embedding_fwd(ids, w, y[:tokens], scale=1.5)
        kt.kt_embedding_bwd(ids, d[:tokens], dw, scale=1.5)
        kt.kt_embedding_bwd(ids, d[:tokens], add, scale=1.5, accumulate=True)
        return y, dw, add

    far_and_near(far, off, dt, run)


# bf16 rows 2^21 apart are the last that are taken as they are
@pytest.mark.parametrize("dtype,far,off", [("bf16", 1 << 21, 0), ("bf16", 1 << 22, 0), ("bf16", (1 << 22) + 1, 1), ("f32", 1 << 20, 0), ("f32", (1 << 22) - 4, 0),
                                           ("f32", (1 << 22) + 1, 1)])
@pytest.mark.parametrize("tokens", [ROWS, 20])
def test_cross_entropy(dtype, far, off, tokens):
    dt, g = DT[dtype], gen(2)
    xs, ws = normal(g, ROWS, 264, dtype=dt), normal(g, ROWS, 264, dtype=dt, scale=0.1)
    targets = torch.randint(-1, ROWS, (tokens,), generator=g, device=DEV)
    targets[0] = ROWS - 1
    dloss = torch.rand(tokens, generator=g, device=DEV)

    def run(row):
        x, w, dx, dw = row.window(264, xs), row.window(264, ws), row.window(264), row.window(264)
        loss, lse = torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV)
        kt.kt_linear_xent_fwd(x[:tokens], w, targets, loss, lse)
        kt.kt_linear_xent_bwd(dloss, x[:tokens], w, targets, lse, dx[:tokens], dw)
        return loss, lse, dx, dw

    far_and_near(far, off, dt, run)

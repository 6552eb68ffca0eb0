"""What the cross entropy calls refuse, before any GPU is touched, and how much workspace they ask for."""
import pytest
import torch

import paper_2505_10183_amd as kt
from paper_2505_10183_amd import ops
from test_host_ops import BF16, EALIGN, EINVAL, EUNSUPPORTED, F32, M, at, call

FWD = dict(dt=F32, it=1, tokens=64, vocab=100, width=64, x=at(0), ldx=64, w=at(1), ldw=64, targets=at(2), loss=at(3), lse=at(4), ws=at(5),
           ws_bytes=8 * M, stream=0)
BWD = dict(dt=F32, it=1, tokens=64, vocab=100, width=64, dloss=at(3), x=at(0), ldx=64, w=at(1), ldw=64, targets=at(2), lse=at(4), dx=at(6), lddx=64,
           dw=at(7), lddw=64, ws=at(8), ws_bytes=8 * M, stream=0)
BOTH = [
    (dict(dt=2), EINVAL, "type"), (dict(dt=-1), EINVAL, "type"), (dict(it=2), EINVAL, "type"), (dict(tokens=-1), EINVAL, "tokens"),
    (dict(vocab=0), EINVAL, "vocab"), (dict(vocab=-3), EINVAL, "vocab"), (dict(width=0), EINVAL, "width"), (dict(ldx=63), EINVAL, "ld"),
    (dict(ldw=63), EINVAL, "ld"), (dict(tokens=1 << 60), EINVAL, "tokens"), (dict(ldw=1 << 62), EINVAL, "ld"),
    (dict(tokens=(1 << 24) + 1), EUNSUPPORTED, "2^24"), (dict(vocab=(1 << 24) + 1), EUNSUPPORTED, "2^24"),
    (dict(x=0), EINVAL, "NULL"), (dict(w=0), EINVAL, "NULL"), (dict(targets=0), EINVAL, "NULL"), (dict(ws=0), EINVAL, "workspace"),
    (dict(ws_bytes=100), EINVAL, "workspace"), (dict(x=at(0) + 2), EALIGN, "x"), (dict(w=at(1) + 2), EALIGN, "w"),
    (dict(targets=at(2) + 4), EALIGN, "targets"), (dict(targets=at(2) + 2, it=0), EALIGN, "targets"), (dict(lse=at(4) + 2), EALIGN, "lse"),
    (dict(dt=BF16, x=at(0) + 1), EALIGN, "x"), (dict(ws=at(0)), EINVAL, "overlaps"), (dict(ws=at(2)), EINVAL, "overlaps"), (dict(ws=at(1)), EINVAL, "overlaps")]


@pytest.mark.parametrize("changes,status,word", BOTH + [
    (dict(width=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), EUNSUPPORTED, "2^20"),
    (dict(tokens=1 << 24, width=1 << 13, ldx=1 << 13, ldw=1 << 13), EUNSUPPORTED, "2^36"),
    (dict(vocab=1 << 24, width=1 << 13, ldx=1 << 13, ldw=1 << 13), EUNSUPPORTED, "2^36"),
    (dict(loss=0), EINVAL, "NULL"), (dict(loss=at(3) + 1), EALIGN, "loss"), (dict(ws=at(5) + 8), EALIGN, "ws"), (dict(loss=at(4)), EINVAL, "overlaps"),
    (dict(loss=at(0) + 4 * 4095), EINVAL, "overlaps"), (dict(lse=at(1)), EINVAL, "overlaps"), (dict(lse=at(2)), EINVAL, "overlaps"),
    (dict(loss=at(5)), EINVAL, "overlaps")])
def test_fwd_refuses(changes, status, word):
    call("kt_linear_xent_fwd", FWD, status, word, **changes)


@pytest.mark.parametrize("changes,status,word", BOTH + [
    (dict(width=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21, lddx=1 << 21, lddw=1 << 21), EUNSUPPORTED, "2^20"),
    (dict(lddx=63), EINVAL, "ld"), (dict(lddw=63), EINVAL, "ld"), (dict(dx=0, dw=0), EINVAL, "NULL"), (dict(dloss=0), EINVAL, "NULL"),
    (dict(lse=0), EINVAL, "NULL"), (dict(dx=at(6) + 2), EALIGN, "dx"), (dict(dw=at(7) + 2), EALIGN, "dw"), (dict(dloss=at(3) + 2), EALIGN, "dloss"),
    (dict(ws=at(8) + 8), EALIGN, "ws"), (dict(dx=at(0)), EINVAL, "overlaps"), (dict(dw=at(1)), EINVAL, "overlaps"), (dict(dx=at(7)), EINVAL, "overlaps"),
    (dict(dw=at(0) + 4 * 4095), EINVAL, "overlaps"), (dict(dx=at(2)), EINVAL, "overlaps"), (dict(dw=at(3)), EINVAL, "overlaps"),
    (dict(dw=at(4)), EINVAL, "overlaps"), (dict(ws=at(7)), EINVAL, "overlaps"), (dict(ws=at(6)), EINVAL, "overlaps")])
def test_bwd_refuses(changes, status, word):
    call("kt_linear_xent_bwd", BWD, status, word, **changes)


def test_workspace():
    L = ops._library()
    for f in (L.kt_linear_xent_fwd_workspace, L.kt_linear_xent_bwd_workspace):
        assert f(F32, 0, 100, 64) == 0 and f(2, 5, 100, 64) == 0 and f(F32, -1, 100, 64) == 0 and f(F32, 5, 100, 1 << 21) == 0
        assert f(F32, 1, 1, 1) > 0
    # dz in 2^27 elements, sums and a copy of x, 128 MiB of the weight, whatever the vocabulary, and what the last piece of it is cut into
    for v in (50304, 1 << 20, 1 << 24):
        assert L.kt_linear_xent_bwd_workspace(BF16, 16384, v, 2048) < 2 * (1 << 27) + 16384 * 2048 * (2 + 4) + (128 << 20) + 64 * 8192 * 2048 * 4


def test_binding_refuses():
    f, n, i = torch.zeros(4, 8), torch.zeros(4), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="current GPU"):
        kt.kt_linear_xent_fwd(f, f, i, n)
    with pytest.raises(ValueError, match="current GPU"):
        kt.kt_linear_xent_bwd(n, f, f, i, n, f)

"""What the embedding calls refuse, before any GPU is touched."""
import math

import pytest
import torch

import paper_2505_10183_amd as kt
from paper_2505_10183_amd import ops
from test_host_ops import EALIGN, EINVAL, EUNSUPPORTED, F32, M, at, call

EMBED_FWD = dict(dt=F32, wdt=F32, it=1, tokens=64, vocab=100, width=64, ids=at(0), w=at(1), ldw=64, scale=1.0, y=at(2), ldy=64, stream=0)
EMBED_BWD = dict(dt=F32, wdt=F32, it=1, tokens=512, vocab=100, width=64, ids=at(0), dy=at(1), lddy=64, scale=1.0, dw=at(2), lddw=64, accumulate=0,
                 ws=at(3), ws_bytes=M, stream=0)
EMBED_SIZES = [
    (dict(dt=2), EINVAL, "type"), (dict(wdt=-1), EINVAL, "type"), (dict(it=2), EINVAL, "type"), (dict(tokens=-1), EINVAL, "tokens"),
    (dict(vocab=0), EINVAL, "vocab"), (dict(vocab=-5), EINVAL, "vocab"), (dict(width=0), EINVAL, "width"),
    (dict(tokens=(1 << 30) + 1), EUNSUPPORTED, "2^30"), (dict(vocab=(1 << 30) + 1), EUNSUPPORTED, "2^30"), (dict(tokens=1 << 60), EINVAL, "tokens"),
    (dict(scale=math.nan), EINVAL, "scale"), (dict(scale=math.inf), EINVAL, "scale"), (dict(ids=0), EINVAL, "NULL"),
    (dict(ids=at(0) + 4), EALIGN, "ids"), (dict(ids=at(0) + 2, it=0), EALIGN, "ids")]


@pytest.mark.parametrize("changes,status,word", EMBED_SIZES + [
    (dict(ldw=63), EINVAL, "ld"), (dict(ldy=63), EINVAL, "ld"), (dict(width=(1 << 24) + 1, ldw=1 << 25, ldy=1 << 25), EUNSUPPORTED, "2^24"),
    (dict(w=0), EINVAL, "NULL"), (dict(y=0), EINVAL, "NULL"), (dict(w=at(1) + 2), EALIGN, "w"), (dict(y=at(2) + 2), EALIGN, "y"),
    (dict(y=at(0)), EINVAL, "overlaps"), (dict(y=at(0) + 8 * 63), EINVAL, "overlaps"), (dict(y=at(1) + 4 * 6399), EINVAL, "overlaps"),
    (dict(y=at(1)), EINVAL, "overlaps")])
def test_embedding_fwd_refuses(changes, status, word):
    call("kt_embedding_fwd", EMBED_FWD, status, word, **changes)


@pytest.mark.parametrize("changes,status,word", EMBED_SIZES + [
    (dict(lddy=63), EINVAL, "ld"), (dict(lddw=63), EINVAL, "ld"), (dict(width=(1 << 24) + 1, lddy=1 << 25, lddw=1 << 25), EUNSUPPORTED, "2^24"),
    (dict(dy=0), EINVAL, "NULL"), (dict(dw=0), EINVAL, "NULL"), (dict(dw=0, tokens=0), EINVAL, "NULL"), (dict(ws=0), EINVAL, "workspace"),
    (dict(ws_bytes=1), EINVAL, "workspace"), (dict(dy=at(1) + 2), EALIGN, "dy"), (dict(dw=at(2) + 2), EALIGN, "dw"), (dict(ws=at(3) + 8), EALIGN, "ws"),
    (dict(dw=at(0)), EINVAL, "overlaps"), (dict(dw=at(1) + 4 * 32767), EINVAL, "overlaps"), (dict(ws=at(2)), EINVAL, "overlaps"),
    (dict(ws=at(1)), EINVAL, "overlaps"), (dict(ws=at(0)), EINVAL, "overlaps")])
def test_embedding_bwd_refuses(changes, status, word):
    call("kt_embedding_bwd", EMBED_BWD, status, word, **changes)


def test_embedding_workspace():
    L = ops._library()
    assert L.kt_embedding_bwd_workspace(0, 100, 64) == 0 and L.kt_embedding_bwd_workspace(-1, 100, 64) == 0
    assert L.kt_embedding_bwd_workspace(1 << 31, 100, 64) == 0 and L.kt_embedding_bwd_workspace(5, 0, 64) == 0
    assert L.kt_embedding_bwd_workspace(256, 100, 64) == 0
    small, large = L.kt_embedding_bwd_workspace(257, 100, 64), L.kt_embedding_bwd_workspace(1 << 30, 1 << 30, 1 << 24)
    assert 2 * 257 * 4 <= small < 65536
    # the four lists of 2^30 numbers, the counts of 512 stretches, two partial sums for each of 512 pieces
    assert large == 4 * (4 << 30) + 512 * 4 * 256 + 512 * 2 * (4 << 24)


def test_embedding_binding_refuses():
    f = torch.zeros(4, 8)
    i = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="current GPU|is on|needed"):
        kt.kt_embedding_fwd(i, f, f)
    with pytest.raises(ValueError, match="current GPU|is on|needed"):
        kt.kt_embedding_bwd(i, f, f)

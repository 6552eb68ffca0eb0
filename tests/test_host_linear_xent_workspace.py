"""The workspace of the cross entropy's gradients against what kt_ops.h says is in it, over the sizes that the call takes."""
import pytest

from paper_2505_10183_amd import ops
from test_host_ops import BF16, F32


def up(n, to):
    return (n + to - 1) // to * to


def parts_of(dt, tokens, vocab, width):
    """Bytes: dz, the copies of x and of w, one set of sums for dx and for a piece's dw, the lists and f32's sums of exponentials; and whether f32 may be in parts."""
    parts = dt == F32 and tokens >= 256 and width >= 128
    size = 6 if parts else 4 if dt == F32 else 2
    rows = min(max((1 << 27) // max(tokens, 1), 256), up(vocab, 256))
    wide = up(width, 64)
    dz = tokens * rows * size
    copies = tokens * wide * size + max((512 if parts else 128) << 20, 256 * wide * size)
    sums = 4 * (up(width, 256) * up(tokens, 256) + up(width, 16) * max(tokens, rows))
    lists = 32 * tokens + 4096 + (tokens * (rows // 16 + 1) * 4 + ops._library().kt_embedding_bwd_workspace(tokens, vocab, width) if dt == F32 else 0)
    return dz, copies, sums, lists


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("tokens", [1, 5, 33, 128, 1000, 16384, 1 << 19, (1 << 19) + 1, 1 << 20, 1 << 22, 1 << 24])
def test_gradients_workspace(tokens, dt):
    f = ops._library().kt_linear_xent_bwd_workspace
    for vocab in (1, 300, 4099, 50304, 1 << 20, 1 << 24):
        for width in (1, 72, 768, 1001, 2048):
            need = f(dt, tokens, vocab, width)
            dz, copies, sums, lists = parts_of(dt, tokens, vocab, width)
            # a product that fills the chip is not cut: more than one set of sums where tokens or the piece are few
            sets = 64 if tokens < 1 << 19 else 2
            # what is cut off to multiples of 256 bytes, for each of the workspace's parts
            assert 0 < need <= dz + copies + sets * sums + lists + 16 * 256, (vocab, width)
            # dz and the copies of x are in it whatever the rest is
            assert need >= min(dz // (3 if dt == F32 else 1), tokens * min(256, vocab) * (4 if dt == F32 else 2)) + tokens * width * (4 if dt == F32 else 2)


def test_dz_is_bounded_by_its_elements_or_by_256_a_token():
    """8 192 tokens more make no difference to dz up to 2^19 of them, and 256 elements each from there on."""
    f = ops._library().kt_linear_xent_bwd_workspace
    width = 64
    for tokens in (1 << 15, 1 << 17, 1 << 19):
        assert f(BF16, tokens, 50304, width) <= 2 * (1 << 27) + (128 << 20) + tokens * (width * 2 + 32) + 4 * 3 * 256 * tokens + (64 << 20)
    more = f(BF16, 1 << 21, 50304, width) - f(BF16, 1 << 20, 50304, width)
    assert (1 << 20) * 256 * 2 <= more <= (1 << 20) * (256 * 2 + width * 2 + 4 * 256 + 32)

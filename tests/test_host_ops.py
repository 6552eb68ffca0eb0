"""What the operators refuse, before any GPU is touched: the C calls get addresses that nothing reads, the binding gets tensors
that are not on a GPU."""
import ctypes
import math

import pytest
import torch

import paper_2505_10183_amd as kt
from paper_2505_10183_amd import ops

EINVAL, EALIGN, EUNSUPPORTED = 1, 2, 5
F32, BF16 = 0, 1
M = 1 << 20                        # each argument has a MiB of addresses of its own


def at(i):
    return (i + 1) * M


def call(name, args, status, word, **changes):
    """The call with some arguments changed is refused with this status and a message that says why."""
    L = ops._library()
    a = dict(args, **changes)
    got = getattr(L, name)(*a.values())
    text = L.kt_last_error().decode()
    assert got == status, (name, changes, got, text)
    assert name in text and word in text, (changes, text)


LN_FWD = dict(dt=F32, pdt=F32, rows=8, cols=64, x=at(0), ldx=64, gamma=at(1), beta=at(2), eps=1e-5, y=at(3), ldy=64, mean=at(4),
              rstd=at(5), y8=at(6), e8=at(7), stream=0)
LN_BWD = dict(dt=F32, pdt=F32, rows=8, cols=64, dy=at(0), lddy=64, x=at(1), ldx=64, x8=0, e8=0, gamma=at(2), mean=at(3), rstd=at(4),
              dx=at(5), lddx=64, dgamma=at(6), dbeta=at(7), ws=at(8), ws_bytes=M, stream=0)
SAVE = dict(dt=F32, rows=8, cols=64, x=at(0), ldx=64, q=at(1), e=at(2), stream=0)
RESTORE = dict(dt=F32, rows=8, cols=64, q=at(1), e=at(2), y=at(0), ldy=64, stream=0)


@pytest.mark.parametrize("changes,status,word", [
    (dict(dt=2), EINVAL, "type"), (dict(pdt=-1), EINVAL, "type"),
    (dict(rows=-1), EINVAL, "rows"), (dict(cols=0), EINVAL, "cols"), (dict(ldx=63), EINVAL, "ld"), (dict(ldy=63), EINVAL, "ld"),
    (dict(rows=1 << 60), EINVAL, "rows"), (dict(ldx=1 << 62), EINVAL, "ld"),
    (dict(cols=16385, ldx=16385, ldy=16385), EUNSUPPORTED, "columns"),
    (dict(eps=-1.0), EINVAL, "eps"), (dict(eps=math.nan), EINVAL, "eps"), (dict(eps=math.inf), EINVAL, "eps"),
    (dict(x=0), EINVAL, "NULL"), (dict(gamma=0), EINVAL, "NULL"), (dict(y=0), EINVAL, "NULL"),
    (dict(mean=0), EINVAL, "together"), (dict(rstd=0), EINVAL, "together"), (dict(y8=0), EINVAL, "together"), (dict(e8=0), EINVAL, "together"),
    (dict(x=at(0) + 2), EALIGN, "x"), (dict(y=at(3) + 1), EALIGN, "y"), (dict(gamma=at(1) + 2), EALIGN, "gamma"),
    (dict(beta=at(2) + 1), EALIGN, "beta"), (dict(mean=at(4) + 2), EALIGN, "mean"), (dict(rstd=at(5) + 1), EALIGN, "rstd"),
    (dict(y8=at(6) + 8), EALIGN, "y8"),
    (dict(y=at(0) + 4), EINVAL, "overlaps"), (dict(y=at(0), ldy=65), EINVAL, "overlaps"), (dict(mean=at(5)), EINVAL, "overlaps"),
    (dict(rstd=at(0) + 4 * 511), EINVAL, "overlaps"), (dict(y8=at(3)), EINVAL, "overlaps"), (dict(e8=at(1)), EINVAL, "overlaps"),
    (dict(y=at(2) - 4 * 511), EINVAL, "overlaps"),
])
def test_layernorm_fwd_refuses(changes, status, word):
    call("kt_layernorm_fwd", LN_FWD, status, word, **changes)


@pytest.mark.parametrize("changes,status,word", [
    (dict(dt=2), EINVAL, "type"), (dict(pdt=2), EINVAL, "type"),
    (dict(rows=-1), EINVAL, "rows"), (dict(cols=0), EINVAL, "cols"), (dict(lddy=63), EINVAL, "ld"), (dict(ldx=63), EINVAL, "ld"),
    (dict(lddx=63), EINVAL, "ld"), (dict(cols=16385, lddy=16385, ldx=16385, lddx=16385), EUNSUPPORTED, "columns"),
    (dict(dy=0), EINVAL, "NULL"), (dict(gamma=0), EINVAL, "NULL"), (dict(mean=0), EINVAL, "NULL"), (dict(rstd=0), EINVAL, "NULL"),
    (dict(dx=0), EINVAL, "NULL"), (dict(dgamma=0), EINVAL, "NULL"), (dict(dgamma=0, rows=0), EINVAL, "NULL"),
    (dict(x=0), EINVAL, "either"), (dict(x8=at(9), e8=at(10)), EINVAL, "either"), (dict(x=0, x8=at(9)), EINVAL, "either"),
    (dict(x=0, e8=at(9)), EINVAL, "either"),
    (dict(ws=0), EINVAL, "workspace"), (dict(ws_bytes=511), EINVAL, "workspace"),
    (dict(ws=at(8) + 4), EALIGN, "ws"), (dict(dy=at(0) + 2), EALIGN, "dy"), (dict(x=at(1) + 2), EALIGN, "x"), (dict(dx=at(5) + 2), EALIGN, "dx"),
    (dict(dgamma=at(6) + 2), EALIGN, "dgamma"), (dict(dbeta=at(7) + 2), EALIGN, "dbeta"), (dict(gamma=at(2) + 2), EALIGN, "gamma"),
    (dict(mean=at(3) + 2), EALIGN, "mean"), (dict(rstd=at(4) + 2), EALIGN, "rstd"), (dict(x=0, x8=at(9) + 8, e8=at(10)), EALIGN, "x8"),
    (dict(dx=at(0) + 4), EINVAL, "overlaps"), (dict(dx=at(1) + 4), EINVAL, "overlaps"), (dict(dgamma=at(2)), EINVAL, "overlaps"),
    (dict(dbeta=at(6) + 4 * 63), EINVAL, "overlaps"), (dict(ws=at(5)), EINVAL, "overlaps"), (dict(dgamma=at(0)), EINVAL, "overlaps"),
    (dict(dx=at(3)), EINVAL, "overlaps"), (dict(x=0, x8=at(5), e8=at(10)), EINVAL, "overlaps"), (dict(x=0, x8=at(9), e8=at(5)), EINVAL, "overlaps"),
])
def test_layernorm_bwd_refuses(changes, status, word):
    call("kt_layernorm_bwd", LN_BWD, status, word, **changes)


@pytest.mark.parametrize("name,args,wide", [("kt_act8_save", SAVE, "x"), ("kt_act8_restore", RESTORE, "y")])
def test_act8_refuses(name, args, wide):
    ld = "ld" + wide
    for changes, status, word in [
            (dict(dt=3), EINVAL, "type"), (dict(rows=-1), EINVAL, "rows"), (dict(cols=0), EINVAL, "cols"), ({ld: 63}, EINVAL, "ld"),
            ({"cols": (1 << 30) + 1, ld: 1 << 31}, EUNSUPPORTED, "columns"),
            ({wide: 0}, EINVAL, "NULL"), (dict(q=0), EINVAL, "NULL"), (dict(e=0), EINVAL, "NULL"),
            ({wide: at(0) + 2}, EALIGN, wide), (dict(q=at(1) + 8), EALIGN, "q"),
            (dict(q=at(0)), EINVAL, "overlaps"), (dict(e=at(0) + 3), EINVAL, "overlaps")]:
        call(name, args, status, word, **changes)
    if name == "kt_act8_save":
        call(name, args, EINVAL, "overlaps", e=at(1) + 511)


WEIGHT_GRAD = dict(dt=BF16, gdt=BF16, tokens=4096, out=64, inn=64, dy=at(0), lddy=64, q=at(1), e=at(2), dw=at(3), lddw=64, ws=at(4),
                   ws_bytes=M, stream=0)


@pytest.mark.parametrize("changes,status,word", [
    (dict(dt=2), EINVAL, "type"), (dict(gdt=2), EINVAL, "type"), (dict(tokens=-1), EINVAL, "tokens"), (dict(out=0), EINVAL, "out"),
    (dict(inn=0), EINVAL, "in"), (dict(lddy=63), EINVAL, "ld"), (dict(lddw=63), EINVAL, "ld"),
    (dict(tokens=(1 << 40) + 1), EUNSUPPORTED, "tokens"), (dict(out=(1 << 24) + 1, lddy=1 << 25), EUNSUPPORTED, "2^24"),
    (dict(inn=(1 << 24) + 1, lddw=1 << 25), EUNSUPPORTED, "2^24"),
    (dict(dy=0), EINVAL, "NULL"), (dict(q=0), EINVAL, "NULL"), (dict(e=0), EINVAL, "NULL"), (dict(dw=0), EINVAL, "NULL"),
    (dict(dw=0, tokens=0), EINVAL, "NULL"), (dict(ws=0), EINVAL, "workspace"), (dict(ws_bytes=1), EINVAL, "workspace"),
    (dict(dy=at(0) + 1), EALIGN, "dy"), (dict(q=at(1) + 8), EALIGN, "q"), (dict(dw=at(3) + 1), EALIGN, "dw"), (dict(ws=at(4) + 8), EALIGN, "ws"),
    (dict(dw=at(0) + 2 * 64 * 100), EINVAL, "overlaps"), (dict(dw=at(1)), EINVAL, "overlaps"), (dict(dw=at(2)), EINVAL, "overlaps"),
    (dict(ws=at(3)), EINVAL, "overlaps"), (dict(ws=at(1)), EINVAL, "overlaps"),
])
def test_weight_grad_refuses(changes, status, word):
    call("kt_act8_weight_grad", WEIGHT_GRAD, status, word, **changes)


def attention(name, status, word, tensors=(), **changes):
    """kt_attention_fwd or _bwd refused; sizes changed by name, tensors by (name, data or None, batch, token, head)."""
    L = ops._library()
    a = dict(dt=BF16, batch=2, nq=16, nk=16, heads=4, kv_heads=2, dim=64, scale=0.125, causal=1, k_lens=at(20))
    a.update({k: v for k, v in changes.items() if k in a})
    names = ["q", "k", "v", "o"] if name == "kt_attention_fwd" else ["d_o", "q", "k", "v", "o", "dq", "dk", "dv"]
    h = {n: ops._Heads(at(i), 16 * 4 * 64, 4 * 64, 64) for i, n in enumerate(names)}
    for n, *f in tensors:
        h[n] = None if f[0] is None else ops._Heads(*f)
    more = dict(lse=at(10), ws=at(11), ws_bytes=M)
    more.update({k: v for k, v in changes.items() if k in more})
    sizes = ops._Attention(*a.values())
    if name == "kt_attention_fwd":
        got = L.kt_attention_fwd(sizes, *h.values(), more["lse"], 0)
    else:
        got = L.kt_attention_bwd(sizes, *(h[n] for n in names[:5]), more["lse"], *(h[n] for n in names[5:]), more["ws"], more["ws_bytes"], 0)
    text = L.kt_last_error().decode()
    assert got == status and name in text and word in text, (got, changes, tensors, text)


@pytest.mark.parametrize("name", ["kt_attention_fwd", "kt_attention_bwd"])
def test_attention_refuses(name):
    I = EINVAL
    s = (16 * 4 * 64, 4 * 64, 64)
    for changes, status, word in [
            (dict(dt=2), I, "type"), (dict(batch=-1), I, "negative"), (dict(nq=-1), I, "negative"), (dict(nk=-1), I, "negative"),
            (dict(heads=0), I, "heads"), (dict(kv_heads=0), I, "heads"), (dict(dim=0), I, "dim"), (dict(kv_heads=3), I, "divide"),
            (dict(scale=0.0), I, "scale"), (dict(scale=-1.0), I, "scale"), (dict(scale=math.nan), I, "scale"), (dict(scale=math.inf), I, "scale"),
            (dict(dim=129), EUNSUPPORTED, "dim"), (dict(nk=(1 << 30) + 1), EUNSUPPORTED, "2^30"), (dict(nq=(1 << 30) + 1), EUNSUPPORTED, "2^30"),
            (dict(heads=1 << 17, kv_heads=1), EUNSUPPORTED, "heads"), (dict(batch=1 << 30), EUNSUPPORTED, "workgroups"),
            (dict(k_lens=at(20) + 2), EALIGN, "k_lens"), (dict(lse=at(10) + 2), EALIGN, "lse")]:
        attention(name, status, word, **changes)
    for n in ["q", "k", "v", "o"] + ([] if name == "kt_attention_fwd" else ["d_o", "dq", "dk", "dv"]):
        attention(name, I, "NULL " + n, [(n, None)])
        attention(name, I, "NULL " + n, [(n, 0, *s)])
        attention(name, EALIGN, n, [(n, at(15) + 1, *s)])
        attention(name, I, "strides of " + n, [(n, at(15), -1, s[1], s[2])])
        attention(name, I, "strides of " + n, [(n, at(15), s[0], (1 << 40) + 1, s[2])])
    for n in ["o"] if name == "kt_attention_fwd" else ["dq", "dk", "dv"]:
        attention(name, I, "share", [(n, at(15), 0, s[1], s[2])])
        attention(name, I, "share", [(n, at(15), s[0], s[1], 0)])
        attention(name, I, "share", [(n, at(15), s[0], s[1], 63)])
        attention(name, I, "share", [(n, at(15), s[0], 127, 64)])
        attention(name, I, "overlaps", [(n, at(1), *s)])
        attention(name, I, "overlaps", [(n, at(1) + 2 * (16 * 4 * 64 + 5), *s)])
        attention(name, I, n + " overlaps k_lens", [(n, at(20), *s)])
    if name == "kt_attention_fwd":
        attention(name, I, "lse overlaps q", lse=at(0))
    else:
        attention(name, I, "NULL lse", lse=0)
        attention(name, I, "workspace", ws=0)
        attention(name, I, "workspace", ws_bytes=2 * 4 * 16 * 4 - 1)
        attention(name, EALIGN, "ws", ws=at(11) + 4)
        attention(name, I, "ws overlaps", ws=at(2))
        attention(name, I, "dq overlaps lse", [("dq", at(10), *s)])


def test_attention_windows_of_one_buffer():
    """dq, dk and dv side by side in a token, in [batch, 3, heads, tokens, dim] or in one allocation after another pass; a window that
    reaches into its neighbour is refused.  (Those that pass are refused for their workspace only.)"""
    name, row = "kt_attention_bwd", (4 + 2 + 2) * 64
    def token(n, start, by=0):
        return (n, at(30) + 2 * (64 * start + by), 16 * row, row, 64)
    three = [token("dq", 0), token("dk", 4), token("dv", 6)]
    attention(name, EINVAL, "workspace", three, ws=0)
    attention(name, EINVAL, "overlaps", [token("dq", 0, 1)] + three[1:])
    attention(name, EINVAL, "overlaps", three[:2] + [token("dv", 5)])
    attention(name, EINVAL, "overlaps", three[:2] + [token("dv", 6, 1)])
    size = 16 * 64
    def plane(n, start, by=0):
        return (n, at(30) + 2 * (size * start + by), 8 * size, 64, size)
    three = [plane("dq", 0), plane("dk", 4), plane("dv", 6)]
    attention(name, EINVAL, "workspace", three, ws=0)
    attention(name, EINVAL, "overlaps", three[:1] + [plane("dk", 4, -1)] + three[2:])


def test_attention_does_nothing_for_no_sequences():
    L = ops._library()
    none = ops._Heads(0, 0, 0, 0)
    a = ops._Attention(BF16, 0, 16, 16, 4, 2, 64, 0.125, 0, 0)
    assert L.kt_attention_fwd(a, none, none, none, none, 0, 0) == 0
    assert L.kt_attention_bwd(a, none, none, none, none, none, 0, none, none, none, 0, 0, 0) == 0
    assert L.kt_attention_bwd_workspace(a) == 0


def test_weight_grad_workspace():
    for args in [(torch.float32, -1, 4, 4), (torch.float32, 4, 0, 4), (torch.bfloat16, 4, 4, 0), (torch.float32, 1, 64, 64)]:
        assert kt.kt_act8_weight_grad_workspace(*args) == 0
    n = kt.kt_act8_weight_grad_workspace(torch.bfloat16, 4096, 64, 65)
    assert n % (64 * 68 * 4) == 0 and n > 0


def test_columns_of_one_buffer_may_lie_side_by_side():
    """Equal distances between rows: x in columns 0..63, dx in 64..127 of a buffer 128 wide.  One column too far is refused (the
    others are refused for their NULL dgamma only, so nothing is launched)."""
    wide = dict(LN_FWD, ldx=128, ldy=128, y8=0, e8=0)
    call("kt_layernorm_fwd", wide, EINVAL, "y overlaps x", y=at(0) + 4 * 63)
    call("kt_layernorm_fwd", wide, EINVAL, "y overlaps x", y=at(0) + 4 * (128 - 63))
    call("kt_layernorm_fwd", wide, EINVAL, "rstd overlaps mean", y=at(0) + 4 * 64, mean=at(5))       # y passed its check
    call("kt_layernorm_fwd", wide, EINVAL, "rstd overlaps mean", y=at(0) - 4 * 64, mean=at(5))


def test_nothing_to_do_touches_no_gpu():
    L = ops._library()
    assert L.kt_layernorm_fwd(*dict(LN_FWD, rows=0).values()) == 0
    assert L.kt_act8_save(*dict(SAVE, rows=0, x=0, q=0, e=0).values()) == 0
    assert L.kt_act8_restore(*dict(RESTORE, rows=0, y=0, q=0, e=0).values()) == 0


def test_layernorm_workspace():
    for rows, cols in [(-1, 64), (8, 0), (8, 16385), (0, 64)]:
        assert kt.kt_layernorm_bwd_workspace(rows, cols) == 0
    for rows in (1, 15, 16, 17, 8191, 8192, 1 << 40):
        for cols in (1, 63, 64, 65, 16384):
            n = kt.kt_layernorm_bwd_workspace(rows, cols)
            assert n % (2 * 64 * 4) == 0 and 2 * 4 * cols <= n <= 2 * 4 * 512 * (cols + 63)


def test_act8_shapes():
    assert kt.kt_act8_shapes(5, 1) == ((5, 32), (5, 1))
    assert kt.kt_act8_shapes(5, 32) == ((5, 32), (5, 1))
    assert kt.kt_act8_shapes(0, 33) == ((0, 64), (0, 2))


def test_the_binding_refuses_tensors_that_are_not_on_the_gpu():
    x, g, v = torch.zeros(4, 64), torch.zeros(64), torch.zeros(4)
    q, e = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8)
    h = torch.zeros(1, 4, 1, 64)
    for f in (lambda: kt.kt_layernorm_fwd(x, g, g, 1e-5, x, v, v),
              lambda: kt.kt_layernorm_bwd(x, x, g, v, v, x, g, g),
              lambda: kt.kt_act8_save(x, q, e),
              lambda: kt.kt_act8_restore(q, e, x),
              lambda: kt.kt_act8_weight_grad(x, q, e, x),
              lambda: kt.kt_attention_fwd(h, h, h, h),
              lambda: kt.kt_attention_bwd(h, h, h, h, h, v, h, h, h)):
        if torch.cuda.is_available():
            with pytest.raises(ValueError, match="current GPU"):
                f()
        else:
            with pytest.raises((ValueError, RuntimeError, AssertionError)):
                f()


def test_attention_refuses_what_hip_cannot_launch():
    """2^24 workgroups of 256 lanes are 2^32 lanes.  One less passes this check: those calls are refused for a NULL tensor only."""
    word, n = "workgroups", 1 << 24
    for name in ("kt_attention_fwd", "kt_attention_bwd"):
        for sizes in (dict(batch=n // 16, heads=16, kv_heads=16, nq=1, nk=1), dict(batch=n // 16, heads=16, kv_heads=1, nq=128, nk=1),
                      dict(batch=n // 32, heads=16, kv_heads=16, nq=129, nk=1), dict(batch=1 << 30, heads=1 << 16, kv_heads=1, nq=1 << 30, nk=1)):
            attention(name, EUNSUPPORTED, word, **sizes)
        for sizes in (dict(batch=n - 1, heads=1, kv_heads=1, nq=128, nk=128), dict(batch=n // 4 - 1, heads=4, kv_heads=4, nq=1, nk=1),
                      dict(batch=1 << 30, heads=1, kv_heads=1, nq=0, nk=0)):
            attention(name, EINVAL, "NULL v", [("v", None)], **sizes)
    keys = dict(batch=1 << 10, heads=16, kv_heads=16, nq=1, nk=(1 << 17) + 1)
    attention("kt_attention_bwd", EUNSUPPORTED, word, **keys)
    attention("kt_attention_fwd", EINVAL, "NULL v", [("v", None)], **keys)


def test_sizes_whose_checkpoint_cannot_be_addressed_are_refused():
    """One column takes 32 bytes of a checkpoint: 2^58 rows are 2^63 bytes of q.  Each address here is far from the others."""
    rows = 1 << 58
    far = dict(rows=rows, cols=1, ldx=1, x=at(0), q=1 << 62, e=1 << 61)
    call("kt_act8_save", dict(SAVE, **far), EINVAL, "rows")
    call("kt_act8_restore", dict(dt=F32, rows=rows, cols=1, q=1 << 62, e=1 << 61, y=at(0), ldy=1, stream=0), EINVAL, "rows")
    call("kt_layernorm_fwd", dict(LN_FWD, rows=rows, cols=1, ldx=1, ldy=1, y=1 << 60, mean=0, rstd=0, y8=1 << 62, e8=1 << 61), EINVAL, "rows")
    # 2^40 tokens of one column of dy, the checkpoint 2^24 columns wide: 2^64 bytes
    call("kt_act8_weight_grad", dict(WEIGHT_GRAD, tokens=1 << 40, out=1, inn=1 << 24, lddy=1, lddw=1 << 24, q=1 << 50, e=1 << 45, dw=1 << 44,
                                     ws=1 << 56, ws_bytes=1 << 50), EINVAL, "tokens")

"""Attention forward and backward against the formulas in 64 bits.

Tolerances, from the roundings of a step (u = 2^-24, HALF half a step of the type; sums of absolute values, so worst cases):
  scores: eS = (D + 10) u scale sum|q k| + 4 u |S|, products of bf16 being exact
  o: p (2 max eS + (N + 20) u + half a step of p in bf16) over |v|, + HALF |o|
  lse: max eS + (N + 8) u + 8 u (|lse| + max|S|)
  p from lse: eP = eS + 8 u (|S| + |lse|), relative
  dS: P (eP |dP - delta| + (D + 10) u (sum|dO v| + sum|dO o|)) + half a step of dS in bf16
  dq, dk: scale (eDS + (N + 20) u |dS|) over |k|, |q|, + HALF;  dv: P (eP + half a step of P + (M + 20) u) over |dO|, + HALF
with N keys and M queries of the heads that share a key head.  A probability under TINY = 2^-126, the smallest normal number of
binary32, may be 0: TINY for p, TINY (|dP - delta| + 1) for dS."""
import math

import pytest
import torch

import paper_2505_10183_amd as kt
from ops_util import DEV, DT, HALF, U, gen, normal, within

pytestmark = pytest.mark.gpu

# batch, queries, keys, heads, key heads, dim
SIZES = [(1, 1, 1, 1, 1, 1), (2, 1, 77, 3, 1, 40), (1, 5, 3, 2, 2, 64), (2, 64, 64, 2, 2, 64), (1, 197, 197, 3, 3, 64), (2, 130, 257, 4, 2, 128),
         (1, 300, 100, 2, 1, 80), (3, 33, 65, 4, 4, 128), (1, 129, 513, 2, 2, 7), (2, 128, 128, 1, 1, 96), (1, 700, 700, 2, 2, 128),
         (1, 257, 31, 6, 2, 65), (1, 31, 2500, 2, 2, 64), (1, 1100, 40, 2, 1, 128)]
TINY = 2.0 ** -126
LAYOUTS = ["together", "contiguous", "heads_first", "odd"]


def tensors(size, dtype, layout, seed, scale=1.0):
    """q, k, v and empty dq, dk, dv in the same layout."""
    B, nq, nk, H, Hk, D = size
    g = gen(seed)
    sets = []
    for values in (True, False):
        make = (lambda *s: normal(g, *s, dtype=dtype, scale=scale)) if values else (lambda *s: torch.full(s, 55.0, dtype=dtype, device=DEV))
        if layout == "together" and nq == nk:
            t = make(B, nq, H + 2 * Hk, D).split([H, Hk, Hk], dim=2)
        elif layout == "heads_first":
            t = [make(B, h, n, D).transpose(1, 2) for n, h in ((nq, H), (nk, Hk), (nk, Hk))]
        elif layout == "odd":            # one element off a 16-byte boundary, gaps between heads and tokens
            t = [make(B * n * (h * (D + 3) + 5) + 1)[1:].as_strided((B, n, h, D), (n * (h * (D + 3) + 5), h * (D + 3) + 5, D + 3, 1), 1)
                 for n, h in ((nq, H), (nk, Hk), (nk, Hk))]
        else:
            t = [make(B, n, h, D) for n, h in ((nq, H), (nk, Hk), (nk, Hk))]
        sets.append(list(t))
    return sets


def seen(size, causal, lens):
    B, nq, nk = size[:3]
    j, i = torch.arange(nk, device=DEV), torch.arange(nq, device=DEV)[:, None]
    m = torch.ones(B, nq, nk, dtype=torch.bool, device=DEV)
    if causal:
        m &= j <= i + nk - nq
    if lens is not None:
        m &= j < lens.clamp(0, nk)[:, None, None]
    return m


def heads64(x, times=1):
    return x.double().transpose(1, 2).repeat_interleave(times, 1).contiguous()


def reference(q, k, v, size, causal, lens, scale, do=None, o=None, lse=None):
    """Forward: (o, tolerance, lse, tolerance); with do, o and lse, backward: ((dq, tol), (dk, tol), (dv, tol))."""
    B, nq, nk, H, Hk, D = size
    t, dtype = H // Hk, q.dtype
    step = HALF[dtype] if dtype == torch.bfloat16 else 0.0
    m = seen(size, causal, lens)[:, None]
    clean = torch.ones(B, nk, 1, 1, dtype=torch.bool, device=DEV) if lens is None else (torch.arange(nk, device=DEV) < lens[:, None])[:, :, None, None]
    k, v = (torch.where(clean, x.double(), 0.0) for x in (k, v))
    Q, Kk, V = heads64(q), heads64(k, t), heads64(v, t)
    KT = Kk.transpose(2, 3).contiguous()
    S = Q @ KT * scale
    eS = (D + 10) * U * scale * (Q.abs() @ KT.abs()) + 4 * U * S.abs()
    eS, absS = (torch.where(m, x, 0.0) for x in (eS, S.abs()))
    if do is None:
        S = torch.where(m, S, -math.inf)
        L = torch.logsumexp(S, 3)
        P = torch.where(m, (S - L[..., None]).exp(), 0.0)
        O = P @ V
        worst = eS.amax(3) if nk else torch.zeros_like(L)
        tol = P @ V.abs() * (2 * worst[..., None] + (nk + 20) * U + step) + HALF[dtype] * O.abs()
        tl = worst + (nk + 8) * U + 8 * U * (L.abs().nan_to_num(posinf=0.0) + (absS.amax(3) if nk else 0))
        back = lambda x: x.transpose(1, 2)  # noqa: E731
        return back(O), back(tol), L, tl
    L = lse.double()
    P = torch.where(m, (S - L[..., None]).exp(), 0.0)
    eP = eS + 8 * U * (absS + L.abs().nan_to_num(posinf=0.0)[..., None])
    dO, Oh = heads64(do), heads64(o)
    VT = V.transpose(2, 3).contiguous()
    dP, delta = dO @ VT, (dO * Oh).sum(3, keepdim=True)
    dS = P * (dP - delta)
    eDS = P * (eP * (dP - delta).abs() + (D + 10) * U * (dO.abs() @ VT.abs() + (dO * Oh).abs().sum(3, keepdim=True))) + step * dS.abs()
    eDS = torch.where(m, eDS + TINY * ((dP - delta).abs() + 1), 0.0)
    T = lambda x: x.transpose(2, 3).contiguous()  # noqa: E731
    dq, eq = scale * (dS @ Kk), scale * ((eDS + (nk + 20) * U * dS.abs()) @ Kk.abs())
    n = nq * t + 20
    dk, ek = scale * (T(dS) @ Q), scale * (T(eDS + n * U * dS.abs()) @ Q.abs())
    dv, ev = T(P) @ dO, T(P * (eP + step + n * U) + torch.where(m, TINY, 0.0)) @ dO.abs()
    shared = lambda x: x.view(B, Hk, t, nk, D).sum(2)  # noqa: E731
    out = []
    for x, e in ((dq, eq), (shared(dk), shared(ek)), (shared(dv), shared(ev))):
        out.append((x.transpose(1, 2), (e + HALF[dtype] * x.abs()).transpose(1, 2)))
    return out


def lens_of(size, kind):
    B, nk = size[0], size[2]
    if kind == "none":
        return None
    n = torch.arange(B, device=DEV) * 37 % (nk + 1)             # 0 first: a sequence without keys
    if kind == "outside":
        n[0] = -5
        n[-1] = nk + 9 if B > 1 else -5
    return n.to(torch.int32)


def check(size, dtype, layout, causal, lens, scale=None, spread=1.0, seed=0):
    B, nq, nk, H, Hk, D = size
    dt = DT[dtype]
    (q, k, v), (dq, dk, dv) = tensors(size, dt, layout, seed + nq + nk, spread)
    if lens is not None:                                        # what lies past a sequence's keys is not read
        for b in range(B):
            k[b, max(0, int(lens[b])):] = float("nan")
            v[b, max(0, int(lens[b])):] = float("inf")
    c = D ** -0.5 if scale is None else scale
    g = gen(seed + 5)
    o = torch.full((B, nq, H, D), 55.0, device=DEV).to(dt)
    lse = torch.full((B, H, nq), 55.0, device=DEV)
    kt.kt_attention_fwd(q, k, v, o, lse, causal=causal, scale=scale, k_lens=lens)
    O, to, L, tl = reference(q, k, v, size, causal, lens, c)
    within(o, O, to, "o")
    within(lse, L, tl, "lse")
    nothing = ~seen(size, causal, lens).any(2)                   # queries without a key
    assert not o[nothing].any() and bool((lse.transpose(1, 2)[nothing] == -math.inf).all())
    do = normal(g, B, nq, H, D, dtype=dt)
    kt.kt_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, causal=causal, scale=scale, k_lens=lens)
    for name, got, (want, tol) in zip(("dq", "dk", "dv"), (dq, dk, dv), reference(q, k, v, size, causal, lens, c, do, o, lse)):
        within(got, want, tol, name)
    unseen = ~seen(size, causal, lens).any(1)                    # keys that no query sees
    assert not dq[nothing].any() and not dk[unseen].any() and not dv[unseen].any()
    return q, k, v, o, lse, do, dq, dk, dv


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_sizes(size, dtype, causal):
    check(size, dtype, LAYOUTS[sum(size) % 4], causal, None)


@pytest.mark.parametrize("kind", ["some", "outside"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 33, 65, 4, 4, 128), (5, 130, 130, 4, 2, 64), (2, 200, 70, 2, 1, 96), (4, 1, 300, 2, 2, 64)])
def test_lengths(size, dtype, causal, kind):
    check(size, dtype, "contiguous", causal, lens_of(size, kind))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [20, 64, 128])
def test_layouts(dim, dtype, layout):
    size = (2, 150, 150, 4, 2, dim)
    q, k, v, o, lse, do, dq, dk, dv = check(size, dtype, layout, True, None, seed=3)
    if layout == "odd":             # the gaps between heads and tokens keep their values
        for t in (dq, dk, dv):
            B, n, h, D = t.shape
            whole = t.as_strided((t.numel() // (h * D) * (h * (D + 3) + 5) + 1,), (1,), 0)
            gaps = torch.ones_like(whole, dtype=torch.bool)
            gaps[1:].as_strided(t.shape, t.stride(), 1).fill_(False)
            assert bool((whole[gaps] == 55).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_from_zero(dtype):
    """Scores of some hundred: the running maximum moves, most probabilities vanish."""
    check((1, 200, 300, 2, 2, 64), dtype, "contiguous", False, None, scale=1.0, spread=4.0)
    check((1, 300, 300, 2, 2, 128), dtype, "contiguous", True, None, scale=0.7, spread=3.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_growing_and_falling_scores(dtype):
    """The largest score of each query is in the first tile, the last tile or in between; the reference of the softmax must
    follow."""
    size = (1, 96, 400, 1, 1, 64)
    dt = DT[dtype]
    for order in (1, -1):
        (q, k, v), _ = tensors(size, dt, "contiguous", 4)
        ramp = order * torch.linspace(-3, 3, 400, device=DEV)
        q[..., 0] = 8.0
        k[0, :, 0, 0] = (ramp * 4).to(dt)
        o, lse = torch.empty_like(q), torch.empty(1, 1, 96, device=DEV)
        kt.kt_attention_fwd(q, k, v, o, lse)
        O, to, L, tl = reference(q, k, v, size, False, None, 0.125)
        within(o, O, to, "o")
        within(lse, L, tl, "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_broadcast_keys(dtype):
    """k and v of one head and one sequence, read by all (strides 0); their gradients are whole tensors."""
    dt = DT[dtype]
    g = gen(9)
    B, n, H, D = 2, 100, 4, 64
    q, k1, v1 = normal(g, B, n, H, D, dtype=dt), normal(g, 1, n, 1, D, dtype=dt), normal(g, 1, n, 1, D, dtype=dt)
    out = []
    for k, v in ((k1.expand(B, n, H, D), v1.expand(B, n, H, D)), (k1.repeat(B, 1, H, 1), v1.repeat(B, 1, H, 1))):
        o, lse = torch.empty_like(q), torch.empty(B, H, n, device=DEV)
        dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
        kt.kt_attention_fwd(q, k, v, o, lse)
        kt.kt_attention_bwd(q, q, k, v, o, lse, dq, dk, dv)
        out.append((o, lse, dq, dk, dv))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_gradient_by_differences():
    """The backward pass is the derivative of the forward pass; f32, values of order 1, Richardson's step.  A forward value
    carries up to 300 u of its size (the o tolerance: 2 eS of about 80 terms, N + 20), over h."""
    size = (2, 21, 37, 4, 2, 24)
    B, nq, nk, H, Hk, D = size
    (q, k, v), _ = tensors(size, torch.float32, "contiguous", 11)
    w = normal(gen(12), B, nq, H, D)
    lens = torch.tensor([37, 25], dtype=torch.int32, device=DEV)
    o, lse = torch.empty(B, nq, H, D, device=DEV), torch.empty(B, H, nq, device=DEV)

    def f(q, k, v):
        kt.kt_attention_fwd(q, k, v, o, lse, causal=True, k_lens=lens)
        return float((o.double() * w.double()).sum())

    f(q, k, v)
    size_of = float((o.double().abs() * w.double().abs()).sum())
    grads = [torch.empty_like(t) for t in (q, k, v)]
    kt.kt_attention_bwd(w, q, k, v, o, lse, *grads, causal=True, k_lens=lens)
    for which, grad in enumerate(grads):
        d = normal(gen(13 + which), *grad.shape)

        def slope(h):
            at = []
            for sign in (1, -1):
                moved = [q, k, v]
                moved[which] = moved[which] + sign * h * d
                at.append(f(*moved))
            return (at[0] - at[1]) / (2 * h)

        h = 2.0 ** -5
        got, want = (4 * slope(h / 2) - slope(h)) / 3, float((grad.double() * d.double()).sum())
        assert abs(got - want) <= (300 * U * 3 / h + 60 * h ** 4) * size_of, (which, got, want)


def test_nothing_to_attend_to():
    g = gen(1)
    q, o = normal(g, 2, 5, 2, 64), torch.full((2, 5, 2, 64), 3.0, device=DEV)
    none = torch.empty(2, 0, 2, 64, device=DEV)
    lse = torch.empty(2, 2, 5, device=DEV)
    kt.kt_attention_fwd(q, none, none, o, lse)
    assert not o.any() and bool((lse == -math.inf).all())
    dq = torch.full_like(q, 3.0)
    kt.kt_attention_bwd(q, q, none, none, o, lse, dq, torch.empty_like(none), torch.empty_like(none))
    assert not dq.any()
    dk, dv = torch.full_like(q, 3.0), torch.full_like(q, 3.0)
    kt.kt_attention_bwd(none, none, q, q, none, torch.empty(2, 2, 0, device=DEV), torch.empty_like(none), dk, dv)
    assert not dk.any() and not dv.any()
    kt.kt_attention_fwd(none, q, q, torch.empty_like(none))
    kt.kt_attention_fwd(q[:0], q[:0], q[:0], o[:0])


def test_the_same_bits_every_time_on_another_stream_and_in_a_graph():
    size = (2, 300, 300, 4, 2, 128)
    (q, k, v), (dq, dk, dv) = tensors(size, torch.bfloat16, "together", 21)
    do = normal(gen(22), 2, 300, 4, 128, dtype=torch.bfloat16)
    o, lse = torch.empty_like(do), torch.empty(2, 4, 300, device=DEV)
    out = (o, lse, dq, dk, dv)
    need = kt.kt_attention_bwd_workspace(q, k)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=DEV)

    def step(stream=None, workspace=None):
        kt.kt_attention_fwd(q, k, v, o, lse, causal=True, stream=stream)
        kt.kt_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, causal=True, workspace=workspace, stream=stream)

    step()
    want = [t.clone() for t in out]
    s = torch.cuda.Stream()
    for stream, workspace in ((None, ws[:need]), (s, None), (s.cuda_stream, None), (s, ws[:need])):
        for t in out:
            t.zero_()
        s.wait_stream(torch.cuda.current_stream())
        step(stream, workspace)
        s.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert bool((ws[need:] == 255).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3):
        q.copy_(normal(gen(seed), *q.shape))
        step()
        want = [t.clone() for t in out]
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("where", ["d_o", "o", "q"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_keys_past_the_length_have_no_gradient_whatever_a_query_holds(dtype, causal, bad, where):
    """Lengths inside a wavefront's 32 keys and a workgroup's 128: the keys past them get 0, and the other sequence the same bits."""
    dt = DT[dtype]
    g = gen(31)
    q, o, do = (normal(g, 2, 200, 2, 64, dtype=dt) for _ in range(3))
    k, v = (normal(g, 2, 200, 1, 64, dtype=dt) for _ in range(2))
    lens = torch.tensor([70, 130], dtype=torch.int32, device=DEV)
    lse = torch.full((2, 2, 200), 6.0, device=DEV)
    out = []
    for value in (None, bad):
        if value is not None:
            {"d_o": do, "o": o, "q": q}[where][0, 150, :, 3] = value
        dq, dk, dv = torch.full_like(q, 5.0), torch.full_like(k, 5.0), torch.full_like(k, 5.0)
        kt.kt_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, causal=causal, k_lens=lens)
        for b in range(2):
            assert not dk[b, int(lens[b]):].any() and not dv[b, int(lens[b]):].any(), (value, b)
        out.append([t[1].clone() for t in (dq, dk, dv)])
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("where", ["d_o", "o"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dk_of_keys_that_a_query_does_not_see(dtype, where):
    """A NaN in d_o or o of query 40 under a causal mask: dk of keys past 40 takes ds = 0 from it, also in its own tile."""
    dt = DT[dtype]
    g = gen(32)
    q, k, v, o, do = (normal(g, 1, 128, 1, 64, dtype=dt) for _ in range(5))
    lse = torch.full((1, 1, 128), 6.0, device=DEV)
    out = []
    for value in (1.0, math.nan):
        {"d_o": do, "o": o}[where][0, 40, 0, 3] = value
        dq, dk, dv = (torch.empty_like(q) for _ in range(3))
        kt.kt_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, causal=True)
        out.append(dk)
    assert torch.equal(out[0][:, 41:], out[1][:, 41:]) and out[1][:, :41].isnan().any()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_queries_without_keys_get_0_whatever_the_keys_hold(dim, dtype, bad):
    """100 queries on 70 keys under a causal mask: the first 30 see none, and share their tile with queries that see keys
    with a NaN or an infinity."""
    dt = DT[dtype]
    g = gen(33)
    q, do = (normal(g, 1, 100, 2, dim, dtype=dt) for _ in range(2))
    for where in ("k", "v"):
        k, v = (normal(g, 1, 70, 2, dim, dtype=dt) for _ in range(2))
        {"k": k, "v": v}[where][0, 0, :, 5] = bad
        o, lse = torch.full_like(q, 5.0), torch.full((1, 2, 100), 5.0, device=DEV)
        kt.kt_attention_fwd(q, k, v, o, lse, causal=True)
        assert not o[:, :30].any() and bool((lse[:, :, :30] == -math.inf).all()), where
        dq, dk, dv = torch.full_like(q, 5.0), torch.empty_like(k), torch.empty_like(k)
        kt.kt_attention_bwd(do, q, k, v, o, lse, dq, dk, dv, causal=True)
        assert not dq[:, :30].any(), where


@pytest.mark.parametrize("dim,gap", [(64, 0), (128, 0), (80, 3), (33, 0)])
@pytest.mark.parametrize("value", [0.1, 0.7, 0.9])
def test_long_sums_of_dk_and_dv_keep_their_digits(value, dim, gap):
    """16 heads of 4 096 queries share a key head: 65 536 terms.  With k = v = 0 and lse = 0 every p is 1, with one element of o at -1
    every ds is d_o's value c, so that dv = dk = 65536 c.  All partial sums have the terms' sign: each addition is off by u of the
    total at most, 512 in a piece, 128 of pieces, 8 for what else there is.  (One chain of 65 536 is 1e-4 off and more.)"""
    c = float(torch.tensor(value))
    B, nq, nk, H = 2, 4096, 40, 16
    wide = lambda n, h, v: torch.full((B, n, h, dim + gap), v, device=DEV)[..., :dim]  # noqa: E731
    q, o, do = wide(nq, H, 1.0), wide(nq, H, 0.0), wide(nq, H, c)
    o[..., 0] = -1.0
    k, v = wide(nk, 1, 0.0), wide(nk, 1, 0.0)
    dq, dk, dv = wide(nq, H, 5.0), wide(nk, 1, math.nan), wide(nk, 1, math.nan)
    lens = torch.tensor([nk, nk - 7], dtype=torch.int32, device=DEV)
    kt.kt_attention_bwd(do, q, k, v, o, torch.zeros(B, H, nq, device=DEV), dq, dk, dv, scale=1.0, k_lens=lens)
    want = torch.full((B, nk, 1, dim), c * nq * H, dtype=torch.float64, device=DEV)
    want[1, nk - 7:] = 0.0
    within(dk, want, (512 + 128 + 8) * U * want, "dk")
    within(dv, want, (512 + 128 + 8) * U * want, "dv")

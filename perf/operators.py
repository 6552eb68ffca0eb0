"""What the operators of a transformer block's training pass are timed on.

A case is one pass through one operator, as the backward or forward pass of a block makes it:

  layernorm_fwd  kt_layernorm_fwd; with `save`, the 8-bit checkpoint of the output is written beside it and
                 restored (what the next linear layer's backward pass does with it)
  layernorm_bwd  kt_layernorm_bwd: gradients of input, weight and bias; with `x8`, the input comes from its
                 8-bit checkpoint
  act8           kt_act8_save, then kt_act8_restore: one activation's way through its checkpoint
  weight_grad    kt_act8_weight_grad: the gradient of a linear layer's weight from the 8-bit input
  attention_fwd  kt_attention_fwd
  attention_bwd  kt_attention_bwd from the forward pass's output and log-sum-exp

Sizes: the ViT-B/16 of workloads.py (f32, width 768, 197 tokens an image), its 1.3B decoder (bf16, width 2048,
2048 positions, MLP 8192), and odd ones (width 1001, as the dense decoder of cases.py).  The number of heads is
the width over a head of 64 or 128.  Query, key and value are views of one product's output [B, N, heads, D].
"""
import math
import random

import torch

own = False

GROUP = 32          # neighbouring columns that share a scale in an 8-bit checkpoint
EPS = 1e-5


def listed():
    return [
        # one image of ViT-B/16: the smallest real call, latency alone
        {"name": "layernorm_fwd_one_image", "op": "layernorm_fwd", "rows": 197, "cols": 768, "dtype": "f32", "save": False},
        # the decoder's block input, 8 sequences: forward pass that leaves the next linear layer's checkpoint
        {"name": "layernorm_fwd_save_decoder", "op": "layernorm_fwd", "rows": 16384, "cols": 2048, "dtype": "bf16", "save": True},
        # ViT-B/16, 128 images: the backward pass with the reduction of the weight's gradient over 25 216 rows
        {"name": "layernorm_bwd_vit", "op": "layernorm_bwd", "rows": 25216, "cols": 768, "dtype": "f32", "x8": False},
        # an odd width, the input kept in 8 bits
        {"name": "layernorm_bwd_x8_odd", "op": "layernorm_bwd", "rows": 9001, "cols": 1001, "dtype": "bf16", "x8": True},
        # the decoder's widest activation (MLP, 8 sequences) through its checkpoint
        {"name": "act8_mlp_decoder", "op": "act8", "rows": 16384, "cols": 8192, "dtype": "bf16"},
        # an odd width in f32
        {"name": "act8_odd", "op": "act8", "rows": 2003, "cols": 1001, "dtype": "f32"},
        # one image of ViT-B/16 through its output projection
        {"name": "weight_grad_one_image", "op": "weight_grad", "tokens": 197, "out": 768, "in": 768, "dtype": "f32", "grad": "f32"},
        # the decoder's MLP output layer, 8 sequences
        {"name": "weight_grad_decoder", "op": "weight_grad", "tokens": 16384, "out": 2048, "in": 8192, "dtype": "bf16", "grad": "bf16"},
        # odd everything, gradient kept in f32 for the optimizer
        {"name": "weight_grad_odd", "op": "weight_grad", "tokens": 4099, "out": 1001, "in": 4004, "dtype": "bf16", "grad": "f32"},
        # ViT-B/16, 32 images: no mask, 197 keys, which fill no tile
        {"name": "attention_bwd_vit", "op": "attention_bwd", "batch": 32, "nq": 197, "nk": 197, "heads": 12, "kv_heads": 12,
         "dim": 64, "dtype": "f32", "causal": False, "lens": False},
        # the decoder's training shape: 8 causal sequences of 2048
        {"name": "attention_bwd_decoder", "op": "attention_bwd", "batch": 8, "nq": 2048, "nk": 2048, "heads": 16, "kv_heads": 16,
         "dim": 128, "dtype": "bf16", "causal": True, "lens": False},
        # long padded sequences with shared key heads, odd length
        {"name": "attention_fwd_long_shared", "op": "attention_fwd", "batch": 2, "nq": 8191, "nk": 8191, "heads": 16, "kv_heads": 4,
         "dim": 128, "dtype": "bf16", "causal": True, "lens": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["layernorm_fwd", "layernorm_bwd", "act8", "weight_grad", "attention_fwd", "attention_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("layernorm_fwd", "layernorm_bwd", "act8"):
        cols = rng.choice([768, 1001, 1024, 2048, 4096, 8192, _log(rng, 33, 10000)])
        rows = _log(rng, 1, max(2, min(40000, (1 << 25) // cols)))
        c = {"op": op, "rows": rows, "cols": cols, "dtype": dtype}
        if op == "layernorm_fwd":
            c["save"] = dtype == "bf16" and rng.random() < 0.5
        if op == "layernorm_bwd":
            c["x8"] = rng.random() < 0.5
        return c
    if op == "weight_grad":
        out, inn = (rng.choice([768, 2048, 2304, 8192, _log(rng, 40, 8192)]) for _ in range(2))
        tokens = _log(rng, 1, min(16384, (1 << 37) // (out * inn)))
        return {"op": op, "tokens": tokens, "out": out, "in": inn, "dtype": dtype,
                "grad": "f32" if dtype == "f32" or rng.random() < 0.5 else "bf16"}
    dim = rng.choice([64, 64, 128, 128, 80, 96, 40])
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    heads = kv * rng.choice([1, 1, 1, 2, 4] if kv <= 4 else [1])
    nk = _log(rng, 1, 4096)
    nq = nk if rng.random() < 0.7 else _log(rng, 1, 4096)
    # the plain forms keep the scores of all heads: at most 2^28 of them
    batch = max(1, min(rng.choice([1, 2, 4, 8, 32]), (1 << 28) // (nq * nk * heads)))
    return {"op": op, "batch": batch, "nq": nq, "nk": nk, "heads": heads, "kv_heads": kv, "dim": dim, "dtype": dtype,
            "causal": rng.random() < 0.6, "lens": rng.random() < 0.3}


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _activation(gen, rows, cols, dtype):
    """Rows of a residual stream: every column with a spread of its own, a few of them ten times as wide, a mean per row."""
    wide = torch.rand(cols, generator=gen, device="cuda") * 1.5 + 0.25
    wide = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, wide * 10, wide)
    x = torch.randn(rows, cols, generator=gen, device="cuda") * wide
    x += torch.randn(rows, 1, generator=gen, device="cuda") * 0.3
    return x.to(dtype)


def _lens(gen, case):
    """Keys of each sequence: one of them full, one empty where there are more than two."""
    if not case["lens"]:
        return None
    n = torch.randint(1, case["nk"] + 1, (case["batch"],), generator=gen, device="cuda", dtype=torch.int32)
    n[0] = case["nk"]
    if case["batch"] > 2:
        n[1] = 0
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    op, dt = case["op"], _type(case["dtype"])
    empty = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    s = {"case": case}
    if op in ("layernorm_fwd", "layernorm_bwd", "act8"):
        rows, cols = case["rows"], case["cols"]
        ld = (cols + GROUP - 1) // GROUP * GROUP
        x = _activation(gen, rows, cols, dt)
        s.update(x=x, q=empty(rows, ld, dtype=torch.int8), e=empty(rows, ld // GROUP, dtype=torch.uint8))
        if op == "act8":
            s["y"] = empty(rows, cols)
            return s
        s["gamma"] = (1 + 0.2 * torch.randn(cols, generator=gen, device="cuda")).to(dt)
        s["beta"] = (0.1 * torch.randn(cols, generator=gen, device="cuda")).to(dt)
        if op == "layernorm_fwd":
            s.update(y=empty(rows, cols), y8=empty(rows, cols), mean=empty(rows, dtype=torch.float32),
                     rstd=empty(rows, dtype=torch.float32))
            return s
        s["dy"] = (torch.randn(rows, cols, generator=gen, device="cuda") * 0.05).to(dt)
        s["mean"], s["rstd"] = _moments(x.float())
        if case["x8"]:
            s["q"], s["e"] = _to8(x)
            del s["x"]
        s.update(dx=empty(rows, cols), dgamma=empty(cols), dbeta=empty(cols))
        return s
    if op == "weight_grad":
        s["q"], s["e"] = _to8(_activation(gen, case["tokens"], case["in"], dt))
        s["dy"] = (torch.randn(case["tokens"], case["out"], generator=gen, device="cuda") * 0.05).to(dt)
        s["dw"] = empty(case["out"], case["in"], dtype=_type(case["grad"]))
        return s
    B, nq, nk, H, Hk, D = (case[k] for k in ("batch", "nq", "nk", "heads", "kv_heads", "dim"))
    # the products that make query, key and value write them side by side
    if nq == nk:
        all3 = torch.randn(B, nq, H + 2 * Hk, D, generator=gen, device="cuda").to(dt)
        s["q"], s["k"], s["v"] = all3.split([H, Hk, Hk], dim=2)
    else:
        s["q"] = torch.randn(B, nq, H, D, generator=gen, device="cuda").to(dt)
        s["k"], s["v"] = torch.randn(B, nk, 2 * Hk, D, generator=gen, device="cuda").to(dt).split([Hk, Hk], dim=2)
    s["lens"] = _lens(gen, case)
    if op == "attention_fwd":
        s.update(o=empty(B, nq, H, D), lse=empty(B, H, nq, dtype=torch.float32))
        return s
    s["do"] = (torch.randn(B, nq, H, D, generator=gen, device="cuda") * 0.05).to(dt)
    s["o"], s["lse"] = _attention(s["q"], s["k"], s["v"], case["causal"], s["lens"])
    if nq == nk:
        s["dq"], s["dk"], s["dv"] = empty(B, nq, H + 2 * Hk, D).split([H, Hk, Hk], dim=2)
    else:
        s.update(dq=empty(B, nq, H, D), dk=empty(B, nk, Hk, D), dv=empty(B, nk, Hk, D))
    return s


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ---------------------------------

def _moments(x):
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, 1 / (var + EPS).sqrt()


def _to8(x):
    rows, cols = x.shape
    ld = (cols + GROUP - 1) // GROUP * GROUP
    g = torch.zeros(rows, ld, dtype=torch.float32, device=x.device)
    g[:, :cols] = x
    g = g.view(rows, ld // GROUP, GROUP)
    power = g.abs().amax(2).view(torch.int32) >> 23                       # biased exponent of the largest magnitude
    bad = power == 255
    e = torch.where(bad, 255, (power - 6).clamp(min=1))
    up = torch.where(bad, 0, (254 - e) << 23).view(torch.float32)         # 2^(127 - e), exact
    q = (g * up[:, :, None]).round().clamp(-127, 127)
    q = torch.where(bad[:, :, None], 0, q)
    return q.to(torch.int8).view(rows, ld), e.to(torch.uint8)


def _from8(q, e, cols):
    down = (e.to(torch.int32) << 23).view(torch.float32)                  # 2^(e - 127); 255: inf, and 0 * inf = nan
    x = q.view(q.shape[0], -1, GROUP).float() * down[:, :, None]
    return x.view(q.shape[0], -1)[:, :cols]


def _seen(nq, nk, causal, lens, device):
    """[B or 1, 1, nq, nk] truth values: the keys that a query sees (causal: the last query sees the last key)."""
    j = torch.arange(nk, device=device)
    seen = torch.ones(1, 1, nq, nk, dtype=torch.bool, device=device)
    if causal:
        seen = seen & (j <= torch.arange(nq, device=device)[:, None] + (nk - nq))
    if lens is not None:
        seen = seen & (j < lens[:, None, None, None])
    return seen


def _heads(x, times=1):
    """[B, N, H, D] -> [B, H * times, N, D] in 32 bits."""
    return x.float().transpose(1, 2).repeat_interleave(times, dim=1).contiguous()


def _attention(q, k, v, causal, lens):
    times = q.shape[2] // k.shape[2]
    qh, kh, vh = _heads(q), _heads(k, times), _heads(v, times)
    s = torch.matmul(qh, kh.transpose(2, 3).contiguous()) / math.sqrt(q.shape[3])
    s = torch.where(_seen(q.shape[1], k.shape[1], causal, lens, q.device), s, -math.inf)
    top = s.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0, top)
    p = (s - top).exp()
    total = p.sum(3, keepdim=True)
    lse = (top + total.log()).squeeze(3)
    o = torch.matmul(p, vh) / torch.where(total == 0, 1, total)
    return o.transpose(1, 2).to(q.dtype).contiguous(), lse


def _attention_bwd(do, q, k, v, o, lse, causal, lens):
    Hk, times, scale = k.shape[2], q.shape[2] // k.shape[2], 1 / math.sqrt(q.shape[3])
    qh, kh, vh, doh = _heads(q), _heads(k, times), _heads(v, times), _heads(do)
    s = torch.matmul(qh, kh.transpose(2, 3).contiguous()) * scale
    p = torch.where(_seen(q.shape[1], k.shape[1], causal, lens, q.device), (s - lse[:, :, :, None]).exp(), 0)
    delta = (doh * _heads(o)).sum(3, keepdim=True)
    ds = p * (torch.matmul(doh, vh.transpose(2, 3).contiguous()) - delta) * scale
    dq = torch.matmul(ds, kh)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), qh)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), doh)
    shared = lambda x: x.view(x.shape[0], Hk, times, x.shape[2], x.shape[3]).sum(2)  # noqa: E731
    return tuple(x.transpose(1, 2).to(q.dtype) for x in (dq, shared(dk), shared(dv)))


def _plain(s):
    case = s["case"]
    op, dt = case["op"], _type(case["dtype"])
    if op == "act8":
        return {"y": _from8(*_to8(s["x"]), case["cols"]).to(dt)}
    if op == "layernorm_fwd":
        x = s["x"].float()
        mean, rstd = _moments(x)
        y = ((x - mean[:, None]) * rstd[:, None] * s["gamma"].float() + s["beta"].float()).to(dt)
        out = {"y": y, "mean": mean, "rstd": rstd}
        if case["save"]:
            out["y8"] = _from8(*_to8(y), case["cols"]).to(dt)
        return out
    if op == "layernorm_bwd":
        x = _from8(s["q"], s["e"], case["cols"]) if case["x8"] else s["x"].float()
        dy = s["dy"].float()
        xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
        t = dy * s["gamma"].float()
        dx = (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
        return {"dx": dx.to(dt), "dgamma": (dy * xh).sum(0).to(dt), "dbeta": dy.sum(0).to(dt)}
    if op == "weight_grad":
        return {"dw": torch.matmul(s["dy"].float().t(), _from8(s["q"], s["e"], case["in"])).to(_type(case["grad"]))}
    if op == "attention_fwd":
        o, lse = _attention(s["q"], s["k"], s["v"], case["causal"], s["lens"])
        return {"o": o, "lse": lse}
    dq, dk, dv = _attention_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], case["causal"], s["lens"])
    return {"dq": dq, "dk": dk, "dv": dv}


def run(state):
    if not own:
        return _plain(state)
    import paper_2505_10183_amd as kt
    s, case = state, state["case"]
    op = case["op"]
    if op == "act8":
        kt.kt_act8_save(s["x"], s["q"], s["e"])
        kt.kt_act8_restore(s["q"], s["e"], s["y"])
        return {"y": s["y"]}
    if op == "layernorm_fwd":
        out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        if case["save"]:
            kt.kt_layernorm_fwd(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"], y8=(s["q"], s["e"]))
            kt.kt_act8_restore(s["q"], s["e"], s["y8"])
            out["y8"] = s["y8"]
        else:
            kt.kt_layernorm_fwd(s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
        return out
    if op == "layernorm_bwd":
        x = (s["q"], s["e"]) if case["x8"] else s["x"]
        kt.kt_layernorm_bwd(s["dy"], x, s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if op == "weight_grad":
        kt.kt_act8_weight_grad(s["dy"], s["q"], s["e"], s["dw"])
        return {"dw": s["dw"]}
    if op == "attention_fwd":
        kt.kt_attention_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], causal=case["causal"], k_lens=s["lens"])
        return {"o": s["o"], "lse": s["lse"]}
    kt.kt_attention_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["dq"], s["dk"], s["dv"],
                        causal=case["causal"], k_lens=s["lens"])
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    op, es = case["op"], 4 if case["dtype"] == "f32" else 2
    if op in ("layernorm_fwd", "layernorm_bwd", "act8"):
        rows, cols = case["rows"], case["cols"]
        n, n8 = rows * cols, rows * (cols + (cols + GROUP - 1) // GROUP)
        if op == "act8":
            return {"bytes": 2 * n * es + 2 * n8, "flops": 6 * n}
        if op == "layernorm_fwd":
            more = 2 * n8 + n * es if case["save"] else 0
            return {"bytes": 2 * n * es + 2 * cols * es + 8 * rows + more, "flops": 8 * n}
        return {"bytes": 2 * n * es + (n8 if case["x8"] else n * es) + 3 * cols * es + 8 * rows, "flops": 14 * n}
    if op == "weight_grad":
        T, O, I = case["tokens"], case["out"], case["in"]
        return {"bytes": T * O * es + T * (I + (I + GROUP - 1) // GROUP) + O * I * (4 if case["grad"] == "f32" else 2),
                "flops": 2 * T * O * I}
    B, nq, nk, H, Hk, D = (case[k] for k in ("batch", "nq", "nk", "heads", "kv_heads", "dim"))
    pairs = nq * nk
    if case["causal"]:
        last = min(nq, nk)                      # the last `last` queries see nk - last + 1 .. nk keys
        pairs = last * (2 * nk - last + 1) // 2
    if case["lens"]:
        pairs = pairs * 3 // 4                  # one sequence in full, the others of any length
    qs, ks = B * nq * H * D * es, B * nk * Hk * D * es
    if op == "attention_fwd":
        return {"bytes": 2 * qs + 2 * ks + 4 * B * nq * H, "flops": 4 * B * H * D * pairs}
    return {"bytes": 4 * qs + 4 * ks + 4 * B * nq * H, "flops": 10 * B * H * D * pairs}


# ---- the operators' definitions in 64 bits, apart from the plain forms -------------------------------------------

def _two_to(n):
    """2^n in 64 bits, from its bits: a power function may be off in the last place, which moves ties."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def _saved64(x):
    """What the 8-bit checkpoint of x [rows, cols] stands for, in 64 bits."""
    rows, cols = x.shape
    short = -cols % GROUP
    g = torch.cat([x.double(), x.new_zeros(rows, short, dtype=torch.float64)], 1).unflatten(1, (-1, GROUP))
    power = torch.frexp(g.abs().max(2).values).exponent - 1               # 2^power <= largest < 2^(power + 1)
    power = torch.where(g.abs().max(2).values == 0, -1000, power)
    step = _two_to((power - 6).clamp(min=-126))[:, :, None]
    return (torch.round(g / step).clamp(-127, 127) * step).flatten(1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "act8":
        return {"y": _saved64(s["x"])}
    if op == "layernorm_fwd":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = torch.rsqrt(var + EPS)
        y = torch.addcmul(s["beta"].double(), (x - mean.unsqueeze(1)) * rstd.unsqueeze(1), s["gamma"].double())
        out = {"y": y, "mean": mean, "rstd": rstd}
        if case["save"]:
            out["y8"] = _saved64(y.to(_type(case["dtype"])))
        return out
    if op == "layernorm_bwd":
        if case["x8"]:
            x = (s["q"].double() * _two_to(s["e"].to(torch.int32) - 127).repeat_interleave(GROUP, 1))[:, :case["cols"]]
        else:
            x = s["x"].double()
        mean, rstd, dy = s["mean"].double().unsqueeze(1), s["rstd"].double().unsqueeze(1), s["dy"].double()
        xh, up = (x - mean) * rstd, dy * s["gamma"].double()
        n = case["cols"]
        dx = rstd / n * (n * up - up.sum(1, True) - xh * (up * xh).sum(1, True))
        return {"dx": dx, "dgamma": xh.mul_(dy).sum(0), "dbeta": dy.sum(0)}
    if op == "weight_grad":
        x = (s["q"].double() * _two_to(s["e"].to(torch.int32) - 127).repeat_interleave(GROUP, 1))[:, :case["in"]]
        return {"dw": s["dy"].double().t().contiguous() @ x}
    B, nq, nk, H, Hk, D = (case[k] for k in ("batch", "nq", "nk", "heads", "kv_heads", "dim"))
    times = H // Hk
    f64 = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    if op == "attention_fwd":
        out = {"o": f64(B, nq, H, D), "lse": f64(B, H, nq)}
    else:
        out = {"dq": f64(B, nq, H, D), "dk": f64(B, nk, Hk, D), "dv": f64(B, nk, Hk, D)}
    hidden = f64(nq, nk)
    if case["causal"]:
        hidden = torch.triu(torch.full_like(hidden, -math.inf), diagonal=nk - nq + 1)
    for b in range(B):
        n = nk if s["lens"] is None else int(s["lens"][b])
        for h in range(H):
            q, k, v = s["q"][b, :, h].double(), s["k"][b, :n, h // times].double(), s["v"][b, :n, h // times].double()
            score = q @ k.t() / math.sqrt(D) + hidden[:, :n]
            lse = torch.logsumexp(score, 1)
            p = torch.where(score == -math.inf, 0.0, torch.exp(score - lse.unsqueeze(1)))
            if op == "attention_fwd":
                out["o"][b, :, h], out["lse"][b, h] = p @ v, lse
                continue
            # the true gradient: the row sums come from the probabilities, not from a rounded output
            do = s["do"][b, :, h].double()
            dp = do @ v.t()
            ds = p * (dp - (p * dp).sum(1, True)) / math.sqrt(D)
            out["dq"][b, :, h] = ds @ k
            out["dk"][b, :n, h // times] += ds.t() @ q
            out["dv"][b, :n, h // times] += p.t() @ do
    return out

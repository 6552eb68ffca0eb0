"""What the operators at the two ends of a language model are timed on: the embedding lookup and the loss over the vocabulary.

A case is one pass through one operator, as a training step or a scoring call makes it:

  embedding_fwd  kt_embedding_fwd: rows of a table by token, scaled
  embedding_bwd  kt_embedding_bwd: the table's whole gradient from that of the rows
  xent_fwd       kt_linear_xent_fwd: cross entropy of x w^T over the vocabulary, and the log-sum-exp
  xent_bwd       kt_linear_xent_bwd: gradients of x and w from that of the losses
  tied_bwd       kt_linear_xent_bwd, then kt_embedding_bwd with accumulate: the gradient of a table that is both ends' weight

Sizes: the 1.3B decoder of workloads.py (bf16, 50304 tokens, width 2048, 2048 positions, 8 sequences), its ViT-B/16 (f32, width
768, 1000 classes, 197 tokens an image), the odd decoder of cases.py (5003 tokens, width 1001), and generic ones.  Tokens
follow the frequencies of text: the n-th most frequent about 1 / n as often as the first.
"""
import math
import random

import numpy as np
import torch

own = False


def listed():
    return [
        # the token that a decoder has just made, on its way into the next step: latency alone
        {"name": "embedding_fwd_one_token", "op": "embedding_fwd", "tokens": 1, "vocab": 50304, "width": 2048, "dtype": "bf16",
         "table": "bf16", "ids": 64, "none": 0.0, "hot": 0.0},
        # the decoder's batch of 8 sequences
        {"name": "embedding_fwd_decoder", "op": "embedding_fwd", "tokens": 16384, "vocab": 50304, "width": 2048, "dtype": "bf16",
         "table": "bf16", "ids": 64, "none": 0.0, "hot": 0.0},
        # odd everything, a tenth of the positions are padding without a token
        {"name": "embedding_fwd_odd", "op": "embedding_fwd", "tokens": 9001, "vocab": 5003, "width": 1001, "dtype": "f32",
         "table": "f32", "ids": 32, "none": 0.1, "hot": 0.0},
        # one short sequence with a small table: the smallest gradient, latency alone
        {"name": "embedding_bwd_one_sequence", "op": "embedding_bwd", "tokens": 197, "vocab": 1000, "width": 768, "dtype": "f32",
         "table": "f32", "ids": 32, "none": 0.0, "hot": 0.0},
        # the decoder's batch of 8 sequences
        {"name": "embedding_bwd_decoder", "op": "embedding_bwd", "tokens": 16384, "vocab": 50304, "width": 2048, "dtype": "bf16",
         "table": "bf16", "ids": 64, "none": 0.0, "hot": 0.0},
        # a long batch half of which is one filling token: one row of the table gets 32 768 of the sums
        {"name": "embedding_bwd_filled", "op": "embedding_bwd", "tokens": 65536, "vocab": 50304, "width": 2048, "dtype": "bf16",
         "table": "bf16", "ids": 64, "none": 0.0, "hot": 0.5},
        # the log-probability of one token, as scoring asks for it: the weight is read once for one row
        {"name": "xent_fwd_one_token", "op": "xent_fwd", "tokens": 1, "vocab": 50304, "width": 2048, "dtype": "bf16", "ids": 64,
         "none": 0.0},
        # the decoder's batch of 8 sequences
        {"name": "xent_fwd_decoder", "op": "xent_fwd", "tokens": 16384, "vocab": 50304, "width": 2048, "dtype": "bf16", "ids": 64,
         "none": 0.0},
        # the classes of ViT-B/16, its global batch of 1024 images
        {"name": "xent_fwd_vit", "op": "xent_fwd", "tokens": 1024, "vocab": 1000, "width": 768, "dtype": "f32", "ids": 32, "none": 0.0},
        # the decoder's batch of 8 sequences, the largest
        {"name": "xent_bwd_decoder", "op": "xent_bwd", "tokens": 16384, "vocab": 50304, "width": 2048, "dtype": "bf16", "ids": 64,
         "none": 0.0},
        # f32, the decoder's vocabulary on the narrower width, two sequences of 2048
        {"name": "xent_bwd_f32", "op": "xent_bwd", "tokens": 4096, "vocab": 50304, "width": 768, "dtype": "f32", "ids": 64, "none": 0.0},
        # odd everything, one weight for both ends, two fifths of the positions have no target (prompts and padding)
        {"name": "tied_bwd_odd", "op": "tied_bwd", "tokens": 4099, "vocab": 5003, "width": 1001, "dtype": "bf16", "ids": 64, "none": 0.4},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choice(["embedding_fwd", "embedding_bwd", "xent_fwd", "xent_bwd", "tied_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    vocab = rng.choice([1000, 5003, 50304, _log(rng, 10, 131072)])
    width = rng.choice([768, 1001, 1024, 2048, 4096, _log(rng, 33, 8192)])
    ids, none = rng.choice([32, 64]), rng.choice([0.0, 0.0, 0.1, 0.5])
    if op in ("embedding_fwd", "embedding_bwd"):
        return {"op": op, "tokens": _log(rng, 1, max(2, min(65536, (1 << 27) // width))), "vocab": vocab, "width": width, "dtype": dtype,
                "table": dtype if rng.random() < 0.7 else "f32", "ids": ids, "none": none, "hot": rng.choice([0.0, 0.0, 0.2])}
    most = (1 << 40 if dtype == "bf16" else 1 << 37) // (vocab * width)
    return {"op": op, "tokens": _log(rng, 1, max(2, min(16384, most))), "vocab": vocab, "width": width, "dtype": dtype, "ids": ids, "none": none}


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _tokens(gen, n, vocab, hot=0.0):
    """Tokens of text: the n-th most frequent about 1 / n as often as the first; a share `hot` of them all one token."""
    t = (torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * math.log(vocab + 1)).exp().long() - 1
    t = torch.randperm(vocab, generator=gen, device="cuda")[t.clamp(0, vocab - 1)]
    return torch.where(torch.rand(n, generator=gen, device="cuda") < hot, vocab // 3, t)


def _without(gen, t, share, mark):
    """A share of the positions has no token: spread ones, and half as many again at the end."""
    n = t.numel()
    out = torch.rand(n, generator=gen, device="cuda") < share / 2
    out |= torch.arange(n, device="cuda") >= n - int(n * share / 2)
    return torch.where(out, mark, t)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 29)
    op, dt, n, V, D = case["op"], _type(case["dtype"]), case["tokens"], case["vocab"], case["width"]
    it = torch.int32 if case["ids"] == 32 else torch.int64
    empty = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    s = {"case": case}
    if op in ("embedding_fwd", "embedding_bwd"):
        wt = _type(case["table"])
        s["ids"] = _without(gen, _tokens(gen, n, V, case["hot"]), case["none"], -1).to(it)
        if op == "embedding_fwd":
            s.update(w=(normal(V, D) * D ** -0.5).to(wt), y=empty(n, D))
        else:
            s.update(dy=(normal(n, D) * 0.05).to(dt), dw=empty(V, D, dtype=wt))
        return s
    # a model that has learned something: its last activation leans to the next token's row
    target = _tokens(gen, n, V)
    w = (normal(V, D) * D ** -0.5).to(dt)
    s["w"], s["x"] = w, (normal(n, D) + 8 * w[target].float()).to(dt)
    s["targets"] = _without(gen, target, case["none"], -100).to(it)
    if op == "xent_fwd":
        s.update(loss=empty(n, dtype=torch.float32), lse=empty(n, dtype=torch.float32))
        return s
    live = s["targets"] >= 0
    s["dloss"] = torch.where(live, 1.0 / live.sum().clamp(min=1), 0.0).float()     # of the mean over the positions with a target
    s["lse"] = _xent(s["x"], w, s["targets"])[1]
    s.update(dx=empty(n, D), dw=empty(V, D))
    if op == "tied_bwd":
        s["ids"] = _tokens(gen, n, V).to(it)
        s["dy"] = (normal(n, D) * (0.05 / n)).to(dt)
    return s


def _scale(case):
    return math.sqrt(case["width"])


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ---------------------------------

def _lookup(ids, w, scale):
    there = (ids >= 0)[:, None]
    return torch.where(there, w[ids.clamp(min=0).long()].float() * scale, 0)


def _collect(ids, dy, into, scale):
    there = ids >= 0
    rows = torch.where(there[:, None], dy.float() * scale, 0)
    return into.index_add_(0, ids.clamp(min=0).long(), rows)


def _logits(x, w):
    return torch.matmul(x.float(), w.float().t())


def _xent(x, w, targets):
    z = _logits(x, w)
    top = z.amax(1, keepdim=True)
    lse = (top + (z - top).exp().sum(1, keepdim=True).log()).squeeze(1)
    there = targets >= 0
    at = z.gather(1, targets.clamp(min=0).long()[:, None]).squeeze(1)
    return torch.where(there, lse - at, 0), torch.where(there, lse, 0)


def _xent_bwd(dloss, x, w, targets, lse):
    there = targets >= 0
    dz = (_logits(x, w) - lse[:, None]).exp()
    n = torch.arange(dz.shape[0], device=dz.device)
    dz[n, targets.clamp(min=0).long()] -= 1
    dz *= torch.where(there, dloss, 0)[:, None]
    return torch.matmul(dz, w.float()), torch.matmul(dz.t(), x.float())


def _plain(s):
    case = s["case"]
    op, dt = case["op"], _type(case["dtype"])
    if op == "embedding_fwd":
        return {"y": _lookup(s["ids"], s["w"], _scale(case)).to(dt)}
    if op == "embedding_bwd":
        zero = torch.zeros(case["vocab"], case["width"], device="cuda")
        return {"dw": _collect(s["ids"], s["dy"], zero, _scale(case)).to(_type(case["table"]))}
    if op == "xent_fwd":
        loss, lse = _xent(s["x"], s["w"], s["targets"])
        return {"loss": loss, "lse": lse}
    dx, dw = _xent_bwd(s["dloss"], s["x"], s["w"], s["targets"], s["lse"])
    if op == "tied_bwd":
        dw = _collect(s["ids"], s["dy"], dw, _scale(case))
    return {"dx": dx.to(dt), "dw": dw.to(dt)}


def run(state):
    if not own:
        return _plain(state)
    import paper_2505_10183_amd as kt
    s, case = state, state["case"]
    op = case["op"]
    if op == "embedding_fwd":
        kt.kt_embedding_fwd(s["ids"], s["w"], s["y"], scale=_scale(case))
        return {"y": s["y"]}
    if op == "embedding_bwd":
        kt.kt_embedding_bwd(s["ids"], s["dy"], s["dw"], scale=_scale(case))
        return {"dw": s["dw"]}
    if op == "xent_fwd":
        kt.kt_linear_xent_fwd(s["x"], s["w"], s["targets"], s["loss"], s["lse"])
        return {"loss": s["loss"], "lse": s["lse"]}
    kt.kt_linear_xent_bwd(s["dloss"], s["x"], s["w"], s["targets"], s["lse"], s["dx"], s["dw"])
    if op == "tied_bwd":
        kt.kt_embedding_bwd(s["ids"], s["dy"], s["dw"], scale=_scale(case), accumulate=True)
    return {"dx": s["dx"], "dw": s["dw"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def _distinct(case):
    """Rows of the table that the tokens name: the expected number."""
    n, V = case["tokens"], case["vocab"]
    live = n * (1 - case["none"]) if case["op"].startswith("embedding") else n
    p = np.diff(np.log(np.arange(1, V + 2))) / math.log(V + 1)
    return float((-np.expm1(live * (1 - case.get("hot", 0.0)) * np.log1p(-np.minimum(p, 0.999999)))).sum())


def work(case):
    op, n, V, D = case["op"], case["tokens"], case["vocab"], case["width"]
    es, ib = (4 if case["dtype"] == "f32" else 2), case["ids"] // 8
    if op in ("embedding_fwd", "embedding_bwd"):
        ws = 4 if case["table"] == "f32" else 2
        live = n * (1 - case["none"])
        if op == "embedding_fwd":
            return {"bytes": int(n * (ib + D * es) + _distinct(case) * D * ws), "flops": int(live * D)}
        return {"bytes": int(n * ib + live * D * es + V * D * ws), "flops": int(2 * live * D)}
    live = n - n * case["none"] * 0.95          # what _without leaves
    if op == "xent_fwd":
        return {"bytes": int((live + V) * D * es + n * (ib + 8)), "flops": int(2 * live * V * D)}
    more = n * (ib + D * es) + 2 * _distinct(case) * D * es if op == "tied_bwd" else 0
    return {"bytes": int((live + n + 2 * V) * D * es + n * (ib + 8) + more), "flops": int(6 * live * V * D)}


# ---- the operators' definitions in 64 bits, apart from the plain forms -------------------------------------------

def _table_grad64(ids, dy, vocab, scale):
    """The sum over each token's positions, by differences of the running sum over the positions in order of their tokens."""
    keep = torch.nonzero(ids >= 0).squeeze(1)
    order = keep[torch.argsort(ids[keep], stable=True)]
    bound = torch.searchsorted(ids[order].long().contiguous(), torch.arange(vocab + 1, device="cuda"))
    out = torch.empty(vocab, dy.shape[1], dtype=torch.float64, device="cuda")
    for c in range(0, dy.shape[1], 512):
        run_ = torch.cumsum(dy[order, c:c + 512].double(), 0)
        run_ = torch.cat([run_.new_zeros(1, run_.shape[1]), run_])
        out[:, c:c + 512] = (run_[bound[1:]] - run_[bound[:-1]]) * scale
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op, n, V, D = case["op"], case["tokens"], case["vocab"], case["width"]
    if op == "embedding_fwd":
        table = torch.cat([s["w"].double(), torch.zeros(1, D, dtype=torch.float64, device="cuda")])
        return {"y": table.index_select(0, torch.where(s["ids"] < 0, V, s["ids"]).long()) * _scale(case)}
    if op == "embedding_bwd":
        return {"dw": _table_grad64(s["ids"], s["dy"], V, _scale(case))}
    f64 = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    w = s["w"].double()
    wt = w.t().contiguous()
    classes = torch.arange(V, device="cuda")
    out = {"loss": f64(n), "lse": f64(n)} if op == "xent_fwd" else {"dx": f64(n, D), "dw": f64(V, D)}
    for a in range(0, n, 2048):
        x, t = s["x"][a:a + 2048].double(), s["targets"][a:a + 2048]
        z = x @ wt
        lse = torch.logsumexp(z, 1)
        hit = classes == t[:, None]             # no column where there is no target
        if op == "xent_fwd":
            out["loss"][a:a + 2048] = ((lse[:, None] - z) * hit).sum(1)
            out["lse"][a:a + 2048] = lse * hit.any(1)
            continue
        dz = (torch.softmax(z, 1) - hit.double()) * (s["dloss"][a:a + 2048].double() * hit.any(1))[:, None]
        out["dx"][a:a + 2048] = dz @ w
        out["dw"] += dz.t().contiguous() @ x
    if op == "tied_bwd":
        out["dw"] += _table_grad64(s["ids"], s["dy"], V, _scale(case))
    return out

"""What is measured of the vocabulary ends of a language model on a prompt-sharing tree: the embedding lookup with its
gradient, and the softmax cross entropy over the vocabulary with its gradient, which never holds the logits.

    embed_fwd    out[t] = s E[id_t]                                     (a row of zeros for id_t < 0)
    embed_bwd    dE[v]  = s sum of d_out[t] over id_t = v                (every row of dE is written)
    score        lse_t  = log sum_v exp(c h_t . W_v),   loss_t = lse_t - c h_t . W_{y_t}
    train        the same, and for the gradient a_t of the sum of the losses with respect to loss_t
                 G_tv = a_t c (exp(c h_t . W_v - lse_t) - [v = y_t]),   dH = G W,   dW = G^T H
                 (y_t < 0: the row is not scored; loss_t = lse_t = 0, dH_t = 0, nothing of it in dW)

Sizes: hidden 3584 (28 heads of 128) with a vocabulary of 152064 is the geometry of the default benchmark; its tree has
24576 tokens, 16384 of them responses, the rows that are scored.  Hidden 256 with a vocabulary of 503 is that of the
model-level test.  The other sizes are generic, ragged ones among them.
"""
import math

import torch

own = False

BF16, F32, F64, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int64
DTYPES = {"bf16": BF16, "f32": F32}


def listed():
    return [
        # one micro-batch of an update step: 8192 response tokens of the default geometry, loss and both gradients
        {"name": "train-8192", "op": "train", "tokens": 8192, "vocab": 152064, "hidden": 3584, "masked": 0.0},
        # a padded batch of a mid-sized model, ragged in every size; a quarter of the rows is not scored
        {"name": "train-2183-masked", "op": "train", "tokens": 2183, "vocab": 32003, "hidden": 1032, "masked": 0.25},
        # a short tail of an update step under the full vocabulary: few rows, the gradient of W is the large part
        {"name": "train-77", "op": "train", "tokens": 77, "vocab": 152064, "hidden": 3584, "masked": 0.0},
        # the model-level test's sizes: latency
        {"name": "train-129-small", "op": "train", "tokens": 129, "vocab": 503, "hidden": 256, "masked": 0.1},
        # log-probabilities of all responses of the default tree under a frozen policy (no gradient)
        {"name": "score-16384", "op": "score", "tokens": 16384, "vocab": 152064, "hidden": 3584, "masked": 0.0},
        # one answer of 300 tokens scored by a mid-sized model
        {"name": "score-300", "op": "score", "tokens": 300, "vocab": 50257, "hidden": 1024, "masked": 0.0},
        # the log-probability of a single sampled token
        {"name": "score-1", "op": "score", "tokens": 1, "vocab": 152064, "hidden": 3584, "masked": 0.0},
        # all tokens of the default tree embedded, bf16 table
        {"name": "embed-24576", "op": "embed_fwd", "tokens": 24576, "vocab": 152064, "hidden": 3584, "dtype": "bf16", "masked": 0.0},
        # one sampled token embedded
        {"name": "embed-1", "op": "embed_fwd", "tokens": 1, "vocab": 152064, "hidden": 3584, "dtype": "bf16", "masked": 0.0},
        # the gradient of that table from all tokens of the default tree
        {"name": "embed-grad-24576", "op": "embed_bwd", "tokens": 24576, "vocab": 152064, "hidden": 3584, "dtype": "bf16", "masked": 0.0},
        # many tokens over a middling table in 32 bits, padding among them: frequent ids own thousands of rows
        {"name": "embed-grad-131071", "op": "embed_bwd", "tokens": 131071, "vocab": 32003, "hidden": 1032, "dtype": "f32", "masked": 0.1},
        # the model-level test's table in 32 bits: latency
        {"name": "embed-grad-743-small", "op": "embed_bwd", "tokens": 743, "vocab": 503, "hidden": 256, "dtype": "f32", "masked": 0.0},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["train", "score", "embed_fwd", "embed_bwd"])
    case = {"op": op, "tokens": _log_uniform(rng, 1, {"train": 8192, "score": 16384, "embed_fwd": 24576, "embed_bwd": 24576}[op]),
            "vocab": _log_uniform(rng, 300, 152064), "hidden": 8 * _log_uniform(rng, 8, 448), "masked": rng.choice([0.0, 0.0, 0.1, 0.5])}
    if op.startswith("embed"):
        case["dtype"] = rng.choice(["bf16", "f32"])
    return case


def _scored(case):
    """How many rows are not masked: a fixed number, so that the work of a case does not hang on the seed."""
    return case["tokens"] - int(case["masked"] * case["tokens"])


def _ids(case, gen):
    """Token ids, frequent ones first (the k-th id is drawn about 1 / k as often), some masked by a negative id."""
    t, v = case["tokens"], case["vocab"]
    ids = torch.exp(torch.rand(t, generator=gen, device="cuda", dtype=F64) * math.log(v)).floor().to(I64).sub_(1).clamp_(0, v - 1)
    off = torch.randperm(t, generator=gen, device="cuda")[_scored(case):]
    ids[off] = -100
    return ids


def _randn(shape, gen, dtype=F32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t, v, k, op = case["tokens"], case["vocab"], case["hidden"], case["op"]
    ids = _ids(case, gen)
    s = {"case": case, "ids": ids}
    if op == "embed_fwd":
        s["table"] = _randn((v, k), gen, DTYPES[case["dtype"]])
        s["scale"] = math.sqrt(k)
    elif op == "embed_bwd":
        s["d_out"] = _randn((t, k), gen, DTYPES[case["dtype"]])
        s["scale"] = math.sqrt(k)
    else:
        # rows of W of about unit length; every hidden row leans towards its target by a push of its own, so that the
        # probability of the target goes from that of any token to near one, as it does over an answer's tokens
        w = (_randn((v, k), gen, BF16) * k ** -0.5)
        push = torch.rand((t, 1), generator=gen, device="cuda") * 16
        s["hidden"] = (_randn((t, k), gen) + push * w[ids.clamp(min=0)].float()).to(BF16)
        s["weight"], s["scale"] = w, 1.0
        if op == "train":
            s["d_loss"] = _randn((t,), gen)       # one advantage for each token
    if own:
        from paper_2609_33133_b200 import binding as B
        lm = B.LM(v, k, device=0, embed_scale=s["scale"] if op.startswith("embed") else 0.0)
        e = lambda shape, dt: torch.empty(shape, device="cuda", dtype=dt)
        s["lm"] = lm
        if op == "embed_fwd":
            s["out"] = e((t, k), s["table"].dtype)
        elif op == "embed_bwd":
            s["d_table"] = e((v, k), s["d_out"].dtype)
        else:
            s["loss"], s["lse"] = e((t,), F32), e((t,), F32)
            if op == "train":
                s["d_hidden"], s["d_weight"] = e((t, k), BF16), e((v, k), BF16)
        s["ws"] = torch.empty(lm.workspace_bytes(t), device="cuda", dtype=torch.uint8)
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    lm, op = s["lm"], s["case"]["op"]
    if op == "embed_fwd":
        lm.embed_fwd(s["table"], s["ids"], s["out"])
        return s["out"]
    if op == "embed_bwd":
        lm.embed_bwd(s["d_out"], s["ids"], s["d_table"], s["ws"])
        return s["d_table"]
    lm.loss_fwd(s["hidden"], s["weight"], s["ids"], s["loss"], s["lse"], s["ws"])
    if op == "score":
        return {"loss": s["loss"], "lse": s["lse"]}
    lm.loss_bwd(s["hidden"], s["weight"], s["ids"], s["lse"], s["d_loss"], s["d_hidden"], s["d_weight"], s["ws"])
    return {"loss": s["loss"], "lse": s["lse"], "d_hidden": s["d_hidden"], "d_weight": s["d_weight"]}


def _run_plain(s):
    ids, op, case = s["ids"], s["case"]["op"], s["case"]
    live = ids >= 0
    at = ids.clamp(min=0)
    if op == "embed_fwd":
        return torch.where(live[:, None], s["table"][at].float() * s["scale"], 0.0).to(s["table"].dtype)
    if op == "embed_bwd":
        d = torch.where(live[:, None], s["d_out"].float() * s["scale"], 0.0)
        return torch.zeros((case["vocab"], case["hidden"]), device="cuda", dtype=F32).index_add_(0, at, d).to(s["d_out"].dtype)
    h, w = s["hidden"].float(), s["weight"].float()
    x = h @ w.t() * s["scale"]
    top = x.amax(dim=1, keepdim=True)
    y = x.gather(1, at[:, None])[:, 0]
    p = (x - top).exp_()
    del x
    total = p.sum(dim=1, keepdim=True)
    lse = (top + total.log())[:, 0]
    out = {"loss": torch.where(live, lse - y, 0.0), "lse": torch.where(live, lse, 0.0)}
    if op == "train":
        a = torch.where(live, s["d_loss"] * s["scale"], 0.0)
        p *= a[:, None] / total
        p.scatter_add_(1, at[:, None], -a[:, None])
        out["d_hidden"] = (p @ w).to(BF16)
        out["d_weight"] = (p.t() @ h).to(BF16)
    return out


def work(case):
    t, v, k, n = case["tokens"], case["vocab"], case["hidden"], _scored(case)
    if case["op"] == "embed_fwd":
        e = DTYPES[case["dtype"]].itemsize
        return {"bytes": min(n, v) * k * e + t * k * e + 8 * t, "flops": n * k}
    if case["op"] == "embed_bwd":
        e = DTYPES[case["dtype"]].itemsize
        return {"bytes": n * k * e + v * k * e + 8 * t, "flops": n * k}
    if case["op"] == "score":
        return {"bytes": 2 * (n + v) * k + 16 * t, "flops": 2 * n * v * k}
    # loss and gradients: the logits, G W and G^T H, each product once
    return {"bytes": 2 * (n + v) * k + 20 * t + 2 * (t + v) * k, "flops": 6 * n * v * k}


def exact(case, seed):
    """The definitions in 64 bits, a block of tokens at a time; only the rows that count take part."""
    s = prepare(case, seed)
    ids, op, v, k, t = s["ids"], case["op"], case["vocab"], case["hidden"], case["tokens"]
    rows = (ids >= 0).nonzero()[:, 0]
    if op == "embed_fwd":
        out = torch.zeros((t, k), device="cuda", dtype=F64)
        out[rows] = s["table"].index_select(0, ids[rows]).to(F64) * s["scale"]
        return out
    if op == "embed_bwd":
        # rows sorted by id, running sums along them, differences at the ids' borders, a slab of columns at a time
        order = rows[torch.sort(ids[rows], stable=True).indices]
        cut = torch.searchsorted(ids[order], torch.arange(v + 1, device="cuda"))
        out = torch.empty((v, k), device="cuda", dtype=F64)
        for c in range(0, k, 256):
            run_sum = torch.zeros((order.numel() + 1, min(256, k - c)), device="cuda", dtype=F64)
            torch.cumsum(s["d_out"][order, c:c + 256].to(F64), 0, out=run_sum[1:])
            out[:, c:c + 256] = (run_sum[cut[1:]] - run_sum[cut[:-1]]) * s["scale"]
        return out
    w = s["weight"].to(F64)
    loss, lse = torch.zeros(t, device="cuda", dtype=F64), torch.zeros(t, device="cuda", dtype=F64)
    d_hidden = torch.zeros((t, k), device="cuda", dtype=F64)
    d_weight = torch.zeros((v, k), device="cuda", dtype=F64) if op == "train" else None
    for b in rows.split(2048):
        h, y = s["hidden"][b].to(F64), ids[b]
        logits = torch.mm(h, w.T).mul_(s["scale"])
        lse[b] = torch.logsumexp(logits, dim=1)
        loss[b] = lse[b] - logits[torch.arange(len(b), device="cuda"), y]
        if op == "train":
            logits.sub_(lse[b][:, None]).exp_()
            logits[torch.arange(len(b), device="cuda"), y] -= 1.0
            logits *= (s["d_loss"][b].to(F64) * s["scale"])[:, None]
            d_hidden[b] = logits @ w
            d_weight.addmm_(logits.T, h)
    out = {"loss": loss, "lse": lse}
    return out if op == "score" else {**out, "d_hidden": d_hidden, "d_weight": d_weight}

"""What is measured of a decoder block's ends and of its activation checkpoints in 8 bits.

    block   y = x + s a(g) z,  z = w_o o / rms(o) (or o without a norm after the block),  h = w_i y / rms(y)
            rms(v) = sqrt(mean(v^2) + eps) over a token's channels; a is the identity or the logistic function; the gate g is one
            number a token, one a channel (a parameter) or one of each; without a branch o the operator is the norm before
            a block alone (y = x).  Under the gradients dy of the residual stream and dh of h:
                dY = dy + (w_i dh - v mean(w_i dh v)) / rms(y),  v = y / rms(y);   dx = dY
                q = s dY;  dz = q a(g);  dg = q z a'(g), summed over what the gate is shared by
                do = (w_o dz - u mean(w_o dz u)) / rms(o),  u = o / rms(o);   dw_i = sum dh v,  dw_o = sum dz u  (over tokens)
            With checkpoints, v and u of the backward pass come from the 8-bit forms of y (as it is stored) and of o.
    glu     a = g sigma(g) u, the activation of a gated MLP; its gradients under da, and a once more (the gradient of the
            product behind it needs it), from g and u or from their 8-bit forms
    ckpt    the 8-bit form and back: 32 neighbouring channels of a token share a power of two 2^e, the smallest with
            max |x| < 127.5 2^e (e >= -126), and each is rounded to the nearest of -127 .. 127 times it, ties to even
    wgrad   dW = dY^T X of a product whose input X was kept in 8 bits, as it is or as the norm before the block left it
            (a factor for each token, one for each channel)

Sizes: hidden 3584 (28 heads of 128) with 24576 tokens, 16384 of them responses, is the geometry of the default benchmark; 256
with 512 inside the MLP is that of the model-level test.  The others are generic, ragged ones among them.
"""
import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DTYPES = {"bf16": BF16, "f32": F32}
EPS, SCALE = 1e-6, 0.7


def _block(name, tokens, hidden, stream, *, train=True, branch=True, post=True, gate="none", sigmoid=False, ckpt=False):
    return {"name": name, "op": "block", "tokens": tokens, "hidden": hidden, "stream": stream, "train": train, "branch": branch,
            "post": post, "gate": gate, "sigmoid": sigmoid, "ckpt": ckpt}


def listed():
    return [
        # an update step over all tokens of the default tree, fp32 residual stream, norms on both sides, forward and backward
        _block("block-24576-f32", 24576, 3584, "f32"),
        # its responses with everything that the backward pass needs kept in 8 bits, a gate for each token
        _block("block-16384-ckpt", 16384, 3584, "bf16", gate="token", sigmoid=True, ckpt=True),
        # a mid-sized model with a full gate (a projection of the stream), ragged in both sizes
        _block("block-2183-full-gate", 2183, 1032, "f32", gate="full", sigmoid=True),
        # the norm before the first block, its input kept in 8 bits, a middling batch
        _block("block-5001-before-ckpt", 5001, 2000, "f32", branch=False, post=False, ckpt=True),
        # the model-level test's width, a learned scale for each channel: latency
        _block("block-743-small", 743, 256, "f32", gate="channel"),
        # one sampled token on its way through a block's end: latency
        _block("block-1-forward", 1, 3584, "bf16", train=False),
        # the widest activation of an update step: the gated MLP of the default tree's responses, g and u kept in 8 bits
        {"name": "glu-16384-ckpt", "op": "glu", "tokens": 16384, "cols": 18944, "ckpt": True},
        # the model-level test's MLP: latency
        {"name": "glu-743-small", "op": "glu", "tokens": 743, "cols": 512, "ckpt": False},
        # the gradient of an MLP's input projection from the norm's 8-bit checkpoint, all responses of the default tree
        {"name": "wgrad-16384", "op": "wgrad", "tokens": 16384, "cols": 3584, "out": 18944, "dtype": "bf16", "factors": True},
        # a ragged batch of a mid-sized model, gradient in 32 bits
        {"name": "wgrad-2183-f32", "op": "wgrad", "tokens": 2183, "cols": 1032, "out": 520, "dtype": "f32", "factors": False},
        # the residual stream of the default tree into 8 bits and back
        {"name": "ckpt-24576", "op": "ckpt", "tokens": 24576, "cols": 3584, "dtype": "f32"},
        # the model-level test's hidden states: latency
        {"name": "ckpt-743-small", "op": "ckpt", "tokens": 743, "cols": 256, "dtype": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["block", "block", "glu", "wgrad", "ckpt"])
    if op == "block":
        branch = rng.random() < 0.8
        ckpt = rng.random() < 0.5
        stream = "bf16" if branch and ckpt else rng.choice(["f32", "bf16"])
        gate = rng.choice(["none", "token", "channel", "full"]) if branch else "none"
        case = _block("", _log_uniform(rng, 1, 24576), 8 * _log_uniform(rng, 8, 448), stream, train=rng.random() < 0.75, branch=branch,
                      post=branch and rng.random() < 0.75, gate=gate, sigmoid=gate != "none" and rng.random() < 0.5, ckpt=ckpt)
        del case["name"]
        return case
    if op == "glu":
        return {"op": op, "tokens": _log_uniform(rng, 1, 16384), "cols": 8 * _log_uniform(rng, 8, 2368), "ckpt": rng.random() < 0.6}
    if op == "wgrad":
        factors = rng.random() < 0.5
        return {"op": op, "tokens": _log_uniform(rng, 1, 16384), "cols": 8 * _log_uniform(rng, 8, 448), "out": 8 * _log_uniform(rng, 8, 2368),
                "dtype": "bf16" if factors else rng.choice(["bf16", "f32"]), "factors": factors}
    return {"op": op, "tokens": _log_uniform(rng, 1, 24576), "cols": 8 * _log_uniform(rng, 8, 448), "dtype": rng.choice(["bf16", "f32"])}


# ------------------------------------------------------------------------------------------------------------- inputs
def _randn(shape, gen, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=F32).mul_(scale)


def _activations(shape, gen, dtype, scale=1.0):
    """Hidden states as models have them: channels of unequal size, one in a hundred ten times the others', tokens too."""
    chan = torch.exp(_randn((1, shape[1]), gen, 0.4))
    chan[torch.rand((1, shape[1]), generator=gen, device="cuda") < 0.01] *= 10.0
    return _randn(shape, gen, scale).mul_(chan).mul_(torch.exp(_randn((shape[0], 1), gen, 0.2))).to(dtype)


def _weight(n, gen, dtype):
    return (1.0 + _randn((n,), gen, 0.2)).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    t, op = case["tokens"], case["op"]
    if op == "block":
        c, dt = case["hidden"], DTYPES[case["stream"]]
        s["x"] = _activations((t, c), gen, dt, 2.0)
        s["w_i"] = _weight(c, gen, dt)
        if case["branch"]:
            s["o"] = _activations((t, c), gen, BF16, 0.5)
            s["w_o"] = _weight(c, gen, dt) if case["post"] else None
            shape = {"token": (t,), "channel": (c,), "full": (t, c)}.get(case["gate"])
            # logits of a logistic gate, or factors around one half
            s["g"] = None if shape is None else _randn(shape, gen).add_(0.5).to(dt if case["gate"] == "channel" else BF16)
        if case["train"]:
            s["dy"], s["dh"] = _randn((t, c), gen, 0.05).to(dt), _randn((t, c), gen, 0.05).to(BF16)
    elif op == "glu":
        s["g"], s["u"] = _activations((t, case["cols"]), gen, BF16), _activations((t, case["cols"]), gen, BF16)
        s["da"] = _randn((t, case["cols"]), gen, 0.05).to(BF16)
    elif op == "wgrad":
        s["x"] = _activations((t, case["cols"]), gen, BF16, 2.0)
        s["dy"] = _randn((t, case["out"]), gen, 0.05).to(BF16)
        s["row"] = (0.5 * torch.exp(_randn((t,), gen, 0.3))) if case["factors"] else None
        s["col"] = _weight(case["cols"], gen, BF16) if case["factors"] else None
    else:
        s["x"] = _activations((t, case["cols"]), gen, DTYPES[case["dtype"]], 2.0)
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The handle and the buffers that a user's program keeps."""
    from paper_2609_33133_b200 import binding as B
    case = s["case"]
    t, op = case["tokens"], case["op"]
    e = lambda shape, dt: torch.empty(shape, device="cuda", dtype=dt)
    box = lambda cols: e((t, B.ckpt_pitch(cols)), torch.uint8)
    if op == "block":
        c, dt = case["hidden"], DTYPES[case["stream"]]
        blk = B.Block(c, device=0, eps=EPS, residual_scale=SCALE, gate=case["gate"], gate_sigmoid=case["sigmoid"])
        s["h"], s["r_i"] = e((t, c), BF16), e((t,), F32)
        branch = case["branch"]
        s["y"] = e((t, c), dt) if branch else None
        s["r_o"] = e((t,), F32) if case["post"] else None
        if case["train"]:
            if case["ckpt"]:
                s["ckpt_y"], s["ckpt_o"] = box(c), box(c) if branch else None
            s["dx"], s["dw_i"] = e((t, c), dt), e((c,), dt)
            if branch:
                s["do"] = e((t, c), BF16)
                s["dw_o"] = e((c,), dt) if case["post"] else None
                s["dg"] = None if s["g"] is None else torch.empty_like(s["g"])
            s["ws"] = e((blk.workspace_bytes(t),), torch.uint8)
    else:
        blk = B.Block(256, device=0)
        if op == "glu":
            for k in ("a", "dg", "du", "a_again"):
                s[k] = torch.empty_like(s["g"])
            s["ckpt_g"], s["ckpt_u"] = (box(case["cols"]), box(case["cols"])) if case["ckpt"] else (None, None)
        elif op == "wgrad":
            s["ckpt"], s["dw"] = box(case["cols"]), e((case["out"], case["cols"]), DTYPES[case["dtype"]])
            s["ws"] = e((blk.wgrad_workspace_bytes(t, case["out"], case["cols"]),), torch.uint8)
        else:
            s["ckpt"], s["out"] = box(case["cols"]), e((t, case["cols"]), BF16)
    s["blk"] = blk


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    case, blk = s["case"], s["blk"]
    op = case["op"]
    if op == "block":
        branch, keep = case["branch"], case["train"] and case["ckpt"]
        o, g, w_o = (s["o"], s["g"], s["w_o"]) if branch else (None, None, None)
        ckpt_y, ckpt_o = (s["ckpt_y"], s["ckpt_o"]) if keep else (None, None)
        blk.fwd(s["x"], o, g, w_o, s["w_i"], s["y"], s["h"], s["r_o"], s["r_i"], ckpt_y, ckpt_o)
        out = {"h": s["h"], "y": s["y"]} if branch else {"h": s["h"]}
        if case["train"]:
            y = ckpt_y if keep else s["y"] if branch else s["x"]
            do, dg, dw_o = (s["do"], s["dg"], s["dw_o"]) if branch else (None, None, None)
            blk.bwd(s["dy"], s["dh"], y, ckpt_o if keep else o, g, w_o, s["w_i"], s["r_o"], s["r_i"], s["dx"], do, dg, dw_o, s["dw_i"], s["ws"])
            more = {"dx": s["dx"], "do": do, "dg": dg, "dw_o": dw_o, "dw_i": s["dw_i"]}
            out |= {k: v for k, v in more.items() if v is not None}
        return out
    if op == "glu":
        blk.glu_fwd(s["g"], s["u"], s["a"], s["ckpt_g"], s["ckpt_u"])
        g, u = (s["ckpt_g"], s["ckpt_u"]) if case["ckpt"] else (s["g"], s["u"])
        blk.glu_bwd(s["da"], g, u, s["dg"], s["du"], s["a_again"])
        return {k: s[k] for k in ("a", "dg", "du", "a_again")}
    blk.pack(s["x"], s["ckpt"])
    if op == "wgrad":
        blk.wgrad(s["dy"], s["ckpt"], s["dw"], s["ws"], s["row"], s["col"])
        return s["dw"]
    blk.unpack(s["ckpt"], s["out"])
    return s["out"]


# ------------------------------------------------------------------------------------------------------------- plain form
def _in_8_bits(x):
    """The values that the 8-bit form of x stands for.  Every step is exact in 32 bits but the rounding itself."""
    t, c = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -c % 32)).view(t, -1, 32)
    m, e = torch.frexp(v.abs().amax(dim=2, keepdim=True))          # max = m 2^e, 1/2 <= m < 1
    e = (e - 7 + (m >= 127.5 / 128).int()).clamp_(min=-126)
    unit, per = ((127 + e) << 23).view(F32), ((127 - e) << 23).view(F32)   # 2^e, 2^-e
    return (v * per).round_().mul_(unit).view(t, -1)[:, :c]


def _rsqrt_mean(v):
    return torch.rsqrt(v.square().mean(dim=1, keepdim=True) + EPS)


def _gate(case, g):
    """a(g) and a'(g), shaped to go with [tokens, channels]."""
    g = g.float()[:, None] if case["gate"] == "token" else g.float()
    if not case["sigmoid"]:
        return g, 1.0
    a = 1.0 / (1.0 + torch.exp(-g))
    return a, a * (1.0 - a)


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "block":
        return _plain_block(s, case)
    if op == "glu":
        return _plain_glu(s, case)
    x = _in_8_bits(s["x"])
    if op == "ckpt":
        return x.to(BF16)
    if s["row"] is not None:
        x = x * s["row"][:, None] * s["col"].float()
    return (s["dy"].float().t() @ x).to(DTYPES[case["dtype"]])


def _plain_block(s, case):
    dt, w_i, branch = DTYPES[case["stream"]], s["w_i"].float(), case["branch"]
    y = s["x"].float()
    if branch:
        o = s["o"].float()
        r_o = _rsqrt_mean(o) if case["post"] else 1.0
        w_o = s["w_o"].float() if case["post"] else 1.0
        a, slope = (1.0, 0.0) if s["g"] is None else _gate(case, s["g"])
        y = y + SCALE * a * (w_o * (o * r_o))
    r_i = _rsqrt_mean(y)
    out = {"h": (w_i * (y * r_i)).to(BF16)}
    if branch:
        out["y"] = y.to(dt)
    if not case["train"]:
        return out
    dh = s["dh"].float()
    v = (_in_8_bits(y.to(dt)) if case["ckpt"] else y) * r_i
    p = w_i * dh
    d = s["dy"].float() + r_i * (p - v * (p * v).mean(dim=1, keepdim=True))
    out["dx"] = d.to(dt)
    if branch:
        u = (_in_8_bits(o) if case["ckpt"] else o) * r_o
        q = SCALE * d
        dz = q * a
        p = w_o * dz
        out["do"] = (r_o * (p - u * (p * u).mean(dim=1, keepdim=True)) if case["post"] else p).to(BF16)
        if s["g"] is not None:
            dg = q * (w_o * u) * slope
            over = {"token": 1, "channel": 0}.get(case["gate"])
            out["dg"] = (dg if over is None else dg.sum(dim=over)).to(s["g"].dtype)
        if case["post"]:
            out["dw_o"] = (dz * u).sum(dim=0).to(dt)
    out["dw_i"] = (dh * v).sum(dim=0).to(dt)
    return out


def _plain_glu(s, case):
    g, u, da = s["g"].float(), s["u"].float(), s["da"].float()
    a = (g / (1.0 + torch.exp(-g)) * u).to(BF16)
    if case["ckpt"]:
        g, u = _in_8_bits(g), _in_8_bits(u)
    sig = 1.0 / (1.0 + torch.exp(-g))
    silu = g * sig
    return {"a": a, "dg": (da * u * sig * (1.0 + g * (1.0 - sig))).to(BF16), "du": (da * silu).to(BF16), "a_again": (silu * u).to(BF16)}


# ------------------------------------------------------------------------------------------------------------- work, exact
def work(case):
    t, op = case["tokens"], case["op"]
    if op == "block":
        c, e = case["hidden"], DTYPES[case["stream"]].itemsize
        n, branch = t * c, case["branch"]
        gate = 2 * {"none": 0, "token": t, "channel": c, "full": n}[case["gate"]]
        reads, writes, flops = n * e + e * c, n * 2, 5 * n                   # x; h
        if branch:
            reads, writes, flops = reads + 2 * n + gate + e * c * case["post"], writes + n * e, flops + 9 * n
        if case["train"]:
            reads, writes, flops = reads + n * (e + 2), writes + n * e + e * c, flops + 10 * n
            if branch:
                writes, flops = writes + 2 * n + gate + e * c * case["post"], flops + 14 * n
        return {"bytes": reads + writes, "flops": flops}
    c = case["cols"]
    if op == "glu":
        return {"bytes": 14 * t * c, "flops": 20 * t * c}
    if op == "wgrad":
        return {"bytes": 2 * t * c + 2 * t * case["out"] + DTYPES[case["dtype"]].itemsize * c * case["out"] + (4 * t + 2 * c) * case["factors"],
                "flops": 2 * t * c * case["out"]}
    return {"bytes": (DTYPES[case["dtype"]].itemsize + 2) * t * c, "flops": 4 * t * c}


def _exact_8_bits(x):
    """From the definition: the exponent from the base-2 logarithm, put right where it is off, quotients in 64 bits."""
    t, c = x.shape
    v = torch.zeros((t, -(-c // 32) * 32), device=x.device, dtype=F64)
    v[:, :c] = x.to(F64)
    v = v.view(t, -1, 32)
    top = v.abs().amax(dim=2, keepdim=True)
    e = torch.where(top > 0, torch.log2(top.clamp(min=2.0 ** -200) / 127.5).floor() + 1.0, -126.0)
    e = torch.where(top < 127.5 * torch.exp2(e - 1.0), e - 1.0, e)
    e = torch.where(top >= 127.5 * torch.exp2(e), e + 1.0, e).clamp(min=-126.0)
    unit = torch.exp2(e)
    return (torch.round(v / unit) * unit).view(t, -1)[:, :c]


def exact(case, seed):
    s = prepare(case, seed)
    op, t = case["op"], case["tokens"]
    if op == "ckpt":
        return _exact_8_bits(s["x"])
    if op == "wgrad":
        out = torch.zeros((case["out"], case["cols"]), device="cuda", dtype=F64)
        for b in torch.arange(t, device="cuda").split(4096):
            x = _exact_8_bits(s["x"][b])
            if case["factors"]:
                x = torch.einsum("tc,t,c->tc", x, s["row"][b].to(F64), s["col"].to(F64))
            out.addmm_(s["dy"][b].to(F64).T, x)
        return out
    if op == "glu":
        out = {k: torch.empty((t, case["cols"]), device="cuda", dtype=F64) for k in ("a", "dg", "du", "a_again")}
        for b in torch.arange(t, device="cuda").split(2048):
            g, u, da = (s[k][b].to(F64) for k in ("g", "u", "da"))
            out["a"][b] = torch.sigmoid(g) * g * u
            if case["ckpt"]:
                g, u = _exact_8_bits(g), _exact_8_bits(u)
            p = torch.sigmoid(g)
            out["a_again"][b] = p * g * u
            out["du"][b] = da * p * g
            out["dg"][b] = da * u * (p + g * p * torch.sigmoid(-g))
        return out
    return _exact_block(s, case)


def _exact_block(s, case):
    dt, c, t = DTYPES[case["stream"]], case["hidden"], case["tokens"]
    names = ["h"] + ["y"] * case["branch"] + (["dx"] + ["do"] * case["branch"] if case["train"] else [])
    out = {k: torch.empty((t, c), device="cuda", dtype=F64) for k in names}
    w_i = s["w_i"].to(F64)
    gated = case["branch"] and s["g"] is not None
    if case["train"]:
        out["dw_i"] = torch.zeros(c, device="cuda", dtype=F64)
        if case["post"]:
            out["dw_o"] = torch.zeros(c, device="cuda", dtype=F64)
        if gated:
            out["dg"] = torch.zeros(s["g"].shape, device="cuda", dtype=F64)
    for b in torch.arange(t, device="cuda").split(4096):
        y = s["x"][b].to(F64)
        if case["branch"]:
            o = s["o"][b].to(F64)
            rms_o = torch.sqrt(o.pow(2).sum(1, keepdim=True) / c + EPS) if case["post"] else torch.ones((len(b), 1), device="cuda", dtype=F64)
            w_o = s["w_o"].to(F64) if case["post"] else torch.ones(c, device="cuda", dtype=F64)
            a, slope = torch.ones((1, 1), device="cuda", dtype=F64), None
            if gated:
                g = s["g"].to(F64) if case["gate"] == "channel" else s["g"][b].to(F64)
                g = g[:, None] if case["gate"] == "token" else g[None, :] if case["gate"] == "channel" else g
                a = torch.sigmoid(g) if case["sigmoid"] else g
                slope = a * torch.sigmoid(-g) if case["sigmoid"] else torch.ones_like(g)
            y = y + o * w_o * a * SCALE / rms_o
            out["y"][b] = y
        rms_y = torch.sqrt(y.pow(2).sum(1, keepdim=True) / c + EPS)
        out["h"][b] = y * w_i / rms_y
        if not case["train"]:
            continue
        dh = s["dh"][b].to(F64)
        v = (_exact_8_bits(y.to(dt)) if case["ckpt"] else y) / rms_y
        along = torch.einsum("tc,tc,c->t", dh, v, w_i)[:, None] / c
        d = s["dy"][b].to(F64) + (dh * w_i - along * v) / rms_y
        out["dx"][b] = d
        out["dw_i"] += torch.einsum("tc,tc->c", dh, v)
        if case["branch"]:
            u = (_exact_8_bits(o) if case["ckpt"] else o) / rms_o
            dz = SCALE * d * a
            if case["post"]:
                along = torch.einsum("tc,tc,c->t", dz, u, w_o)[:, None] / c
                out["do"][b] = (dz * w_o - along * u) / rms_o
                out["dw_o"] += torch.einsum("tc,tc->c", dz, u)
            else:
                out["do"][b] = dz
            if gated:
                dg = SCALE * d * u * w_o * slope
                if case["gate"] == "channel":
                    out["dg"] += dg.sum(0)
                else:
                    out["dg"][b] = dg.sum(1) if case["gate"] == "token" else dg
    return out

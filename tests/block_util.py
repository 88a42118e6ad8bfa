"""Plain 64-bit forms of a decoder block's ends, the 8-bit checkpoints, the gated MLP and the weight gradient, and the error bounds of
the kernels' arithmetic."""
import torch

F64, F32, BF16, F16, U8 = torch.float64, torch.float32, torch.bfloat16, torch.float16, torch.uint8
U = 2.0 ** -24                      # half a step of fp32
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}      # half a step of a type, relative
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -25}   # half a step (or more) below the smallest normal number


def rounding(dtype, ref):
    return HALF[dtype] * ref.abs() + TINY[dtype]


# ---------------------------------------------------------------- the 8-bit form
def encode(x):
    """(integers [n, cols], exponent bytes [n, groups]) by the definition, in 64 bits."""
    n, c = x.shape
    v = torch.zeros(n, -(-c // 32) * 32, dtype=F64)
    v[:, :c] = x.to(F64)
    v = v.view(n, -1, 32)
    bad = ~torch.isfinite(v).all(2, keepdim=True)
    top = torch.where(bad, 0.0, v.abs().amax(2, keepdim=True))
    e = torch.full_like(top, -126.0)
    for k in range(-126, 123):      # the smallest power of two with top < 127.5 2^e
        e = torch.where(top >= 127.5 * 2.0 ** k, float(k + 1), e)
    q = torch.where(bad, 0.0, torch.round(v / torch.exp2(e)))
    return q.view(n, -1)[:, :c], torch.where(bad, 255.0, e + 127)[:, :, 0]


def decode(q, byte, cols):
    unit = torch.where(byte == 255, float("nan"), torch.exp2(byte.to(F64) - 127))
    return (q.to(F64) * unit.repeat_interleave(32, 1)[:, :cols])


def in_8_bits(x):
    return decode(*encode(x), x.shape[1])


def split(ckpt, cols):
    """(integers, exponent bytes) of a checkpoint tensor."""
    at, groups = -(-cols // 16) * 16, -(-cols // 32)
    return ckpt[:, :cols].view(torch.int8).to(F64), ckpt[:, at:at + groups].to(F64)


# ---------------------------------------------------------------- block ends
def gate_form(g, kind, sigmoid, n, c):
    """a(g) and a'(g) as [n, c]."""
    if g is None:
        return torch.ones(n, c, dtype=F64), torch.zeros(n, c, dtype=F64)
    g = g.to(F64)
    g = g[:, None].expand(n, c) if kind == "token" else g[None, :].expand(n, c) if kind == "channel" else g
    if not sigmoid:
        return g, torch.ones_like(g)
    a = torch.sigmoid(g)
    return a, a * torch.sigmoid(-g)


def block_fwd(x, o, g, w_out, w_in, *, kind, sigmoid, scale, eps, y_type, h_type):
    """{name: (value, bound)}.  Bounds: a sum over a row is 16 additions in a thread, 5 over a warp, up to 19 over warps, of terms >= 0, so within 40
    half steps; half of that and two steps of rsqrt reach r: 24 half steps, which with three products stay below 30.  logistic: 1e-6 = 17."""
    n, c = x.shape
    x = x.to(F64)
    out = {}
    y, ey = x, torch.zeros_like(x)
    if o is not None:
        o = o.to(F64)
        r = torch.rsqrt(o.pow(2).mean(1, keepdim=True) + eps) if w_out is not None else torch.ones(n, 1, dtype=F64)
        a, _ = gate_form(g, kind, sigmoid, n, c)
        z = scale * a * o * r * (1.0 if w_out is None else w_out.to(F64))
        y = x + z
        ey = 50 * U * z.abs() + U * y.abs()
        out["y"] = (y, ey + rounding(y_type, y))
        out["r_out"] = (r[:, 0], 30 * U * r[:, 0])
    if w_in is not None:
        r = torch.rsqrt(y.pow(2).mean(1, keepdim=True) + eps)
        off = ey.norm(dim=1, keepdim=True) / y.norm(dim=1, keepdim=True).clamp(min=1e-300)
        h = w_in.to(F64) * y * r
        out["h"] = (h, w_in.to(F64).abs() * r * ey + h.abs() * (30 * U + off) + rounding(h_type, h))
        out["r_in"] = (r[:, 0], r[:, 0] * (30 * U + off[:, 0]))
    return out


def block_bwd(dy, dh, y, o, g, w_out, w_in, r_out, r_in, *, kind, sigmoid, scale, types, lanes=148):
    """{name: (value, bound)} from the very y, o, r_out, r_in that the kernel is given (y, o: the values that checkpoints stand for).
    A sum over a row: 40 half steps of the sum of magnitudes, three more for its terms' products.  A sum over tokens: n / lanes and a block more in a
    thread, then at most 15 groups, lanes / 8 and 8 more; n / lanes + 80 half steps of the sum of magnitudes in all."""
    lead = dy if dy is not None else dh
    n, c = lead.shape
    out = {}
    chain = n / lanes + 80
    d = torch.zeros(n, c, dtype=F64) if dy is None else dy.to(F64)
    ed = torch.zeros_like(d)
    if dh is not None:
        dh, y, r, w = dh.to(F64), y.to(F64), r_in.to(F64)[:, None], w_in.to(F64)
        v, p = y * r, w * dh
        s = (p * v).sum(1, keepdim=True) / c
        es = 45 * U * (p * v).abs().sum(1, keepdim=True) / c
        t = r * (p - v * s)
        d = d + t
        ed = r * (v.abs() * es + 6 * U * (p.abs() + (v * s).abs())) + 2 * U * (d.abs() + t.abs())
        out["dw_in"] = ((dh * v).sum(0), (chain + 3) * U * (dh * v).abs().sum(0) + rounding(types["w"], (dh * v).sum(0)))
    out["dx"] = (d, ed + rounding(types["x"], d))
    if o is None:
        return out
    o = o.to(F64)
    r = r_out.to(F64)[:, None] if w_out is not None else torch.ones(n, 1, dtype=F64)
    w = w_out.to(F64) if w_out is not None else torch.ones(c, dtype=F64)
    a, slope = gate_form(g, kind, sigmoid, n, c)
    u = o * r
    q, eq = scale * d, abs(scale) * (ed + U * d.abs())
    dz, edz = q * a, eq * a.abs() + 20 * U * (q * a).abs()
    if w_out is not None:
        p, ep = w * dz, w.abs() * edz + U * (w * dz).abs()
        s = (p * u).sum(1, keepdim=True) / c
        es = ((ep * u.abs()).sum(1, keepdim=True) + 45 * U * (p * u).abs().sum(1, keepdim=True)) / c + 20 * U * s.abs()
        do = r * (p - u * s)
        edo = r * (ep + u.abs() * es + 6 * U * (p.abs() + (u * s).abs()))
        out["dw_out"] = ((dz * u).sum(0), ((edz + 3 * U * dz.abs()) * u.abs()).sum(0) + (chain + 20) * U * (dz * u).abs().sum(0)
                         + rounding(types["w"], (dz * u).sum(0)))
    else:
        do, edo = dz, edz
    out["d_o"] = (do, edo + rounding(types["o"], do))
    if g is not None:
        m, em = q * w * u * slope, (eq + 4 * U * q.abs()) * (w * u * slope).abs() + 40 * U * (q * w * u * slope).abs()
        em = em + 2e-7 * (q * w * u).abs() * sigmoid       # (1 - a loses half a step of one where a is near one)
        if kind == "full":
            out["d_gate"] = (m, em + rounding(types["gate"], m))
        else:
            dim = 1 if kind == "token" else 0
            val = m.sum(dim)
            out["d_gate"] = (val, em.sum(dim) + (45 if dim else chain + 20) * U * m.abs().sum(dim) + rounding(types["gate"], val))
    return out


# ---------------------------------------------------------------- gated MLP
def glu(g, u, da, dtype):
    """a, dg, du with bounds: the logistic function is within 1e-6 relative for |g| < 8 (its argument's product with log2(e), 2^x, the
    reciprocal) and keeps an absolute error below 1e-6 elsewhere; 1 + g (1 - s) adds three roundings of terms up to 1 + |g|."""
    g, u, da = g.to(F64), u.to(F64), da.to(F64)
    s = torch.sigmoid(g)
    es = 1.2e-6 * s * (1 + g.abs() / 8)
    a, du = g * s * u, da * g * s
    t = 1 + g * torch.sigmoid(-g)
    dg = da * u * s * t
    et = g.abs() * (es + 2 * U) + 2 * U * (1 + (g * torch.sigmoid(-g)).abs())
    ea = (g * u).abs() * es + 4 * U * a.abs()
    return {"a": (a, ea + rounding(dtype, a)), "du": (du, (da * g).abs() * es + 4 * U * du.abs() + rounding(dtype, du)),
            "dg": (dg, (da * u).abs() * (es * t.abs() + s * et) + 4 * U * dg.abs() + rounding(dtype, dg))}


# ---------------------------------------------------------------- weight gradient
def wgrad(dy, x, row, col, dtype):
    """x: what the checkpoint stands for.  Products of bf16 numbers are exact in fp32; the tensor core's adder loses up to 2^-23 of the running sum of
    magnitudes for each of its additions (one for 16 tokens, at most 128 in a row), rounded additions follow; a token's factor rounds the operand, 2^-8."""
    dy, x = dy.to(F64), x.to(F64)
    n = dy.shape[0]
    if row is not None:
        x = x * row.to(F64)[:, None]
    f = col.to(F64) if col is not None else torch.ones(x.shape[1], dtype=F64)
    val = dy.T @ x * f
    mag = dy.abs().T @ x.abs() * f.abs()
    adds = 2 * min(n / 16 + 1, 128) + n / 2048 + 40
    return val, adds * U * mag + (2.0 ** -8 * mag if row is not None else 0.0) + 4 * U * val.abs() + rounding(dtype, val)


def wgrad_exact_operand(dy, x, row, col, dtype, chain=128):
    """As wgrad, from the operand that the tensor core is given: a token's factor rounds it once, to a number that can be formed exactly here, so that what is left are the
    additions, of which `chain` come in a row inside the tensor core.  Returns the value before its delivery and the bound of that."""
    n = dy.shape[0]
    x = x.to(F32)
    if row is not None:
        x = (x * row.to(F32)[:, None]).to(BF16)
    dy, x = dy.to(F64), x.to(F64)
    f = col.to(F64) if col is not None else torch.ones(x.shape[1], dtype=F64)
    val = dy.T @ x * f
    return val, (2 * min(n / 16 + 1, chain) + n / 2048 + 44) * U * (dy.abs().T @ x.abs() * f.abs())


def check_delivered(got, want, what=""):
    """A rounding of a value within the bound: rounding keeps the order, so what is delivered lies between the roundings of the interval's ends."""
    (val, bound), got = want, got.detach().cpu()
    lo, hi = (val - bound).to(got.dtype), (val + bound).to(got.dtype)
    bad = ~((lo <= got) & (got <= hi))      # (NaN is bad)
    assert got.shape == val.shape and not bad.any(), (what, int(bad.sum()), float((got.to(F64) - val).abs()[bad].max()), bad.nonzero()[0].tolist())


def check(got, want, what=""):
    val, bound = want
    got = got.detach().cpu().to(F64)
    assert got.shape == val.shape, (what, got.shape, val.shape)
    off = (got - val).abs()
    bad = ~(off <= bound)       # (NaN is bad)
    assert not bad.any(), (what, int(bad.sum()), float((off / bound)[bad].max()), float(off[bad].max()), bad.nonzero()[0].tolist())
    return float((off / bound).max()) if off.numel() else 0.0

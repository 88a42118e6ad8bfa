"""Plain 64-bit forms of the embedding lookup and the vocabulary cross entropy, and the error bounds of the kernels' arithmetic."""
import math

import torch

F64, F32, BF16 = torch.float64, torch.float32, torch.bfloat16


def make_loss(tokens, vocab, hidden, seed, masked=0.0, push=16.0, ids_dtype=torch.int64):
    """bf16 hidden states leaning towards their targets by a random amount, bf16 weights with rows of about unit length."""
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(vocab, hidden, generator=g) * hidden ** -0.5).to(BF16)
    y = torch.randint(0, vocab, (tokens,), generator=g)
    h = (torch.randn(tokens, hidden, generator=g) + push * torch.rand(tokens, 1, generator=g) * w[y].float()).to(BF16)
    y[torch.randperm(tokens, generator=g)[: int(masked * tokens)]] = -100
    a = torch.randn(tokens, generator=g)
    return h, w, y.to(ids_dtype), a


def loss_reference(h, w, y, a, scale=1.0):
    """lse, loss, dH, dW and, elementwise, the sums of magnitudes that the error bounds are made of.  Rows with a negative
    target are left out (they may hold NaN)."""
    rows = (y >= 0).nonzero()[:, 0]
    hv, wv, yv, av = h[rows].to(F64), w.to(F64), y[rows].long(), a[rows].to(F64)
    x = scale * hv @ wv.T
    lse = torch.logsumexp(x, 1)
    hot = torch.nn.functional.one_hot(yv, w.shape[0]).to(F64)
    p = torch.exp(x - lse[:, None])
    g = (av * scale)[:, None] * (p - hot)
    mag = (av * scale).abs()[:, None] * (p + hot)
    full = lambda v, shape: torch.zeros(shape, dtype=F64).index_copy_(0, rows, v)
    t, k = h.shape
    return {"lse": full(lse, (t,)), "loss": full(lse - x[torch.arange(len(rows)), yv], (t,)),
            "d_hidden": full(g @ wv, (t, k)), "d_weight": g.T @ hv,
            "g_dh": full(g.abs() @ wv.abs(), (t, k)), "g_dw": g.abs().T @ hv.abs(),
            "m_dh": full(mag @ wv.abs(), (t, k)), "m_dw": mag.T @ hv.abs(),
            "low_dh": full(((av * scale).abs()[:, None] + 1) * wv.abs().sum(0), (t, k)),
            "low_dw": (((av * scale).abs()[:, None] + 1) * hv.abs()).sum(0),
            "reach": float(scale * hv.norm(dim=1).max() * wv.norm(dim=1).max()) if len(rows) else 0.0}


def loss_bounds(ref, vocab, hidden, tokens):
    """Bounds of the absolute error.
    logit: `hidden` products, exact in fp32, added up with an error of at most 2^-23 of the running magnitude each (the
      tensor core's adder does not round to nearest): hidden 2^-23 sum |h w| <= hidden 2^-23 |h| |w|; scaled into base 2
      and back, two more roundings.
    lse: the error of its logits, of exp2 (2 units in the last place) and of at most 128 + vocab / 512 additions, all of
      terms >= 0, and the rounding of the result (three steps: m ln 2, the logarithm, their sum).
    G: relative error of p from its logit, its lse and exp2; the subtraction at the target; one rounding to bf16, 2^-8.
    dH, dW: that, carried through sums of `vocab` or `tokens` products added in fp32, and one rounding to bf16.
    underflow: exp2 returns zero for results below the smallest normal number, 2^-126, so p is off by less than that and
      G by less than 2^-126 (|a c| + 1), whatever its size (the 1 covers G's own rounding there); carried through the
      sums (low_dh, low_dw); products and sums below 2^-126 may be lost as well, one for each addition."""
    u = 2.0 ** -23
    x = (hidden + 2) * u * ref["reach"]
    lse = x + (4 + 128 + vocab / 512) * u + 3 * u * (ref["lse"].abs() + ref["reach"])
    p = x + lse.max().item() + 4 * u + 3 * u * ref["reach"]
    dh = 2 ** -8 * ref["g_dh"] + (p + vocab * u) * 1.01 * ref["m_dh"]
    dw = 2 ** -8 * ref["g_dw"] + (p + tokens * u) * 1.01 * ref["m_dw"]
    low = 2.0 ** -126
    dh, dw = dh + low * (ref["low_dh"] + vocab + 1), dw + low * (ref["low_dw"] + tokens + 1)
    return {"lse": lse, "loss": lse + x, "d_hidden": dh * (1 + 2 ** -8) + 2 ** -8 * ref["d_hidden"].abs(),
            "d_weight": dw * (1 + 2 ** -8) + 2 ** -8 * ref["d_weight"].abs()}


def embed_grad_reference(d_out, ids, vocab, scale):
    """The sums in 64 bits, and their error bound in fp32 before the delivery rounding: n additions of 2^-24 each and the product."""
    live = ids >= 0
    d, i = d_out[live].to(F64), ids[live].long()
    out = torch.zeros(vocab, d_out.shape[1], dtype=F64).index_add_(0, i, d) * scale
    mag = torch.zeros(vocab, d_out.shape[1], dtype=F64).index_add_(0, i, d.abs()) * abs(scale)
    n = torch.bincount(i, minlength=vocab).to(F64)[:, None]
    return out, mag * (n + 1) * 2.0 ** -24


def assert_within(got, ref, bound, name=""):
    got = got.detach().cpu().to(F64)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert torch.isfinite(got).all(), (name, "not finite")
    over = (got - ref).abs() - bound
    assert not got.numel() or over.max().item() <= 0, (name, over.max().item(), (got - ref).abs().max().item())


def gradient_bounds_two_halves(ref, vocab, hidden, tokens):
    """Bounds of dH and dW before they are delivered, for up to 256 rows: as in loss_bounds, but G is hi + lo with hi = bf16(G) and
    lo = bf16(G - hi), which leaves 2^-8 of 2^-8 of an element, and the contractions run over both halves, twice as many additions."""
    u, low = 2.0 ** -23, 2.0 ** -126
    x = (hidden + 2) * u * ref["reach"]
    lse = x + (4 + 128 + vocab / 512) * u + 3 * u * (ref["lse"].abs().max().item() + ref["reach"])
    p = x + lse + 4 * u + 3 * u * ref["reach"]
    return {"d_hidden": 2 ** -16 * ref["g_dh"] + (p + 2 * vocab * u) * 1.01 * ref["m_dh"] + low * (ref["low_dh"] + 2 * vocab + 2),
            "d_weight": 2 ** -16 * ref["g_dw"] + (p + 2 * tokens * u) * 1.01 * ref["m_dw"] + low * (ref["low_dw"] + 2 * tokens + 2)}


def half_step_bf16(x):
    """Half the distance of neighbouring bf16 numbers at x: 2^(e - 9) for |x| = m 2^e with m in [1/2, 1)."""
    return torch.exp2((torch.frexp(x.to(F64).abs())[1] - 9).to(F64))


def delivered_bf16(ref, bound):
    """Bound of a result that is within `bound` of ref before it is rounded to bf16."""
    return bound + half_step_bf16(ref.abs() + bound)


LONG_CASES = [(40, 513, 65536), (600, 700, 33024)]   # a row of 128 KB; hidden states of more than a row group


def make_long(tokens, vocab, hidden, seed):
    """Long contractions whose bounds still see a wrong result: |h| |w| near one, so that hidden 2^-23 |h| |w| is under 1e-2, and losses
    that differ by up to one from row to row."""
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(vocab, hidden, generator=g) * hidden ** -0.5).to(BF16)
    y = torch.randint(0, vocab, (tokens,), generator=g)
    h = (torch.randn(tokens, hidden, generator=g) * 0.3 * hidden ** -0.5 + torch.rand(tokens, 1, generator=g) * w[y].float()).to(BF16)
    return h, w, y, torch.randn(tokens, generator=g)

"""Embedding lookup and vocabulary cross entropy, forward and backward, against plain 64-bit forms: every type, sizes from
one token to several tiles in each direction, masked rows that hold NaN, pieces of the vocabulary, repeated ids."""
import numpy as np
import pytest
import torch

from tests import lm_util as lu

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
GUARD = 2048


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import binding
    return binding


def guarded(shape, dtype, fill=float("nan")):
    """A tensor with `GUARD` bytes of a pattern on both sides: (tensor, check)."""
    n = int(np.prod(shape)) * dtype.itemsize
    raw = torch.full((n + 2 * GUARD,), 0x5A, device="cuda", dtype=torch.uint8)
    t = raw[GUARD:GUARD + n].view(dtype).view(shape)
    t.fill_(fill)

    def check():
        assert (raw[:GUARD] == 0x5A).all() and (raw[GUARD + n:] == 0x5A).all(), "written outside the tensor"
    return t, check


def workspace(lm, tokens):
    """Scratch full of NaN patterns: nothing may be read before it is written."""
    return torch.full((lm.workspace_bytes(tokens),), 0xFF, device="cuda", dtype=torch.uint8)


def run_loss(B, h, w, y, a, scale=1.0, piece_bytes=0, dw_dtype=BF16, lm=None):
    t, k, v = h.shape[0], h.shape[1], w.shape[0]
    lm = lm or B.LM(v, k, device=0, logit_scale=scale, piece_bytes=piece_bytes)
    hc, wc, yc, ac = h.cuda(), w.cuda(), y.cuda(), a.cuda()
    ws = workspace(lm, t)
    out, checks = {}, []
    for name, shape, dt in (("loss", (t,), F32), ("lse", (t,), F32), ("d_hidden", (t, k), BF16), ("d_weight", (v, k), dw_dtype)):
        out[name], c = guarded(shape, dt)
        checks.append(c)
    lm.loss_fwd(hc, wc, yc, out["loss"], out["lse"], ws)
    ws.fill_(0xFF)
    lm.loss_bwd(hc, wc, yc, out["lse"], ac, out["d_hidden"], out["d_weight"], ws)
    torch.cuda.synchronize()
    assert lm.device_status() == (0, 0)
    for c in checks:
        c()
    return out


LOSS_CASES = [
    # tokens, vocab, hidden, masked, scale, piece_bytes
    (1, 1, 8, 0.0, 1.0, 0),
    (1, 503, 256, 0.0, 1.0, 0),
    (2, 129, 72, 0.0, 0.7, 0),
    (17, 257, 64, 0.2, 1.0, 0),
    (33, 700, 320, 0.0, 1.0, 0),
    (64, 1000, 128, 0.0, 1.0, 0),
    (77, 3001, 1000, 0.1, 1.0, 0),
    (90, 300, 4104, 0.0, 1.0, 1),           # two pieces of 256 columns, seventeen tiles of hidden columns
    (100, 40000, 64, 0.0, 1.0, 0),          # more tiles than SMs
    (128, 2000, 192, 0.3, 1.0, 0),
    (65, 255, 120, 0.0, 1.0, 0),
    (127, 513, 264, 0.1, 1.3, 0),
    (129, 503, 256, 0.1, 1.0, 0),
    (200, 2049, 520, 0.5, 1.0, 1),          # nine pieces of 256 columns
    (257, 3001, 1032, 0.25, 1.0, 0),
    (300, 1500, 200, 0.0, 1.0, 700 * 1024),  # two pieces
    (256, 5000, 136, 0.0, 1.0, 1 << 20),
    (700, 777, 328, 0.0, 1.0, 0),
    (300, 600, 288, 0.0, 1.0, 0),           # hidden sizes whose last tile has 32, 64, 128, 40 and 192 columns
    (300, 600, 320, 0.0, 1.0, 0),
    (260, 600, 384, 0.1, 1.0, 0),
    (260, 600, 296, 0.0, 1.0, 0),
    (150, 600, 448, 0.0, 1.0, 0),
    (1500, 300, 24, 0.6, 1.0, 0),
    (40, 513, 65536, 0.0, 1.0, 0),          # a row of 128 KB
    (600, 700, 33024, 0.0, 1.0, 0),         # hidden states of more than a row group: groups of one tile of rows
]


@pytest.mark.parametrize("t,v,k,masked,scale,piece", LOSS_CASES)
def test_loss_matches_plain_form(B, t, v, k, masked, scale, piece):
    h, w, y, a = lu.make_loss(t, v, k, seed=t * 7 + v, masked=masked)
    h[y < 0] = float("nan")
    a[y < 0] = float("inf")
    out = run_loss(B, h, w, y, a, scale, piece)
    ref = lu.loss_reference(h, w, y, a, scale)
    bound = lu.loss_bounds(ref, v, k, t)
    for n in ("lse", "loss", "d_hidden", "d_weight"):
        lu.assert_within(out[n], ref[n], bound[n], n)


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
def test_loss_fp32_weight_gradient_and_accumulation(B, ids):
    t, v, k = 150, 700, 96
    h, w, y, a = lu.make_loss(t, v, k, seed=5, masked=0.1, ids_dtype=ids)
    out = run_loss(B, h, w, y, a, dw_dtype=F32, piece_bytes=1)
    ref = lu.loss_reference(h, w, y, a)
    bound = lu.loss_bounds(ref, v, k, t)
    lu.assert_within(out["d_weight"], ref["d_weight"], bound["d_weight"], "d_weight")
    lm = B.LM(v, k, device=0)
    acc = torch.ones(v, k, device="cuda", dtype=F32)
    ws = workspace(lm, t)
    lm.loss_bwd(h.cuda(), w.cuda(), y.cuda(), out["lse"], a.cuda(), None, acc, ws, accumulate=True)
    lu.assert_within(acc, ref["d_weight"] + 1, bound["d_weight"] + 2.0 ** -23 * (ref["d_weight"].abs() + 1), "accumulated")


def test_either_gradient_alone_is_bitwise_the_pair(B):
    t, v, k = 200, 900, 136
    h, w, y, a = lu.make_loss(t, v, k, seed=6)
    out = run_loss(B, h, w, y, a)
    lm = B.LM(v, k, device=0)
    ws = workspace(lm, t)
    dh, dw = torch.empty(t, k, device="cuda", dtype=BF16), torch.empty(v, k, device="cuda", dtype=BF16)
    args = (h.cuda(), w.cuda(), y.cuda(), out["lse"], a.cuda())
    lm.loss_bwd(*args, dh, None, ws)
    lm.loss_bwd(*args, None, dw, ws)
    lm.loss_bwd(*args, None, None, ws)
    assert torch.equal(dh, out["d_hidden"]) and torch.equal(dw, out["d_weight"])


def test_loss_is_bitwise_repeatable(B):
    h, w, y, a = lu.make_loss(333, 2222, 264, seed=7, masked=0.1)
    one, two = run_loss(B, h, w, y, a), run_loss(B, h, w, y, a)
    for n in one:
        assert torch.equal(one[n], two[n]), n


@pytest.mark.parametrize("t", [1, 40, 300])
def test_no_row_scored(B, t):
    """Every row masked and full of NaN: zeros everywhere, and an accumulator that stays as it was."""
    v, k = 300, 64
    h = torch.full((t, k), float("nan"), dtype=BF16)
    _, w, _, _ = lu.make_loss(1, v, k, seed=8)
    y, a = torch.full((t,), -1), torch.ones(t)
    out = run_loss(B, h, w, y, a)
    for n, x in out.items():
        assert (x == 0).all(), n
    lm = B.LM(v, k, device=0)
    acc = torch.full((v, k), 3.0, device="cuda")
    lm.loss_bwd(h.cuda(), w.cuda(), y.cuda(), out["lse"], a.cuda(), None, acc, workspace(lm, t), accumulate=True)
    assert (acc == 3).all()


def test_no_tokens(B):
    v, k = 300, 64
    lm = B.LM(v, k, device=0)
    e = lambda *s, dt=BF16: torch.zeros(s, device="cuda", dtype=dt)
    ids, f = e(0, dt=torch.int64), e(0, dt=F32)
    dw = torch.full((v, k), float("nan"), device="cuda", dtype=BF16)
    ws = workspace(lm, 0)
    lm.loss_fwd(e(0, k), e(v, k), ids, f, f, ws)
    lm.loss_bwd(e(0, k), e(v, k), ids, f, f, e(0, k), dw, ws)
    assert (dw == 0).all()
    dw.fill_(float("nan"))
    lm.embed_bwd(e(0, k), ids, dw, ws)
    assert (dw == 0).all()
    lm.embed_fwd(e(v, k), ids, e(0, k))
    assert lm.device_status() == (0, 0)


@pytest.mark.parametrize("t", [5, 200])
def test_confident_and_large_logits(B, t):
    """Targets with probability near one and logits of several hundred: the maximum has to be subtracted."""
    v, k = 600, 128
    h, w, y, a = lu.make_loss(t, v, k, seed=9, push=400.0)
    out = run_loss(B, h, w, y, a)
    ref = lu.loss_reference(h, w, y, a)
    bound = lu.loss_bounds(ref, v, k, t)
    for n in ("lse", "loss", "d_hidden", "d_weight"):
        lu.assert_within(out[n], ref[n], bound[n], n)


@pytest.mark.parametrize("t", [7, 150, 400])
def test_confident_rows_keep_their_gradient(B, t):
    """Targets with 1 - p from 1e-3 to 1/2 at a long contraction.  dH of a row is (1 - p) a times a mean difference of rows of W, so an error
    dz of the target's logit less lse is dz / (1 - p) of it.  dz: lse and its roundings, 4 half steps of numbers below 32, 4 x 2^-20;
    the dot product, chains of at most 16 + 9 additions of partial sums below 32, 25 x 2^-20.  The other elements of G are as exact as
    their logits, hidden x 2^-23 |h| |w| relative.  Two roundings to bf16."""
    v, k = 300, 3584
    g = torch.Generator().manual_seed(t)
    w = (torch.randn(v, k, generator=g) * k ** -0.5).to(BF16)
    y = torch.randint(0, v, (t,), generator=g)
    h = (0.3 * torch.randn(t, k, generator=g) + (6.0 + 6.5 * torch.rand(t, 1, generator=g)) * w[y].float()).to(BF16)
    a = torch.ones(t)
    out = run_loss(B, h, w, y, a)
    ref = lu.loss_reference(h, w, y, a)
    left = 1 - torch.exp(-ref["loss"])
    assert left.min() > 5e-4 and (left < 5e-3).any()
    err = (out["d_hidden"].cpu().double() - ref["d_hidden"]).norm(dim=1) / ref["d_hidden"].norm(dim=1)
    size = h.double().norm(dim=1) * w.double().norm(dim=1).max()
    assert (err <= 2 * 2.0 ** -8 + 29 * 2.0 ** -20 / left + k * 2.0 ** -23 * size).all(), err.max()
    if t <= 256:   # (G in two halves: its rounding to bf16 is gone)
        assert (err <= 2.0 ** -8 + 29 * 2.0 ** -20 / left + k * 2.0 ** -23 * size).all(), err.max()


def test_nan_in_one_scored_row_stays_in_it(B):
    t, v, k = 140, 400, 64
    h, w, y, a = lu.make_loss(t, v, k, seed=10)
    h[3] = float("nan")
    lm = B.LM(v, k, device=0)
    loss, lse = torch.zeros(t, device="cuda"), torch.zeros(t, device="cuda")
    lm.loss_fwd(h.cuda(), w.cuda(), y.cuda(), loss, lse, workspace(lm, t))
    bad = torch.isnan(loss).cpu()
    assert bad[3] and bad.sum() == 1 and torch.isnan(lse).cpu().sum() == 1


def test_gradient_against_differences(B):
    """dH and dW along random directions against central differences of the summed loss (fp64 step on the plain form's inputs is
    not needed: the loss itself is differenced in 64 bits by the plain form, the kernel's gradient is projected)."""
    t, v, k = 60, 333, 72
    h, w, y, a = lu.make_loss(t, v, k, seed=11, push=4.0)
    out = run_loss(B, h, w, y, a)
    g = torch.Generator().manual_seed(12)
    u_h, u_w = torch.randn(t, k, generator=g, dtype=torch.float64), torch.randn(v, k, generator=g, dtype=torch.float64)
    f = lambda e: float((lu.loss_reference(h.double() + e * u_h, w.double() + e * u_w, y, a)["loss"] * a.double()).sum())
    diff = (f(1e-5) - f(-1e-5)) / 2e-5
    got = float((out["d_hidden"].cpu().double() * u_h).sum() + (out["d_weight"].cpu().double() * u_w).sum())
    ref = lu.loss_reference(h, w, y, a)
    b = lu.loss_bounds(ref, v, k, t)
    bound = float((b["d_hidden"] * u_h.abs()).sum() + (b["d_weight"] * u_w.abs()).sum())
    # the bound adds every rounding with the same sign; independent ones give its root of squares
    six = 6 * float(((b["d_hidden"] * u_h) ** 2).sum() + ((b["d_weight"] * u_w) ** 2).sum()) ** 0.5
    assert abs(got - diff) <= min(bound, six) + 1e-6 * abs(diff), (got, diff, bound, six)


def test_token_id_out_of_range_is_reported_and_left_out(B):
    t, v, k = 50, 100, 64
    h, w, y, a = lu.make_loss(t, v, k, seed=13)
    y[7] = v
    ref = y.clone()
    ref[7] = -1
    lm = B.LM(v, k, device=0)
    ws = workspace(lm, t)
    loss, lse = torch.zeros(t, device="cuda"), torch.zeros(t, device="cuda")
    lm.loss_fwd(h.cuda(), w.cuda(), y.cuda(), loss, lse, ws)
    assert lm.device_status() == (-1, 7)
    want = run_loss(B, h, w, ref, a)
    assert torch.equal(loss, want["loss"]) and torch.equal(lse, want["lse"])
    out = torch.full((t, k), float("nan"), device="cuda", dtype=BF16)
    lm.embed_fwd(w.cuda(), y.cuda(), out)
    assert lm.device_status() == (-1, 7) and (out[7] == 0).all()
    dw, dw2 = torch.empty(v, k, device="cuda", dtype=F32), torch.empty(v, k, device="cuda", dtype=F32)
    lm.embed_bwd(h.cuda(), y.cuda(), dw, ws)
    assert lm.device_status() == (-1, 7)
    lm.embed_bwd(h.cuda(), ref.cuda(), dw2, ws)
    assert lm.device_status() == (0, 0) and torch.equal(dw, dw2)


# ------------------------------------------------------------------------------------------------ embedding
TYPES = [BF16, F16, F32]


@pytest.mark.parametrize("table_dtype", TYPES)
@pytest.mark.parametrize("out_dtype", TYPES)
@pytest.mark.parametrize("t,v,k", [(1, 1, 8), (1, 5000, 2056), (37, 503, 256), (1000, 333, 1032)])
def test_embedding_is_rounded_once(B, table_dtype, out_dtype, t, v, k):
    g = torch.Generator().manual_seed(t + v)
    table = torch.randn(v, k, generator=g).to(table_dtype).cuda()
    ids = torch.randint(-1, v, (t,), generator=g).cuda()
    lm = B.LM(v, k, device=0, embed_scale=k ** 0.5)
    out, check = guarded((t, k), out_dtype)
    for i in (ids, ids.int()):
        out.fill_(float("nan"))
        lm.embed_fwd(table, i, out)
        torch.cuda.synchronize()
        scale = torch.tensor(k ** 0.5, dtype=F32).cuda()
        want = torch.where(ids[:, None] >= 0, table[ids.clamp(min=0)].float() * scale, 0.0).to(out_dtype)
        assert torch.equal(out, want)
        check()
    assert lm.device_status() == (0, 0)


def ids_of(kind, t, v, g):
    if kind == "one":
        return torch.full((t,), v - 1)
    if kind == "masked":
        return torch.full((t,), -5)
    if kind == "frequent":
        return torch.exp(torch.rand(t, generator=g, dtype=torch.float64) * np.log(v)).floor().long().sub(1).clamp(0, v - 1)
    i = torch.randint(0, v, (t,), generator=g)
    i[torch.randperm(t, generator=g)[: t // 10]] = -100
    return i


@pytest.mark.parametrize("kind", ["uniform", "frequent", "one", "masked"])
@pytest.mark.parametrize("t,v,k", [(1, 1, 8), (1, 700, 264), (31, 3, 64), (743, 503, 256), (4097, 1030, 40), (9000, 20000, 64)])
@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32), (F16, F16), (F32, BF16)])
def test_embedding_gradient(B, kind, t, v, k, types):
    d_dtype, w_dtype = types
    g = torch.Generator().manual_seed(t * 3 + v)
    ids = ids_of(kind, t, v, g)
    d = torch.randn(t, k, generator=g).to(d_dtype)
    d[ids < 0] = float("nan")
    lm = B.LM(v, k, device=0, embed_scale=2.5)
    ws = workspace(lm, t)
    out, check = guarded((v, k), w_dtype)
    lm.embed_bwd(d.cuda(), ids.cuda(), out, ws)
    torch.cuda.synchronize()
    check()
    ref, bound = lu.embed_grad_reference(d, ids, v, 2.5)
    half_step = torch.finfo(w_dtype).eps / 2
    tiny = 2.0 ** -25 if w_dtype == F16 else 0.0      # half of fp16's smallest step
    lu.assert_within(out, ref, bound * (1 + half_step) + half_step * ref.abs() + tiny, "d_table")
    again = torch.empty_like(out)
    lm.embed_bwd(d.cuda(), ids.int().cuda(), again, ws)
    assert torch.equal(out, again)
    if w_dtype == F32:
        acc = torch.ones(v, k, device="cuda")
        lm.embed_bwd(d.cuda(), ids.cuda(), acc, ws, accumulate=True)
        lu.assert_within(acc, ref + 1, bound + 2.0 ** -23 * (ref.abs() + 1), "accumulated")
    assert lm.device_status() == (0, 0)


# ------------------------------------------------------------------------------------------------ streams, graphs, refusals
def test_on_a_side_stream_and_in_a_graph(B):
    t, v, k = 130, 700, 136
    h, w, y, a = (x.cuda() for x in lu.make_loss(t, v, k, seed=21, masked=0.1))
    want = run_loss(B, h, w, y, a)
    lm = B.LM(v, k, device=0)
    ws = workspace(lm, t)
    e = lambda s, dt: torch.zeros(s, device="cuda", dtype=dt)
    loss, lse, dh, dw, tab, out = e((t,), F32), e((t,), F32), e((t, k), BF16), e((v, k), BF16), e((v, k), F32), e((t, k), BF16)

    def step():
        lm.embed_fwd(w, y, out)
        lm.loss_fwd(h, w, y, loss, lse, ws)
        lm.loss_bwd(h, w, y, lse, a, dh, dw, ws)
        lm.embed_bwd(h, y, tab, ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    for n, x in (("loss", loss), ("lse", lse), ("d_hidden", dh), ("d_weight", dw)):
        assert torch.equal(x, want[n]), n
    tab_eager, out_eager = tab.clone(), out.clone()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
    # the graph reads its inputs when it is replayed: other rows, another mask
    h2, _, y2, a2 = (x.cuda() for x in lu.make_loss(t, v, k, seed=22, masked=0.4))
    want2 = run_loss(B, h2, w, y2, a2)
    h_old, y_old, a_old = h.clone(), y.clone(), a.clone()
    for src, ref in (((h2, y2, a2), want2), ((h_old, y_old, a_old), want)):
        for dst, x in zip((h, y, a), src):
            dst.copy_(x)
        for x in (loss, lse, dh, dw, tab, out):
            x.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for n, x in (("loss", loss), ("lse", lse), ("d_hidden", dh), ("d_weight", dw)):
            assert torch.equal(x, ref[n]), n
    assert torch.equal(tab, tab_eager) and torch.equal(out, out_eager)
    assert lm.device_status() == (0, 0)


def test_two_streams_with_workspaces_of_their_own(B):
    t, v, k = 300, 1111, 72
    lm = B.LM(v, k, device=0)
    sets = []
    for seed in (31, 32):
        h, w, y, a = lu.make_loss(t, v, k, seed=seed, masked=0.1)
        sets.append(dict(want=run_loss(B, h, w, y, a), args=[x.cuda() for x in (h, w, y, a)], ws=workspace(lm, t), s=torch.cuda.Stream(),
                         out=[torch.zeros(s, device="cuda", dtype=d) for s, d in (((t,), F32), ((t,), F32), ((t, k), BF16), ((v, k), BF16))]))
    torch.cuda.synchronize()
    for _ in range(3):
        for q in sets:
            h, w, y, a = q["args"]
            loss, lse, dh, dw = q["out"]
            with torch.cuda.stream(q["s"]):
                lm.loss_fwd(h, w, y, loss, lse, q["ws"])
                lm.loss_bwd(h, w, y, lse, a, dh, dw, q["ws"])
    torch.cuda.synchronize()
    for q in sets:
        for n, x in zip(("loss", "lse", "d_hidden", "d_weight"), q["out"]):
            assert torch.equal(x, q["want"][n]), n


def test_one_workspace_for_every_smaller_call(B):
    """A program keeps the scratch for its largest batch: every smaller call runs in it, whatever ran before."""
    v, k, most = 2100, 72, 5400
    lm = B.LM(v, k, device=0)
    ws, check = guarded((lm.workspace_bytes(most),), torch.uint8, fill=0xFF)
    h, w, y, a = lu.make_loss(most, v, k, seed=51, masked=0.1)
    hc, wc, yc, ac = h.cuda(), w.cuda(), y.cuda(), a.cuda()
    tab = torch.empty(v, k, device="cuda")
    for t in (5400, 1, 4096, 128, 129, 256, 257, 511, 2000, 64, 5000, 4097):
        loss, lse = torch.empty(t, device="cuda"), torch.empty(t, device="cuda")
        dh, dw = torch.empty(t, k, device="cuda", dtype=BF16), torch.empty(v, k, device="cuda", dtype=BF16)
        lm.loss_fwd(hc[:t], wc, yc[:t], loss, lse, ws)
        lm.loss_bwd(hc[:t], wc, yc[:t], lse, ac[:t], dh, dw, ws)
        lm.embed_bwd(hc[:t], yc[:t], tab, ws)
        ref = lu.loss_reference(h[:t], w, y[:t], a[:t])
        b = lu.loss_bounds(ref, v, k, t)
        for n, x in (("loss", loss), ("d_hidden", dh), ("d_weight", dw)):
            lu.assert_within(x, ref[n], b[n], (t, n))
        check()
    assert lm.device_status() == (0, 0)


@pytest.mark.parametrize("t", [20, 140, 300, 5000])
def test_tensors_and_scratch_on_odd_16_byte_boundaries(B, t):
    """Everything 16 bytes off the allocator's boundaries, which is all that the interface asks for."""
    v, k = 777, 72

    def off(x):
        raw = torch.empty(x.nbytes + 16, device="cuda", dtype=torch.uint8)
        y = raw[16:].view(x.dtype).view(x.shape)
        y.copy_(x)
        assert y.data_ptr() % 32 == 16
        return y
    h, w, y, a = lu.make_loss(t, v, k, seed=81, masked=0.1)
    lm = B.LM(v, k, device=0)
    hc, wc, ws = off(h.cuda()), off(w.cuda()), off(workspace(lm, t))
    dh, dw, tab = off(torch.zeros(t, k, device="cuda", dtype=BF16)), off(torch.zeros(v, k, device="cuda", dtype=BF16)), off(torch.zeros(v, k, device="cuda"))
    loss, lse = torch.zeros(t, device="cuda"), torch.zeros(t, device="cuda")
    lm.loss_fwd(hc, wc, y.cuda(), loss, lse, ws)
    lm.loss_bwd(hc, wc, y.cuda(), lse, a.cuda(), dh, dw, ws)
    lm.embed_bwd(hc, y.cuda(), tab, ws)
    ref = lu.loss_reference(h, w, y, a)
    b = lu.loss_bounds(ref, v, k, t)
    for n, x in (("loss", loss), ("d_hidden", dh), ("d_weight", dw)):
        lu.assert_within(x, ref[n], b[n], n)
    want, bound = lu.embed_grad_reference(h, y, v, 1.0)
    lu.assert_within(tab, want, bound, "d_table")
    lm.embed_fwd(wc, y.cuda(), dh)
    assert torch.equal(dh, torch.where(y.cuda()[:, None] >= 0, wc[y.cuda().clamp(min=0)].float(), 0.0).to(BF16))


@pytest.mark.parametrize("lanes", [1, 3, 7, 1000])
@pytest.mark.parametrize("t", [20, 140, 900])
def test_any_number_of_lanes(B, lanes, t):
    """Few CTAs walk many tiles each, through every turn of the rings and accumulators; more CTAs than the GPU holds queue."""
    v, k = 3333, 328
    h, w, y, a = lu.make_loss(t, v, k, seed=61, masked=0.1)
    lm = B.LM(v, k, device=0, n_lanes=lanes, piece_bytes=1 << 21)
    out = run_loss(B, h, w, y, a, lm=lm)
    ref = lu.loss_reference(h, w, y, a)
    b = lu.loss_bounds(ref, v, k, t)
    for n in ("lse", "loss", "d_hidden", "d_weight"):
        lu.assert_within(out[n], ref[n], b[n], n)
    d = torch.randn(t, k, generator=torch.Generator().manual_seed(1))
    tab = torch.empty(v, k, device="cuda")
    lm.embed_bwd(d.cuda(), y.cuda(), tab, workspace(lm, t))
    want, bound = lu.embed_grad_reference(d, y, v, 1.0)
    lu.assert_within(tab, want, bound, "d_table")


@pytest.mark.parametrize("t,v,k", [(5000, 300, 16), (6000, 300000, 8), (70000, 5, 8), (40000, 1 << 20, 8), (3000, 1500000, 8)])
def test_embedding_gradient_sort_passes(B, t, v, k):
    """One, two and three radix passes, a table of five rows under 70000 tokens, vocabularies beyond the one-block sort's."""
    g = torch.Generator().manual_seed(t)
    ids = ids_of("frequent", t, v, g)
    ids[::9] = -1
    d = torch.randn(t, k, generator=g)
    lm = B.LM(v, k, device=0)
    out = torch.full((v, k), float("nan"), device="cuda")
    lm.embed_bwd(d.cuda(), ids.cuda(), out, workspace(lm, t))
    want, bound = lu.embed_grad_reference(d, ids, v, 1.0)
    lu.assert_within(out, want, bound, "d_table")


def test_negative_and_tiny_scales(B):
    t, v, k = 60, 500, 64
    h, w, y, a = lu.make_loss(t, v, k, seed=71)
    for scale in (-1.5, 1e-3, 7.0):
        out = run_loss(B, h, w, y, a, scale)
        ref = lu.loss_reference(h, w, y, a, scale)
        ref["reach"] = abs(ref["reach"])
        b = lu.loss_bounds(ref, v, k, t)
        for n in ("lse", "loss", "d_hidden", "d_weight"):
            lu.assert_within(out[n], ref[n], b[n], (scale, n))


def test_refusals(B):
    t, v, k = 10, 100, 64
    lm = B.LM(v, k, device=0)
    h, w, y, a = (x.cuda() for x in lu.make_loss(t, v, k, seed=1))
    f, ws = torch.zeros(t, device="cuda"), workspace(lm, t)
    with pytest.raises(ValueError):
        lm.loss_fwd(h.float(), w, y, f, f, ws)                       # type
    with pytest.raises(ValueError):
        lm.loss_fwd(h, w.t().contiguous().t(), y, f, f, ws)          # layout
    with pytest.raises(ValueError):
        lm.loss_fwd(h, w[:50], y, f, f, ws)                          # shape
    with pytest.raises(ValueError):
        lm.loss_fwd(h, w, y.float(), f, f, ws)                       # ids
    with pytest.raises(ValueError):
        lm.loss_fwd(h.cpu(), w, y, f, f, ws)                         # device
    with pytest.raises(B.AugtreeError) as e:
        lm.loss_fwd(h, w, y, f, f, ws[:256])
    assert e.value.code == -3
    with pytest.raises(B.AugtreeError) as e:
        lm.loss_bwd(h, w, y, f, f, h, torch.empty_like(w), ws, accumulate=True)   # accumulation in bf16
    assert e.value.code == -2
    with pytest.raises(B.AugtreeError) as e:
        lm.embed_bwd(h, y, torch.empty_like(w), ws, accumulate=True)
    assert e.value.code == -2
    with pytest.raises(B.AugtreeError) as e:
        lm.embed_bwd(h, y, torch.empty_like(w), ws[:256])
    assert e.value.code == -3
    odd = torch.zeros(t * k + 1, device="cuda", dtype=BF16)[1:].view(t, k)        # 2 bytes off a 16-byte boundary
    with pytest.raises(B.AugtreeError) as e:
        lm.loss_fwd(odd, w, y, f, f, ws)
    assert e.value.code == -1
    host = B.LM(v, k, device=None, n_lanes=148)
    with pytest.raises(ValueError):
        host.loss_fwd(h, w, y, f, f, ws)
    assert B.lib.augtree_lm_loss_fwd(host._h, None, None, None, 8, 1, None, None, None, 0, None) == -1
    assert lm.device_status() == (0, 0)


@pytest.mark.parametrize("t", [20, 130])
def test_a_wait_that_runs_out_is_reported(B, t):
    """A tile that is never loaded: the call returns, the status word names the wait, the next call is right."""
    v, k = 700, 136
    h, w, y, a = lu.make_loss(t, v, k, seed=41)
    bad = B.LM(v, k, device=0, flags=B.FLAG_TEST_SHORT_WAIT | B.FLAG_TEST_SKIP_FWD_LOAD)
    ws = workspace(bad, t)
    f = torch.zeros(t, device="cuda")
    bad.loss_fwd(h.cuda(), w.cuda(), y.cuda(), f, f.clone(), ws)
    status, site = bad.device_status()
    assert status == -5 and 80 <= site < 90
    out = run_loss(B, h, w, y, a)
    ref = lu.loss_reference(h, w, y, a)
    lu.assert_within(out["loss"], ref["loss"], lu.loss_bounds(ref, v, k, t)["loss"], "loss")

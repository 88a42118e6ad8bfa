"""Vocabulary operators where they can go wrong at their edges: batches of which nothing is scored, forbidden words, very large
logits, the border between G in one and in two halves, long contractions, matrices of more than 2^31 elements, refusals."""
import numpy as np
import pytest
import torch

from tests import lm_util as lu
from tests.test_gpu_lm import B, guarded, run_loss, workspace  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


@pytest.mark.parametrize("dw_dtype", [BF16, F32])
@pytest.mark.parametrize("piece", [0, 1])                    # one piece of the vocabulary, three of them
@pytest.mark.parametrize("t", [128, 129, 200, 256, 257])
def test_no_row_scored_either_side_of_every_limit(B, t, piece, dw_dtype):
    """Every row masked and full of NaN, scratch full of NaN: zeros everywhere, an accumulator that stays as it was."""
    v, k = 700, 72
    h = torch.full((t, k), float("nan"), dtype=BF16)
    _, w, _, _ = lu.make_loss(1, v, k, seed=8)
    y, a = torch.full((t,), -1), torch.full((t,), float("nan"))
    out = run_loss(B, h, w, y, a, piece_bytes=piece, dw_dtype=dw_dtype)
    for n, x in out.items():
        assert (x == 0).all(), n
    if dw_dtype == F32:
        lm = B.LM(v, k, device=0, piece_bytes=piece)
        acc = torch.full((v, k), 3.0, device="cuda")
        lm.loss_bwd(h.cuda(), w.cuda(), y.cuda(), out["lse"], a.cuda(), None, acc, workspace(lm, t), accumulate=True)
        assert (acc == 3).all()


def test_no_row_scored_because_every_id_is_out_of_range(B):
    t, v, k = 200, 300, 64
    h, w, y, a = lu.make_loss(t, v, k, seed=14)
    lm = B.LM(v, k, device=0)
    ws, y = workspace(lm, t), (y + v).cuda()
    loss, lse, dh, dw = (torch.full(s, float("nan"), device="cuda", dtype=d) for s, d in (((t,), F32), ((t,), F32), ((t, k), BF16), ((v, k), BF16)))
    lm.loss_fwd(h.cuda(), w.cuda(), y, loss, lse, ws)
    ws.fill_(0xFF)
    lm.loss_bwd(h.cuda(), w.cuda(), y, lse, a.cuda(), dh, dw, ws)
    assert lm.device_status()[0] == -1
    for x in (loss, lse, dh, dw):
        assert (x == 0).all()


def test_no_row_scored_through_autograd(B):
    """A wholly masked micro-batch of a training loop, its scratch where the allocator last held NaN."""
    from paper_2609_33133_b200 import autograd as A
    t, v, k = 200, 300, 64
    h, w, _, _ = lu.make_loss(t, v, k, seed=15)
    lm = B.LM(v, k, device=0)
    hc, wc = h.cuda().requires_grad_(True), w.cuda().requires_grad_(True)
    loss = A.lm_loss(lm, hc, wc, torch.full((t,), -100, device="cuda"))
    stale = torch.full((lm.workspace_parts(t)[1],), 0xFF, device="cuda", dtype=torch.uint8)
    del stale
    loss.sum().backward()
    assert (loss == 0).all() and (hc.grad == 0).all() and (wc.grad == 0).all()


@pytest.mark.parametrize("t", [6, 140, 300])
@pytest.mark.parametrize("value", [float("-inf"), torch.finfo(BF16).min])
def test_forbidden_words(B, t, value):
    """Words that a column of the weight rules out, with minus infinity or with the type's lowest value (under a hidden state of one there):
    nothing changes for the others, and a row whose target is one of them has the lse of the others and an infinite loss (or one of
    3.4e38).  The gradient of the target's logit is then -a, as p is zero."""
    v, k, out_of = 300, 64, 20
    h, w, y, a = lu.make_loss(t, v - out_of, k, seed=16, push=4.0)
    h[:, 0] = 1
    w = torch.cat([w[:out_of], w])
    w[:out_of, 0] = value
    ref = lu.loss_reference(h, w[out_of:], y, a)
    bound = lu.loss_bounds(ref, v, k, t)
    y = y + out_of
    y[1], y[4] = 7, 13
    lost = torch.tensor([1, 4])
    kept = torch.ones(t, dtype=torch.bool).index_fill_(0, lost, False)
    out = run_loss(B, h, w, y, a)
    lu.assert_within(out["lse"], ref["lse"], bound["lse"], "lse")
    lu.assert_within(out["loss"].cpu()[kept], ref["loss"][kept], bound["loss"][kept], "loss")
    loss = out["loss"].cpu()[lost]
    if value == float("-inf"):
        assert (loss == float("inf")).all(), loss
    else:     # (lse - value, one product and a rounding or two)
        assert (loss.double() / -value - 1).abs().max() <= 2.0 ** -22, loss
    # dW: relative to the magnitudes the bound of the unrestricted words has, at these rows' own p
    x = h.double() @ w[out_of:].double().T
    p = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
    hot = torch.nn.functional.one_hot(y, v).double()
    p = torch.cat([torch.zeros(t, out_of, dtype=F64), p], 1)
    want = (a.double()[:, None] * (p - hot)).T @ h.double()
    mag = (a.double().abs()[:, None] * (p + hot)).T @ h.double().abs()
    p_err = 2 * (k + 2) * 2.0 ** -23 * ref["reach"] + 2.0 ** -15      # logit and lse; exp2, sums and their roundings
    lu.assert_within(out["d_weight"], want, (2.0 ** -7 + p_err) * mag + 2.0 ** -100, "d_weight")


@pytest.mark.parametrize("t", [5, 140, 300])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_loss_of_certain_targets_with_large_logits(B, t, scale):
    """Targets ahead of every other word by more than 200: the loss is zero, exp(-200) aside.  The target is the row's maximum, so the sum
    is 1, and with d the difference of the exact and the tensor core's logit the loss is log(1 + expm1(d)) - d, whatever d is: one
    rounding of the sum, 2^-24 (1 + |d|), and eight of numbers as large as d, which is at most (hidden + 2) 2^-23 |h| |w| < 0.1.  Together
    under 4 x 2^-24.  (A logit near 2000 has a half step of 6e-5: nothing of that may be left in the result.)"""
    v, k = 300, 256
    g = torch.Generator().manual_seed(t)
    w = (torch.randn(v, k, generator=g) * k ** -0.5).to(BF16)
    y = torch.randint(0, v, (t,), generator=g)
    h = ((1000 + 1000 * torch.rand(t, 1, generator=g)) * w[y].float()).to(BF16)
    ref = lu.loss_reference(h, w, y, torch.ones(t), scale)
    assert ref["loss"].max() < 1e-80 and (k + 2) * 2.0 ** -23 * ref["reach"] < 0.1
    out = run_loss(B, h, w, y, torch.ones(t), scale)
    assert out["loss"].abs().max().item() <= 2.0 ** -22, out["loss"].abs().max().item()


def test_lookup_of_as_many_tokens_as_there_can_be(B):
    """2^31 - 4096 tokens of eight columns: the last step of a block's walk over them ends beyond 2^31."""
    t, v, k = (1 << 31) - 4096, 4, 8
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 43 GB of device memory")
    lm = B.LM(v, k, device=0)
    table = (torch.arange(v * k, device="cuda").view(v, k) + 1).to(BF16)
    ids = torch.empty(t, device="cuda", dtype=torch.int32)
    step = 1 << 27
    for b in range(0, t, step):                                  # -1, 0, 1, 2, 3, -1, ..
        n = min(step, t - b)
        ids[b:b + n] = torch.arange(b, b + n, device="cuda").remainder_(5).sub_(1)
    out = torch.full((t, k), float("nan"), device="cuda", dtype=BF16)
    lm.embed_fwd(table, ids, out)
    padded = torch.cat([torch.zeros(1, k, device="cuda", dtype=BF16), table])
    for b in range(0, t, step):
        n = min(step, t - b)
        assert torch.equal(out[b:b + n], padded[ids[b:b + n].long() + 1]), b
    assert lm.device_status() == (0, 0)
    del ids, out
    torch.cuda.empty_cache()


def test_a_handle_that_cannot_be_made_leaves_no_error_behind(B):
    """The failure is the return value's: a call on another handle or plan that follows does not report it again."""
    from paper_2609_33133_b200 import autograd as A
    plan, lm = B.Plan([130], [[64, 33]], 4, 2, 64, device=0), B.LM(100, 64, device=0)
    g = torch.Generator().manual_seed(17)
    x = [torch.randn(n, h, 64, generator=g).to(BF16).cuda() for n, h in ((130, 4), (130, 2), (130, 2), (97, 4), (97, 2), (97, 2))]
    want = A.tree_attention(plan, *x)
    with pytest.raises(B.AugtreeError) as e:
        B.LM(100, 64, device=torch.cuda.device_count() + 7)
    assert e.value.code == -4
    got = A.tree_attention(plan, *x)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    table, out = torch.ones(100, 64, device="cuda"), torch.zeros(3, 64, device="cuda")
    lm.embed_fwd(table, torch.arange(3, device="cuda"), out)
    assert (out == 1).all() and lm.device_status() == (0, 0) and plan.device_status() == (0, 0)


def test_arrays_of_a_number_per_token_off_their_elements_boundaries_are_refused(B):
    """Through the C interface (torch makes no such tensor): refused before anything is launched or written."""
    t, v, k = 10, 100, 64
    lm = B.LM(v, k, device=0)
    h, w, y, a = (x.cuda() for x in lu.make_loss(t, v, k, seed=18))
    f, dh, dw, ws = torch.full((t + 1,), 7.0, device="cuda"), torch.full_like(h, 7), torch.full_like(w, 7), workspace(lm, t)
    p = lambda x: x.data_ptr()
    st = torch.cuda.current_stream().cuda_stream
    fwd = dict(targets=p(y), id_bytes=8, loss=p(f), lse=p(f))
    bwd = dict(targets=p(y), id_bytes=8, lse=p(f), d_loss=p(a))
    for name, off in (("targets", 4), ("targets", 1), ("loss", 2), ("lse", 1)):
        q = {**fwd, name: fwd[name] + off}
        assert B.lib.augtree_lm_loss_fwd(lm._h, p(h), p(w), q["targets"], q["id_bytes"], t - 1, q["loss"], q["lse"], p(ws), ws.nbytes, st) == -1
    for name, off in (("targets", 4), ("lse", 2), ("d_loss", 1)):
        q = {**bwd, name: bwd[name] + off}
        assert B.lib.augtree_lm_loss_bwd(lm._h, p(h), p(w), q["targets"], q["id_bytes"], q["lse"], q["d_loss"], t - 1, p(dh), p(dw), 0, 0,
                                         p(ws), ws.nbytes, st) == -1
    for off, id_bytes in ((4, 8), (2, 4), (1, 8)):
        assert B.lib.augtree_embed_fwd(lm._h, p(w), 0, p(y) + off, id_bytes, t - 1, p(dh), 0, st) == -1
        assert B.lib.augtree_embed_bwd(lm._h, p(h), 0, p(y) + off, id_bytes, t - 1, p(dw), 0, 0, p(ws), ws.nbytes, st) == -1
    torch.cuda.synchronize()
    assert (f == 7).all() and (dh == 7).all() and (dw == 7).all() and lm.device_status() == (0, 0)
    # int32 ids on a boundary of four bytes are in order
    y4 = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int32), y.int()])[1:]
    lm.embed_fwd(w, y4, dh)
    assert torch.equal(dh, w[y])


@pytest.mark.parametrize("t", [3, 128, 129, 256])
def test_gradients_of_few_rows_carry_no_rounding_of_the_logit_gradient(B, t):
    """Up to 256 rows G has two halves; both gradients to within their sums' errors and their own delivery.  (With hi alone they are out of
    these bounds: tests/test_lm_host.py.)"""
    v, k = 257, 64
    h, w, y, a = lu.make_loss(t, v, k, seed=t, push=4.0)
    ref = lu.loss_reference(h, w, y, a)
    bound = lu.gradient_bounds_two_halves(ref, v, k, t)
    for piece in (0, 1):
        out = run_loss(B, h, w, y, a, dw_dtype=F32, piece_bytes=piece)
        lu.assert_within(out["d_weight"], ref["d_weight"], bound["d_weight"] + 2.0 ** -24 * ref["d_weight"].abs(), "d_weight fp32")
        lu.assert_within(out["d_hidden"], ref["d_hidden"], lu.delivered_bf16(ref["d_hidden"], bound["d_hidden"]), "d_hidden")
        out = run_loss(B, h, w, y, a, piece_bytes=piece)
        lu.assert_within(out["d_weight"], ref["d_weight"], lu.delivered_bf16(ref["d_weight"], bound["d_weight"]), "d_weight bf16")


@pytest.mark.parametrize("t,v,k", lu.LONG_CASES)
def test_long_contractions(B, t, v, k):
    """(That these bounds see zeros, swapped rows and swapped tiles: tests/test_lm_host.py.)"""
    h, w, y, a = lu.make_long(t, v, k, seed=t)
    ref = lu.loss_reference(h, w, y, a)
    bound = lu.loss_bounds(ref, v, k, t)
    out = run_loss(B, h, w, y, a)
    for n in ("lse", "loss", "d_hidden", "d_weight"):
        lu.assert_within(out[n], ref[n], bound[n], n)


@pytest.mark.parametrize("t", [3, 130, 300])
def test_matrices_of_more_than_2_31_elements(B, t):
    """600064 x 3584, 2.15e9 elements: ids, targets and rows of the gradients on both sides of element 2^31."""
    v, k = 600064, 3584
    assert v * k > 1 << 31
    if torch.cuda.mem_get_info()[0] < 50 << 30:
        pytest.skip("needs 40 GB of device memory")
    g = torch.Generator(device="cuda").manual_seed(t)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=BF16)
    w = rn(v, k).mul_(k ** -0.5)
    y = torch.randint(0, v, (t,), generator=g, device="cuda")
    y[0], y[1], y[2] = v - 1, 599187, 5                            # row 599186 holds element 2^31
    h = (rn(t, k).float() + 8 * w[y].float()).to(BF16)
    a = torch.randn(t, generator=g, device="cuda")
    lm = B.LM(v, k, device=0)
    ws = torch.full((lm.workspace_bytes(t),), 0xFF, device="cuda", dtype=torch.uint8)
    loss, lse, dh = torch.empty(t, device="cuda"), torch.empty(t, device="cuda"), torch.empty_like(h)
    dw = torch.full_like(w, float("nan"))
    lm.loss_fwd(h, w, y, loss, lse, ws)
    lm.loss_bwd(h, w, y, lse, a, dh, dw, ws)
    assert lm.device_status() == (0, 0)
    # the plain form in 64 bits, a block of words at a time; bounds as everywhere (loss_bounds), sums of magnitudes likewise
    hd, ad = h.double(), a.double()
    blocks = [slice(b, min(b + 40000, v)) for b in range(0, v, 40000)]
    want_lse = torch.logsumexp(torch.stack([torch.logsumexp(hd @ w[s].double().T, 1) for s in blocks]), 0)
    want_loss = want_lse - (hd * w[y].double()).sum(1)
    u = 2.0 ** -23
    reach = float(hd.norm(dim=1).max() * max(w[s].double().norm(dim=1).max() for s in blocks))
    x = (k + 2) * u * reach
    b_lse = x + (4 + 128 + v / 512) * u + 3 * u * (want_lse.abs() + reach)
    assert ((lse.double() - want_lse).abs() <= b_lse).all() and ((loss.double() - want_loss).abs() <= b_lse + x).all()
    p_err = x + b_lse.max().item() + 4 * u + 3 * u * reach
    want_dh, mag_dh, abs_dh = (torch.zeros(t, k, device="cuda", dtype=F64) for _ in range(3))
    step = lambda z: 2.0 ** -8 * z.abs()
    for s in blocks:
        wd = w[s].double()
        p = torch.exp(hd @ wd.T - want_lse[:, None])
        hot = (y[:, None] == torch.arange(s.start, s.stop, device="cuda")).double()
        gr, mag = ad[:, None] * (p - hot), ad.abs()[:, None] * (p + hot)
        want_dh += gr @ wd
        mag_dh += mag @ wd.abs()
        abs_dh += gr.abs() @ wd.abs()
        ref = gr.T @ hd
        off = 2 ** -8 * (gr.abs().T @ hd.abs()) + (p_err + t * u) * 1.01 * (mag.T @ hd.abs()) + 2.0 ** -100
        assert ((dw[s].double() - ref).abs() <= off * (1 + 2 ** -8) + step(ref)).all(), s
    off = 2 ** -8 * abs_dh + (p_err + v * u) * 1.01 * mag_dh + 2.0 ** -100
    assert ((dh.double() - want_dh).abs() <= off * (1 + 2 ** -8) + step(want_dh)).all()
    # the embedding of the same words, and its gradient
    ids = torch.cat([y, torch.tensor([599185, 599186, v - 1, -1], device="cuda")])
    out = torch.empty(len(ids), k, device="cuda", dtype=BF16)
    lm.embed_fwd(w, ids, out)
    assert torch.equal(out[:-1], w[ids[:-1]]) and (out[-1] == 0).all()
    dw.fill_(float("nan"))
    lm.embed_bwd(out, ids, dw, ws)
    want = torch.zeros(len(ids), k, device="cuda", dtype=F64)
    rows, back = torch.unique(ids[:-1], return_inverse=True)
    want.index_add_(0, back, out[:-1].double())
    assert (dw[rows].double() - want[: len(rows)]).abs().le(step(want[: len(rows)]) * (1 + 2.0 ** -14)).all()
    dw[rows] = 0
    for s in blocks:
        assert (dw[s] == 0).all(), s
    assert lm.device_status() == (0, 0)
    del w, dw, ws
    torch.cuda.empty_cache()


def test_calls_behind_an_event_of_another_stream(B):
    """Launches are programmatic dependents of the kernel before them in their stream; what another stream's event stands for is waited
    for all the same, right behind such a kernel."""
    t, v, k = 64, 300, 64
    lm = B.LM(v, k, device=0)
    h, w, y, a = (x.cuda() for x in lu.make_loss(t, v, k, seed=31, masked=0.1))
    want = run_loss(B, h, w, y, a)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    ws, other = workspace(lm, t), workspace(lm, t)
    e = lambda s, d: torch.zeros(s, device="cuda", dtype=d)
    loss, lse, junk, tab = e((t,), F32), e((t,), F32), e((t,), F32), e((t, k), BF16)
    for _ in range(5):
        src = torch.zeros_like(h)
        torch.cuda.synchronize()
        with torch.cuda.stream(two):
            torch.cuda._sleep(3_000_000)
            src.copy_(h)
            ready = two.record_event()
        with torch.cuda.stream(one):
            lm.loss_fwd(h, w, y, junk, junk.clone(), other)
            lm.embed_fwd(w, y, tab)
            one.wait_event(ready)
            lm.loss_fwd(src, w, y, loss, lse, ws)
        torch.cuda.synchronize()
        assert torch.equal(loss, want["loss"]) and torch.equal(lse, want["lse"])


def test_a_graph_with_branches(B):
    """Two branches of a captured graph, each with a workspace of its own, that part behind one kernel and join before another."""
    t, v, k = 140, 500, 64
    lm = B.LM(v, k, device=0)
    h, w, y, a = (x.cuda() for x in lu.make_loss(t, v, k, seed=32, masked=0.1))
    e = lambda s, d: torch.full(s, float("nan"), device="cuda", dtype=d)
    x, loss, lse, dh, dw, tab, back = e((t, k), BF16), e((t,), F32), e((t,), F32), e((t, k), BF16), e((v, k), BF16), e((v, k), F32), e((t, k), F32)
    ws, ws2 = workspace(lm, t), workspace(lm, t)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()

    def step():
        lm.embed_fwd(w, y, x)                           # both branches read it
        side.wait_stream(main)
        lm.loss_fwd(h, w, y, loss, lse, ws)
        lm.loss_bwd(h, w, y, lse, a, dh, dw, ws)
        with torch.cuda.stream(side):
            lm.embed_bwd(x, y, tab, ws2)
        main.wait_stream(side)
        lm.embed_fwd(tab, y, back)                      # reads the side branch's result
    main.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(main):
        step()
        main.synchronize()
        want = [z.clone() for z in (x, loss, lse, dh, dw, tab, back)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=main):
            step()
    for _ in range(20):
        for z in (x, loss, lse, dh, dw, tab, back):
            z.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(z, r) for z, r in zip((x, loss, lse, dh, dw, tab, back), want))
    assert lm.device_status() == (0, 0)


def test_no_tokens_through_autograd(B):
    from paper_2609_33133_b200 import autograd as A
    v, k = 300, 64
    lm = B.LM(v, k, device=0)
    table = torch.ones(v, k, device="cuda", requires_grad=True)
    none = torch.zeros(0, device="cuda", dtype=torch.int64)
    A.embed(lm, table, none).sum().backward()
    h = torch.zeros(0, k, device="cuda", dtype=BF16, requires_grad=True)
    w = torch.ones(v, k, device="cuda", dtype=BF16, requires_grad=True)
    loss = A.lm_loss(lm, h, w, none).sum()
    loss.backward()
    assert loss == 0 and (table.grad == 0).all() and (w.grad == 0).all() and h.grad.shape == h.shape


def test_a_graph_of_a_backward_pass_beside_an_eager_one(B):
    """The gradients of leaves whose eager backward pass has run, and whose eager graph still lives, captured and replayed."""
    from paper_2609_33133_b200 import autograd as A
    t, v, k = 140, 500, 64
    lm = B.LM(v, k, device=0)
    h, w, y, a = (x.cuda() for x in lu.make_loss(t, v, k, seed=33, masked=0.1))
    h.requires_grad_(True), w.requires_grad_(True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        eager = A.lm_loss(lm, h, w, y)
        want = torch.autograd.grad((eager * a).sum(), (h, w), retain_graph=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = torch.autograd.grad((A.lm_loss(lm, h, w, y) * a).sum(), (h, w))
    again = torch.autograd.grad((eager * a).sum(), (h, w))
    for z in got:
        z.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(got, want, again))


@pytest.mark.parametrize("what", ["handle", "plan"])
def test_a_handle_or_plan_that_dies_during_a_capture(B, what):
    """Python's collector may end an old handle anywhere, in the middle of a capture too: freeing its memory does not spoil that."""
    t, v, k = 40, 300, 64
    lm = B.LM(v, k, device=0)
    _, w, y, _ = (x.cuda() for x in lu.make_loss(t, v, k, seed=34))
    out = torch.zeros(t, k, device="cuda", dtype=BF16)
    lm.embed_fwd(w, y, out)
    old = B.LM(77, 64, device=0) if what == "handle" else B.Plan([130], [[64, 33]], 4, 2, 64, device=0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            lm.embed_fwd(w, y, out)
            del old
            lm.embed_fwd(w, y, out)
    out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, w[y])

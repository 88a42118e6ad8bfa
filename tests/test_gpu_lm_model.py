"""The vocabulary operators as a model uses them: autograd, the loss on a tree with its first-token seam, and a training step from
token ids to the gradient of every weight, tied and untied."""
import copy

import pytest
import torch

from tests import lm_util as lu

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
HIDDEN, H_Q, H_KV, D, MLP, VOCAB = 256, 4, 2, 64, 512, 503


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import autograd, binding, layer
    return binding, autograd, layer


def test_embedding_gradient_is_the_adjoint_of_the_lookup(mods):
    """<d_out, lookup(E + U) - lookup(E)> = <dE, U>: the lookup is linear, so the difference is exact but for rounding."""
    B, A, _ = mods
    g = torch.Generator().manual_seed(1)
    v, k, t = 300, 72, 900
    lm = B.LM(v, k, device=0, embed_scale=3.0)
    e = torch.randn(v, k, generator=g).cuda().requires_grad_(True)
    u, d = torch.randn(v, k, generator=g).cuda(), torch.randn(t, k, generator=g).cuda()
    ids = torch.randint(-1, v, (t,), generator=g).cuda()
    out = A.embed(lm, e, ids)
    out.backward(d)
    with torch.no_grad():
        diff = A.embed(lm, e + u, ids).double() - out.double()
    left, right = (d.double() * diff).sum(), (e.grad.double() * u.double()).sum()
    # each looked-up value is rounded twice (sum e + u, product), 2^-24 of at most 3 (|e| + |u|) each, on both lookups; the sums in
    # dE: up to t additions of 2^-24 each of |d| times 3
    size = (d.abs().sum() * 3 * 2 * (e.abs().max() + u.abs().max())).item() * 2.0 ** -24 * 4
    size += (u.abs().max() * d.abs().sum() * 3).item() * t * 2.0 ** -24
    assert abs(left - right).item() <= size
    out16 = A.embed(lm, e.detach().to(BF16), ids, torch.float16)
    assert out16.dtype == torch.float16


@pytest.mark.parametrize("tokens", [50, 300])
def test_loss_autograd(mods, tokens):
    B, A, _ = mods
    h, w, y, a = lu.make_loss(tokens, 700, 136, seed=3, masked=0.2)
    lm = B.LM(700, 136, device=0)
    hc, wc = h.cuda().requires_grad_(True), w.cuda().requires_grad_(True)
    loss = A.lm_loss(lm, hc, wc, y.cuda())
    (loss * a.cuda()).sum().backward()
    ref = lu.loss_reference(h, w, y, a)
    b = lu.loss_bounds(ref, 700, 136, tokens)
    lu.assert_within(loss, ref["loss"], b["loss"], "loss")
    lu.assert_within(hc.grad, ref["d_hidden"], b["d_hidden"], "d_hidden")
    lu.assert_within(wc.grad, ref["d_weight"], b["d_weight"], "d_weight")
    # an expanded upstream gradient, a frozen weight, a frozen hidden state
    h2 = h.cuda().requires_grad_(True)
    A.lm_loss(lm, h2, w.cuda(), y.cuda()).sum().backward()
    ref1 = lu.loss_reference(h, w, y, torch.ones(tokens))
    lu.assert_within(h2.grad, ref1["d_hidden"], lu.loss_bounds(ref1, 700, 136, tokens)["d_hidden"], "d_hidden, frozen weight")
    w2 = w.cuda().requires_grad_(True)
    A.lm_loss(lm, h.cuda(), w2, y.cuda()).sum().backward()
    lu.assert_within(w2.grad, ref1["d_weight"], lu.loss_bounds(ref1, 700, 136, tokens)["d_weight"], "d_weight, frozen hidden")


def test_loss_gradients_captured_in_a_graph(mods):
    B, A, _ = mods
    h, w, y, _ = (x.cuda() for x in lu.make_loss(140, 600, 64, seed=4))
    lm = B.LM(600, 64, device=0)
    h.requires_grad_(True), w.requires_grad_(True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want = [x.clone() for x in torch.autograd.grad(A.lm_loss(lm, h, w, y).sum(), (h, w))]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = torch.autograd.grad(A.lm_loss(lm, h, w, y).sum(), (h, w))
    for x in got:
        x.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def tree(B):
    prompt_len, branch_len = [300, 129], [[130, 64, 257, 1], [200, 33]]
    plan = B.Plan(prompt_len, branch_len, H_Q, H_KV, D, device=0)
    g = torch.Generator().manual_seed(5)
    return plan, torch.randint(0, VOCAB, (plan.total_p,), generator=g).cuda(), torch.randint(0, VOCAB, (plan.total_r,), generator=g).cuda()


def test_tree_loss_with_the_seam(mods):
    """tree_lm_loss through the kernels against the definition in 64 bits: the sum, and the gradients of the prompt states (the last
    one of a group is used once per branch), the response states and the head."""
    B, _, L = mods
    plan, _, tok = tree(B)
    g = torch.Generator().manual_seed(6)
    h_p, h_r = torch.randn(plan.total_p, HIDDEN, generator=g), torch.randn(plan.total_r, HIDDEN, generator=g)
    head = torch.randn(VOCAB, HIDDEN, generator=g) * HIDDEN ** -0.5
    tok = tok.clone()
    tok[7::11] = -100
    lm = B.LM(VOCAB, HIDDEN, device=0)
    leaves = [x.cuda().requires_grad_(True) for x in (h_p, h_r, head)]
    loss = L.tree_lm_loss(plan, *leaves, tok, lm=lm)
    loss.backward()
    from_prompt, index = (x.cpu() for x in L.seam_index(plan))
    src = torch.where(from_prompt[:, None], h_p[index.clamp(max=plan.total_p - 1)], h_r[index.clamp(max=plan.total_r - 1)])
    n = src.shape[0]
    ref = lu.loss_reference(src.to(BF16), head.to(BF16), tok.cpu(), torch.ones(n))
    b = lu.loss_bounds(ref, VOCAB, HIDDEN, n)
    assert abs(loss.item() - ref["loss"].sum().item()) <= b["loss"].sum().item() + n * 2.0 ** -24 * ref["loss"].sum().item()
    lu.assert_within(leaves[2].grad, ref["d_weight"], b["d_weight"], "head")
    for leaf, mask in ((leaves[0], from_prompt), (leaves[1], ~from_prompt)):
        # rows that several targets share are added up in bf16 or fp32 by autograd: one more rounding of the sum each
        want = torch.zeros(leaf.shape, dtype=F64).index_add_(0, index[mask], ref["d_hidden"][mask])
        off = torch.zeros(leaf.shape, dtype=F64).index_add_(0, index[mask], b["d_hidden"][mask])
        mag = torch.zeros(leaf.shape, dtype=F64).index_add_(0, index[mask], ref["d_hidden"][mask].abs())
        lu.assert_within(leaf.grad, want, off + 2.0 ** -8 * 8 * (mag + off) * (torch.bincount(index[mask], minlength=leaf.shape[0]) > 1)[:, None], "states")


class TinyLM(torch.nn.Module):
    def __init__(self, L, tied):
        super().__init__()
        self.emb = torch.nn.Parameter(torch.randn(VOCAB, HIDDEN) * (HIDDEN ** -0.5 if tied else 0.5))
        self.layers = torch.nn.ModuleList([L.TreeDecoderLayer(HIDDEN, H_Q, H_KV, D, MLP) for _ in range(2)])
        self.norm = torch.nn.Parameter(torch.ones(HIDDEN))
        self.head = self.emb if tied else torch.nn.Parameter(torch.randn(VOCAB, HIDDEN) * HIDDEN ** -0.5)


def step(L, model, plan, ptok, rtok, lm, scale):
    pos_p, pos_r = L.tree_positions(plan)
    if lm is not None:
        x_p, x_r = L.tree_embed(lm, model.emb, ptok, rtok)
    else:
        x_p, x_r = model.emb[ptok] * scale, model.emb[rtok] * scale
    for layer in model.layers:
        x_p, x_r = layer(plan, x_p, x_r, pos_p, pos_r)
    return L.tree_lm_loss(plan, L.rms_norm(x_p, model.norm), L.rms_norm(x_r, model.norm), model.head, rtok, lm=lm)


@pytest.mark.parametrize("tied", [False, True])
def test_training_step_from_ids_to_gradients(mods, tied):
    """Loss and every weight gradient of a two-layer model on a tree with the vocabulary kernels at both ends, against the same
    model with torch's indexing, GEMM and cross entropy.  That side rounds logits (up to about 5, so by up to 2e-2, 2e-3 in the
    mean) and their gradients to bf16, which both reach every gradient below: 2e-2 relative L2, as between the two executions of the
    layer's own test."""
    B, _, L = mods
    plan, ptok, rtok = tree(B)
    torch.manual_seed(9)
    scale = 16.0 if tied else 1.0
    ours = TinyLM(L, tied).cuda()
    plain = copy.deepcopy(ours)
    lm = B.LM(VOCAB, HIDDEN, device=0, embed_scale=scale)
    a, b = step(L, ours, plan, ptok, rtok, lm, scale), step(L, plain, plan, ptok, rtok, None, scale)
    a.backward()
    b.backward()
    assert lm.device_status() == (0, 0) and plan.device_status() == (0, 0)
    assert abs(a.item() - b.item()) <= 2e-3 * abs(b.item())
    for (name, p), (_, q) in zip(ours.named_parameters(), plain.named_parameters()):
        rel = ((p.grad - q.grad).norm() / q.grad.norm()).item()
        assert rel <= 2e-2, (name, rel)


def test_score_then_train_then_score_in_one_run(mods):
    """The order of an update step: log-probabilities under the old weights, loss and gradients, an SGD step on the table in place, the
    log-probabilities again; single tokens and whole rows through the same handle."""
    B, A, _ = mods
    h, w, y, a = lu.make_loss(260, 900, 96, seed=12, masked=0.1)
    lm = B.LM(900, 96, device=0)
    hc, yc, ac = h.cuda(), y.cuda(), a.cuda()
    wc = w.cuda().requires_grad_(True)
    for _ in range(2):
        with torch.no_grad():
            whole = A.lm_loss(lm, hc, wc, yc)
            singles = torch.cat([A.lm_loss(lm, hc[i:i + 1], wc, yc[i:i + 1]) for i in range(0, 260, 37)])
        ref = lu.loss_reference(h, wc.detach().cpu(), y, a)
        b = lu.loss_bounds(ref, 900, 96, 260)
        lu.assert_within(whole, ref["loss"], b["loss"], "whole")
        lu.assert_within(singles, ref["loss"][::37], b["loss"][::37], "singles")
        wc.grad = None
        (A.lm_loss(lm, hc, wc, yc) * ac).sum().backward()
        lu.assert_within(wc.grad, ref["d_weight"], b["d_weight"], "d_weight")
        with torch.no_grad():
            wc -= 0.01 * wc.grad

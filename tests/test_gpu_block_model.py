"""The block ends, checkpoints and gated MLP through autograd and through a stack of layers on a tree: gradients against differences, against the
same model in plain torch, with and without 8-bit checkpoints; the order of a training step."""
import copy

import pytest
import torch

from tests import block_util as bu

pytestmark = pytest.mark.gpu
F64, F32, BF16, U8 = torch.float64, torch.float32, torch.bfloat16, torch.uint8
HIDDEN, H_Q, H_KV, D, MLP, VOCAB = 256, 4, 2, 64, 512, 503


@pytest.fixture(scope="module")
def mods():
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import autograd, binding, layer
    return binding, autograd, layer


def leaf(shape, seed, scale=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda().requires_grad_(True)


@pytest.mark.parametrize("kind", ["none", "token", "channel", "full"])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_gradients_against_differences(mods, kind, sigmoid):
    """Everything in fp32.  Along a random direction v the loss changes by 2 t <grad, v> + O(t^3); with t = 2^-6 of directions of the inputs' own size
    the third-order term is t^2 = 2.4e-4 of the loss' curvature, whose size is that of the loss itself, and rounding adds 2^-24 |terms| / t = 4e-6 of
    the sum of magnitudes over its root count: within 2e-3 of (|grad| |v| / root(n) + |derivative|)."""
    B, A, _ = mods
    n, c = 24, 72
    blk = B.Block(c, device=0, eps=1e-5, residual_scale=0.7, gate=kind, gate_sigmoid=sigmoid)
    shape = {"token": (n,), "channel": (c,), "full": (n, c)}.get(kind)
    leaves = {"x": leaf((n, c), 1), "o": leaf((n, c), 2), "w_out": leaf((c,), 3), "w_in": leaf((c,), 4)}
    if shape:
        leaves["gate"] = leaf(shape, 5)
    cy, ch = leaf((n, c), 6).detach().double(), leaf((n, c), 7).detach().double()

    def loss(v):
        y, h, _ = A.block(blk, v["x"], v["o"], v.get("gate"), v["w_out"], v["w_in"], h_dtype=F32)
        return (y.double() * cy).sum() + (h.double() * ch).sum()
    loss(leaves).backward()
    for k, p in leaves.items():
        g = torch.Generator().manual_seed(11)
        v = torch.randn(p.shape, generator=g).cuda()
        t = 2.0 ** -6
        with torch.no_grad():
            up = loss({**leaves, k: p + t * v})
            down = loss({**leaves, k: p - t * v})
        d, want = ((up - down) / (2 * t)).item(), (p.grad.double() * v.double()).sum().item()
        size = (p.grad.norm() * v.norm()).item()
        assert abs(d - want) <= 2e-3 * (size / p.numel() ** 0.5 * 4 + abs(want)), (k, d, want, size)


def test_norm_and_glu_through_autograd(mods):
    B, A, _ = mods
    n, c, m = 50, 136, 264
    blk = B.Block(c, device=0, eps=1e-5)
    x, w = leaf((n, c), 1, dtype=BF16), leaf((c,), 2, dtype=BF16)
    dh = leaf((n, c), 3).detach().to(BF16)
    for ckpt in (False, True):
        x.grad = w.grad = None
        h, kept = A.norm(blk, x, w, ckpt=ckpt)
        h.backward(dh)
        v = x.detach().cpu()
        r = torch.rsqrt(v.double().pow(2).mean(1) + 1e-5)
        ref = bu.block_bwd(None, dh.cpu(), bu.in_8_bits(v) if ckpt else v, None, None, None, w.detach().cpu(), None, r.float(), kind="none", sigmoid=False, scale=1.0,
                           types={"x": BF16, "o": BF16, "w": BF16, "gate": BF16})
        # (r of the kernel is within 30 half steps of this one: 2e-6 of every term, far under the rounding to bf16)
        bu.check(x.grad, (ref["dx"][0], ref["dx"][1] + 1e-4 * ref["dx"][0].abs().max()), "dx")
        bu.check(w.grad, (ref["dw_in"][0], ref["dw_in"][1] + 1e-4 * ref["dw_in"][0].abs().max()), "dw")
        assert (kept is None) != ckpt
        g, u, wd = leaf((n, m), 5, dtype=BF16), leaf((n, m), 6, dtype=BF16), leaf((c, m), 7, 0.1, BF16)
        A.glu_linear(blk, g, u, wd, ckpt=ckpt).backward(dh)
        gs, us = (bu.in_8_bits(t.detach().cpu()) if ckpt else t.detach().cpu() for t in (g, u))
        da = (dh @ wd.detach()).cpu()
        ref = bu.glu(gs, us, da, BF16)
        bu.check(g.grad, ref["dg"], "dg")
        bu.check(u.grad, ref["du"], "du")
        a = ref["a"][0].to(BF16)
        want = dh.cpu().double().T @ a.double()
        mag = dh.cpu().double().abs().T @ a.double().abs()      # (a library product of bf16 operands; a may round to either neighbour: 2^-7)
        assert ((wd.grad.cpu().double() - want).abs() <= 2.0 ** -7 * mag + 2.0 ** -8 * want.abs() + 1e-6 * mag).all()


def test_linear_takes_its_gradient_from_the_checkpoint(mods):
    B, A, _ = mods
    n, c, out = 300, 264, 136
    blk = B.Block(c, device=0, eps=1e-5)
    x, w, weight, d = leaf((n, c), 1), leaf((c,), 2), leaf((out, c), 3, 0.1, BF16), leaf((n, out), 4).detach().to(BF16)
    h, kept = A.norm(blk, x, w, ckpt=True)
    y = A.linear(blk, h, weight, kept)
    assert torch.equal(y, torch.nn.functional.linear(h, weight))
    y.backward(d)
    val, bound = bu.wgrad(d.cpu(), bu.in_8_bits(x.detach().cpu()), kept.row.cpu(), w.detach().cpu(), BF16)
    bu.check(weight.grad, (val, bound))


def test_linear_with_a_transposed_weight(mods):
    B, A, _ = mods
    n, c, out = 70, 72, 136
    blk = B.Block(c, device=0)
    x, w, d = leaf((n, c), 1), leaf((c,), 2), leaf((n, out), 4).detach().to(BF16)
    base = leaf((c, out), 3, 0.1, BF16)
    h, kept = A.norm(blk, x, w, ckpt=True)
    A.linear(blk, h, base.t(), kept).backward(d)
    val, bound = bu.wgrad(d.cpu(), bu.in_8_bits(x.detach().cpu()), kept.row.cpu(), w.detach().cpu(), BF16)
    bu.check(base.grad.t(), (val, bound))


def test_a_norm_weight_changed_before_the_backward_pass_is_an_error(mods):
    B, A, _ = mods
    blk = B.Block(64, device=0)
    x, w, weight = leaf((5, 64), 1).detach(), leaf((64,), 2).detach(), leaf((72, 64), 3, dtype=BF16)
    h, kept = A.norm(blk, x, w, ckpt=True)      # (nothing of the norm wants a gradient: its own backward pass will not run)
    y = A.linear(blk, h, weight, kept)
    w.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.float().sum().backward()


def test_memory_kept_between_forward_and_backward(mods):
    """What a block end and a gated MLP keep: y and o in full (6 bytes a value), or two checkpoints (2.1)."""
    B, A, _ = mods
    n, c = 4096, 1024
    blk = B.Block(c, device=0)
    kept = []
    for ckpt in (False, True):
        x, o, w = leaf((n, c), 1), leaf((n, c), 2, dtype=BF16), leaf((c,), 3)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        y, h, k = A.block(blk, x, o.clone(), None, w, w, ckpt=ckpt)
        s = (y * 1.0).sum() * 0 + h.float().sum()
        del y, h, k
        kept.append(torch.cuda.memory_allocated() - before)
        s.backward()
        del x, o, w, s
    assert kept[0] >= 6 * n * c and kept[1] <= 2.2 * n * c + (1 << 20)


class Model(torch.nn.Module):
    def __init__(self, L, **kw):
        super().__init__()
        self.emb = torch.nn.Parameter(torch.randn(VOCAB, HIDDEN) * 0.5)
        self.layers = torch.nn.ModuleList([L.TreeDecoderLayer(HIDDEN, H_Q, H_KV, D, MLP, **kw) for _ in range(2)])
        self.norm = torch.nn.Parameter(1 + 0.1 * torch.randn(HIDDEN))
        self.head = torch.nn.Parameter(torch.randn(VOCAB, HIDDEN) * HIDDEN ** -0.5)
        for layer in self.layers:
            for p in (layer.norm1, layer.norm2, layer.post1, layer.post2, layer.scale1, layer.scale2):
                if p is not None:
                    p.data.mul_(1 + 0.1 * torch.randn(HIDDEN))


def tree(B):
    prompt, branch = [70, 33], [[40, 17], [25, 60, 1]]
    plan = B.Plan(prompt, branch, H_Q, H_KV, D, device=0)
    g = torch.Generator().manual_seed(5)
    tok = lambda n: torch.randint(0, VOCAB, (n,), generator=g).cuda()
    return plan, tok(plan.total_p), tok(plan.total_r)


def step(L, model, plan, ptok, rtok, blk=None, ckpt=False, lm=None):
    pos_p, pos_r = L.tree_positions(plan)
    if lm is not None:
        x_p, x_r = L.tree_embed(lm, model.emb, ptok, rtok)
    else:
        x_p, x_r = model.emb[ptok], model.emb[rtok]
    if blk is not None:
        h_p, h_r = L.tree_stack(blk, model.layers, plan, x_p, x_r, pos_p, pos_r, model.norm, ckpt=ckpt)
    else:
        for layer in model.layers:
            x_p, x_r = layer(plan, x_p, x_r, pos_p, pos_r)
        h_p, h_r = L.rms_norm(x_p, model.norm), L.rms_norm(x_r, model.norm)
    return L.tree_lm_loss(plan, h_p, h_r, model.head, rtok, lm=lm)


@pytest.mark.parametrize("kw", [{}, dict(post_norm=True), dict(post_norm=True, layer_scale=0.5)])
@pytest.mark.parametrize("ckpt", [False, True])
def test_a_stack_of_layers_against_plain_torch(mods, kw, ckpt):
    """Loss and every weight gradient of a two-layer model.  Without checkpoints both sides round to bf16 in the same places but for the gradients inside
    a block end and the MLP's activation, as far apart as the two executions of the layer's own test: 2e-2 relative L2.  A checkpoint is off by a
    uniform error of up to half of 2^e: at most 1 / 127.5 / root 3 = 0.0045 of its group's largest value, which is 2 to 3 times the group's rms, so by
    0.014 of the tensor's norm at most; a gradient passes at most five of them on its way (two norms and what they add, the MLP) in each of two layers,
    with independent errors: root 10 x 0.014 = 0.044, beside the 2e-2."""
    B, _, L = mods
    plan, ptok, rtok = tree(B)
    torch.manual_seed(3)
    ours = Model(L, **kw).cuda()
    plain = copy.deepcopy(ours)
    blk = B.Block(HIDDEN, device=0, gate="channel" if "layer_scale" in kw else "none")
    a, b = step(L, ours, plan, ptok, rtok, blk, ckpt), step(L, plain, plan, ptok, rtok)
    a.backward()
    b.backward()
    assert blk.device_status() == (0, 0)
    assert abs(a.item() - b.item()) <= 2e-3 * abs(b.item())
    for (name, p), (_, q) in zip(ours.named_parameters(), plain.named_parameters()):
        rel = ((p.grad - q.grad).norm() / q.grad.norm()).item()
        assert rel <= (6.4e-2 if ckpt else 2e-2), (name, rel)


def test_a_training_step_with_all_handles(mods):
    """Embedding, stack with checkpoints, vocabulary loss, SGD: two steps run, gradients are finite and repeat to the bit."""
    B, _, L = mods
    plan, ptok, rtok = tree(B)
    torch.manual_seed(4)
    model = Model(L).cuda()
    blk, lm = B.Block(HIDDEN, device=0), B.LM(VOCAB, HIDDEN, device=0)
    for _ in range(2):
        grads = []
        for _ in range(2):
            model.zero_grad(set_to_none=True)
            step(L, model, plan, ptok, rtok, blk, True, lm).backward()
            grads.append({k: p.grad.clone() for k, p in model.named_parameters()})
        assert all(torch.isfinite(g).all() and torch.equal(g, grads[1][k]) for k, g in grads[0].items())
        with torch.no_grad():
            for p in model.parameters():
                p -= 1e-3 * p.grad
    assert blk.device_status() == (0, 0) and lm.device_status() == (0, 0)


def test_prompts_without_responses(mods):
    """A plan with no response tokens: empty tensors through the stack."""
    B, _, L = mods
    plan = B.Plan([40, 9], [[], []], H_Q, H_KV, D, device=0)
    torch.manual_seed(6)
    model = Model(L).cuda()
    blk = B.Block(HIDDEN, device=0)
    pos_p, pos_r = L.tree_positions(plan)
    x_p = model.emb[torch.arange(49, device="cuda")]
    h_p, h_r = L.tree_stack(blk, model.layers, plan, x_p, x_p[:0], pos_p, pos_r, model.norm, ckpt=True)
    h_p.float().pow(2).sum().backward()
    assert h_r.shape == (0, HIDDEN) and all(torch.isfinite(p.grad).all() for p in model.layers.parameters())


def test_a_captured_backward_pass_beside_an_eager_graph(mods):
    """The gradients of leaves whose eager backward pass has run, and whose eager graph still lives, captured and replayed."""
    B, A, _ = mods
    n, c = 60, 264
    blk = B.Block(c, device=0)
    x, o, w, wt, d = leaf((n, c), 1), leaf((n, c), 2, dtype=BF16), leaf((c,), 3), leaf((72, c), 4, 0.1, BF16), leaf((n, 72), 5).detach().to(BF16)

    def loss():
        y, h, kept = A.block(blk, x, o, None, w, w, ckpt=True)
        z = A.linear(blk, h, wt, kept)
        return (z * d).sum().float() + A.glu(blk, h, h, ckpt=True).float().sum() + y.sum()
    leaves = (x, o, w, wt)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        eager = loss()
        want = torch.autograd.grad(eager, leaves, retain_graph=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = torch.autograd.grad(loss(), leaves)
    again = torch.autograd.grad(eager, leaves)
    for z in got:
        z.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(got, want, again))


def test_refusals_through_autograd(mods):
    B, A, _ = mods
    blk = B.Block(64, device=0)
    x, w = leaf((4, 64), 1), leaf((64,), 2)
    with pytest.raises(ValueError):
        A.norm(blk, x.t(), w)
    with pytest.raises(ValueError):
        A.norm(blk, x, w.to(BF16)[:32])
    with pytest.raises(ValueError):
        A.block(blk, x, x, x, None, w)       # a gate for a handle without one
    with pytest.raises(ValueError):
        A.glu(blk, x, x.to(BF16))

"""Block ends, 8-bit checkpoints and the weight gradient where a type, a size or a hand-over reaches its limit."""
import pytest
import torch

from tests import block_util as bu

pytestmark = pytest.mark.gpu
F64, F32, BF16, F16, U8 = torch.float64, torch.float32, torch.bfloat16, torch.float16, torch.uint8


@pytest.fixture(scope="module")
def B():
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import binding
    return binding


@pytest.mark.parametrize("n,out,c", [(129, 256, 256), (64, 520, 1032), (2183, 512, 136), (4096, 512, 1024)])
def test_a_weight_gradient_of_whole_numbers_is_exact(B, n, out, c):
    """From the bits (no bf16 copy in the scratch): both CTAs of a pair write operands for one MMA.  Integers whose sums stay below 2^24 leave nothing to round, so a
    stale byte anywhere shows; 40 calls behind one another, each with other inputs."""
    blk = B.Block(64, device=0)
    size = blk.wgrad_workspace_bytes(n, out, c)
    assert size < n * c * 2 or (size - 256) % (-(-out // 256) * 256 * c * 4) == 0
    ws, ckpt = torch.empty(size, device="cuda", dtype=U8), torch.empty((n, B.ckpt_pitch(c)), device="cuda", dtype=U8)
    gen = torch.Generator(device="cuda").manual_seed(n)
    draw = lambda shape, top: torch.randint(-top, top + 1, shape, generator=gen, device="cuda")
    for _ in range(40):
        x, dy = draw((n, c), 100), draw((n, out), 9)
        x[:, ::32] = 100                          # a group's largest magnitude is 100: its power of two is 2^0
        dw = torch.full((out, c), float("nan"), device="cuda")
        blk.pack(x.float(), ckpt)
        blk.wgrad(dy.to(BF16), ckpt, dw, ws)
        assert torch.equal(dw.double(), dy.double().t() @ x.double())
    assert blk.device_status() == (0, 0)


def test_memory_after_the_backward_pass_while_the_loss_is_held(B):
    """Checkpoints (2.1 bytes a value of a block end, the same again of a gated MLP) are gone as the uncheckpointed tensors are."""
    from paper_2609_33133_b200 import autograd as A
    n, c = 4096, 1024
    blk = B.Block(c, device=0)
    x = torch.randn(n, c, device="cuda").requires_grad_(True)
    o = torch.randn(n, c, device="cuda").to(BF16).requires_grad_(True)
    w, wt = torch.ones(c, device="cuda", requires_grad=True), torch.randn(c, c, device="cuda").mul_(0.03).to(BF16).requires_grad_(True)

    def loss(ckpt):
        _, h, kept = A.block(blk, x, o, None, w, w, ckpt=ckpt)
        return A.glu(blk, A.linear(blk, h, wt, kept), h, ckpt=ckpt).float().sum()
    for ckpt in (False, True):
        loss(ckpt).backward()              # (gradients of the leaves and the library's workspaces are there from here on)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        s = loss(ckpt)
        assert torch.cuda.memory_allocated() - before > 4 * n * c
        s.backward()
        assert torch.cuda.memory_allocated() - before <= 1 << 16, ckpt
        del s


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,lanes", [(32768, 2), (32769, 2), ((1 << 20) + 37, 2), ((1 << 20) + 37, 0)])
def test_a_weight_gradient_over_many_tokens_of_one_sign(B, n, lanes, dtype):
    """Two lanes: one share.  The tensor core's adder loses up to 2^-23 of its sum for every 16 tokens, always downwards: over 32768 tokens in one accumulator 2049 times; in
    pieces of 2048 tokens 128 times, and one rounding for each piece and share."""
    out, c = 64, 72
    gen = torch.Generator(device="cuda").manual_seed(n)
    rand = lambda *s: torch.rand(s, generator=gen, device="cuda")
    blk = B.Block(64, device=0, n_lanes=lanes)
    dy, x, col = ((0.5 + rand(n, out)) * (1 + rand(out))).to(BF16), 0.5 + rand(n, c), 1 + rand(c)     # (products spread over a factor of four: their roundings differ)
    ckpt, dw = torch.empty((n, B.ckpt_pitch(c)), device="cuda", dtype=U8), torch.full((out, c), float("nan"), device="cuda", dtype=dtype)
    blk.pack(x, ckpt)
    blk.wgrad(dy, ckpt, dw, torch.empty(blk.wgrad_workspace_bytes(n, out, c), device="cuda", dtype=U8), None, col)
    blk.unpack(ckpt, x)
    val = torch.zeros((out, c), device="cuda", dtype=F64)
    for i in range(0, n, 1 << 17):
        val += dy[i:i + (1 << 17)].double().t() @ x[i:i + (1 << 17)].double()
    val *= col.double()
    one = dtype is BF16 and n <= 32768 and lanes == 2
    adds = 2 * 2049 if one else 2 * 128 + n / 2048 + 40
    bu.check_delivered(dw, (val.cpu(), (adds + 4) * bu.U * val.cpu()))
    assert blk.device_status() == (0, 0)


@pytest.mark.parametrize("kind", ["full", "channel"])
@pytest.mark.parametrize("c", [8112, 8120, 8192])
@pytest.mark.parametrize("x_grad", [False, True])
def test_the_widest_rows_through_autograd(B, kind, c, x_grad):
    """Everything in fp32: from 8120 channels on the rows of all of the backward pass' inputs do not fit a CTA together.  r of the reference is a rounding of the 64-bit one, the
    kernel's is within 30 half steps of it, and every term of a gradient has at most three factors r: 100 half steps of the terms' sizes, which the largest gradient of a
    tensor bounds within a factor of ten."""
    from paper_2609_33133_b200 import autograd as A
    n, eps = 5, 1e-5
    gen = torch.Generator().manual_seed(c)
    leaf = lambda *s: torch.randn(s, generator=gen).cuda().requires_grad_(True)
    x, o, w_out, w_in, g = leaf(n, c), leaf(n, c), leaf(c), leaf(c), leaf(n, c) if kind == "full" else leaf(c)
    dy, dh = torch.randn(n, c, generator=gen).cuda(), torch.randn(n, c, generator=gen).cuda()
    blk = B.Block(c, device=0, eps=eps, residual_scale=0.7, gate=kind)
    y, h, _ = A.block(blk, x if x_grad else x.detach(), o, g, w_out, w_in, h_dtype=F32)
    torch.autograd.backward((y, h), (dy, dh))
    d = lambda t: t.detach().cpu()
    r = lambda t: torch.rsqrt(t.double().pow(2).mean(1) + eps).float()
    ref = bu.block_bwd(d(dy), d(dh), d(y), d(o), d(g), d(w_out), d(w_in), r(d(o)), r(d(y)), kind=kind, sigmoid=False, scale=0.7,
                       types={"x": F32, "o": F32, "w": F32, "gate": F32})
    assert (x.grad is not None) == x_grad
    for name, t in (("dx", x), ("d_o", o), ("d_gate", g), ("dw_out", w_out), ("dw_in", w_in)):
        val, bound = ref[name]
        if t.grad is not None:
            bu.check(t.grad, (val, bound + 1000 * bu.U * val.abs().max()), name)
    assert blk.device_status() == (0, 0)


def test_the_largest_values_stay_finite(B):
    """The power of two stops at 2^121: with 2^122 the integer 64 would stand for 2^128.  Integers stop at 127, so that a finite value never reads as an infinity; either
    side of the border, both signs, alone and beside zeros, small values and values that are the largest already."""
    top, border = torch.finfo(F32).max, 127.5 * 2.0 ** 121
    below = torch.nextafter(torch.tensor(border), torch.tensor(0.0)).item()
    x = torch.zeros(8, 96)
    x[0, :4] = torch.tensor([top, -top, 1.0, 2.0 ** 121 * 64.5])
    x[1, 32] = border
    x[2, 31], x[2, 32], x[2, 95] = -border, below, -below
    x[3] = torch.finfo(BF16).max
    x[4] = -torch.finfo(BF16).max
    x[5] = torch.linspace(-1, 1, 96) * top
    x[6, ::2], x[6, 5] = 2.0 ** 127, 2.0 ** 120
    x[7, 40], x[7, 70] = float("inf"), top

    def want(t):
        v = t.to(F64).view(8, 3, 32)
        bad = ~torch.isfinite(v).all(2, keepdim=True)
        _, byte = bu.encode(torch.where(bad.expand_as(v), 0.0, v).reshape(8, 96))
        e = (byte - 127).clamp(max=121)[:, :, None]
        return torch.where(bad, float("nan"), torch.round(v / torch.exp2(e)).clamp(-127, 127) * torch.exp2(e)).view(8, 96)
    blk = B.Block(96, device=0)
    for dtype in (F32, BF16):
        t = x.to(dtype) if dtype is F32 else x.clamp(-torch.finfo(BF16).max, torch.finfo(BF16).max).to(BF16)
        t[7, 40] = float("inf")
        ckpt = torch.full((8, B.ckpt_pitch(96)), 173, device="cuda", dtype=U8)
        blk.pack(t.cuda(), ckpt)
        for out in (torch.empty(8, 96, device="cuda"), torch.empty(8, 96, device="cuda", dtype=BF16)):
            blk.unpack(ckpt, out)
            assert torch.equal(out.cpu().double().nan_to_num(nan=7.0), want(t).nan_to_num(nan=7.0))
            assert torch.isfinite(out[:7]).all()
        # the block end and the gated MLP keep the same bytes
        z, h, fused = torch.zeros_like(t).cuda(), torch.empty(8, 96, device="cuda", dtype=BF16), torch.full_like(ckpt, 173)
        one = torch.ones(96, device="cuda")
        blk.fwd(t.cuda(), z.to(BF16), None, None, one, torch.empty_like(z), h, None, torch.empty(8, device="cuda"), fused, None)
        used = slice(0, 99)                # 96 integers, three exponents
        assert torch.equal(fused[:, used], ckpt[:, used])
        for k in (torch.full_like(ckpt, 173), torch.full_like(ckpt, 173)):
            blk.glu_fwd(t.cuda(), t.cuda(), torch.empty_like(z), fused, k)
            assert torch.equal(fused[:, used], ckpt[:, used]) and torch.equal(k[:, used], ckpt[:, used])
    assert blk.device_status() == (0, 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", [(40, 248), (700, 1032), (9, 8192)])
@pytest.mark.parametrize("branch", [False, True])
def test_block_ends_keep_the_largest_values_as_pack_does(B, dtype, n, c, branch):
    """Rows with groups at the end of the range among ordinary ones: the fused checkpoints of y and of o are those of pack to the byte, and read as finite values."""
    gen = torch.Generator(device="cuda").manual_seed(c)
    draw = lambda t: torch.randn(n, c, generator=gen, device="cuda").to(t)
    big = lambda t: torch.where(torch.rand(n, c, generator=gen, device="cuda") < 0.002, torch.finfo(t).max * torch.randn(n, c, generator=gen, device="cuda").sign(), draw(F32)).to(t)
    blk = B.Block(c, device=0, residual_scale=1e-30)
    new = lambda: torch.full((n, B.ckpt_pitch(c)), 173, device="cuda", dtype=U8)
    x, o, one = big(dtype), big(BF16) if branch else None, torch.ones(c, device="cuda")
    y, h, r = torch.empty_like(x) if branch else None, torch.empty(n, c, device="cuda", dtype=BF16), torch.empty(n, device="cuda")
    for w_out in (None, one) if branch else (None,):
        ky, ko = new(), new() if branch else None
        blk.fwd(x, o, None, w_out, one, y, h, None, r, ky, ko)
        at = -(-c // 16) * 16
        for kept, t in ((ky, y if branch else x), (ko, o)):
            if t is None:
                continue
            same, out = new(), torch.empty(n, c, device="cuda")
            blk.pack(t, same)
            blk.unpack(kept, out)
            assert torch.equal(kept[:, :c], same[:, :c]) and torch.equal(kept[:, at:at + -(-c // 32)], same[:, at:at + -(-c // 32)])
            assert (t.float().abs() == torch.finfo(t.dtype).max).any() and torch.isfinite(t).all() and torch.isfinite(out).all()
    assert blk.device_status() == (0, 0)


@pytest.mark.parametrize("n,out,c,lanes", [(1, 8, 8, 0), (65, 264, 200, 0), (129, 256, 512, 0), (743, 520, 1032, 0), (2183, 512, 136, 0), (5000, 72, 328, 0), (4160, 640, 576, 0),
                                           (700, 520, 328, 2), (2200, 72, 264, 2), (5000, 328, 520, 4)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_tokens_factor_rounds_the_operand_once(B, n, out, c, lanes, dtype):
    """From the bits (all lanes) and by way of bf16 scratch (few): against the very operand, so that the additions' bound alone is left."""
    blk = B.Block(64, device=0, n_lanes=lanes)
    gen = torch.Generator().manual_seed(n + c)
    randn = lambda *s: torch.randn(*s, generator=gen)
    dy, x, row, col = randn(n, out).to(BF16), (2 * randn(n, c) * torch.exp(0.5 * randn(c))).to(BF16), randn(n).abs() + 0.1, 1 + 0.2 * randn(c)
    ckpt, dw = torch.full((n, B.ckpt_pitch(c)), 173, device="cuda", dtype=U8), torch.full((out, c), float("nan"), device="cuda", dtype=dtype)
    blk.pack(x.cuda(), ckpt)
    ws = torch.empty(blk.wgrad_workspace_bytes(n, out, c), device="cuda", dtype=U8)
    for r, f in ((row, col), (row, None)):
        blk.wgrad(dy.cuda(), ckpt, dw, ws, r.cuda(), None if f is None else f.cuda())
        bu.check_delivered(dw, bu.wgrad_exact_operand(dy, bu.in_8_bits(x), r, f, dtype, chain=128 if dtype is F32 else n / 16 + 1))
    assert blk.device_status() == (0, 0)


@pytest.mark.parametrize("kind", ["token", "channel", "full"])
def test_saturated_gates_keep_a_gradient(B, kind):
    """Logits up to 80 either way: the slope e^-|g| / (1 + e^-|g|)^2 is within a relative error that grows with |g| alone (its exponent is rounded, 2^-24 |g| log2(e) and 2 units of
    2^x), like the gate's value for negative logits.  Everything in fp32, residual stream's gradient alone, so that d_gate = s dy o slope summed over what shares it."""
    n, c, scale = 64, 264, 0.7
    gen = torch.Generator().manual_seed(5)
    blk = B.Block(c, device=0, residual_scale=scale, gate=kind, gate_sigmoid=True)
    shape = {"token": (n,), "channel": (c,), "full": (n, c)}[kind]
    g = torch.linspace(-80, 80, torch.Size(shape).numel()).view(shape)
    dy, o = torch.randn(n, c, generator=gen).abs() + 0.1, torch.randn(n, c, generator=gen).abs() + 0.1      # (terms of one sign)
    d_o, d_gate = torch.empty(n, c, device="cuda"), torch.empty(shape, device="cuda")
    ws = torch.empty(blk.workspace_bytes(n), device="cuda", dtype=U8)
    blk.bwd(dy.cuda(), None, None, o.cuda(), g.cuda(), None, None, None, None, None, d_o, d_gate, None, None, ws)
    wide = g.double()
    wide = wide[:, None].expand(n, c) if kind == "token" else wide.expand(n, c)
    t = torch.exp(-wide.abs())
    a, slope = torch.where(wide < 0, t, torch.ones_like(t)) / (1 + t), t / (1 + t) ** 2
    rel = (4 * wide.abs() + 40) * bu.U
    term = scale * dy.double() * o.double() * slope
    chain = 0 if kind == "full" else 120
    off = (rel + chain * bu.U) * term
    if kind != "full":
        term, off = term.sum(1 if kind == "token" else 0), off.sum(1 if kind == "token" else 0)
    bu.check(d_gate, (term, off + 2.0 ** -149), "d_gate")
    v = scale * dy.double() * a
    bu.check(d_o, (v, rel * v + 2.0 ** -149), "d_o")
    assert blk.device_status() == (0, 0)

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

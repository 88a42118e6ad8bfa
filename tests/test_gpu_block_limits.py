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

"""Host side of the block ends and checkpoints: descriptor checks, sizes, refusals; no GPU."""
import ctypes as C

import pytest
import torch

from tests import block_util as bu

F32, BF16, U8 = torch.float32, torch.bfloat16, torch.uint8


@pytest.fixture(scope="module")
def B():
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import binding
    return binding


@pytest.mark.parametrize("kw,code", [
    (dict(hidden=0), -1), (dict(hidden=-8), -1), (dict(hidden=60), -2), (dict(hidden=8200), -2), (dict(hidden=64, n_lanes=0), -1),
    (dict(hidden=64, n_lanes=-1), -1), (dict(hidden=64, n_lanes=(1 << 20) + 1), -2), (dict(hidden=64, eps=-1.0), -1), (dict(hidden=64, eps=float("nan")), -1),
    (dict(hidden=64, residual_scale=float("inf")), -1)])
def test_descriptor_checks(B, kw, code):
    with pytest.raises(B.AugtreeError) as e:
        B.Block(**{"device": None, "n_lanes": 148, **kw})
    assert e.value.code == code


def test_python_checks(B):
    for kw in (dict(gate="half"), dict(eps=1e-60), dict(residual_scale=1e-60), dict(hidden=1 << 32), dict(flags=-1)):
        with pytest.raises(ValueError):
            B.Block(**{"hidden": 64, "device": None, "n_lanes": 148, **kw})


def test_bad_pointers_and_struct(B):
    h = C.c_void_p()
    assert B.lib.augtree_block_create(None, -1, C.byref(h)) == -1 and not h.value
    for size, version, gate in ((4, 1, 0), (C.sizeof(B.BlockDescC), 99, 0), (C.sizeof(B.BlockDescC), 1, 4), (C.sizeof(B.BlockDescC), 1, -1)):
        d = B.BlockDescC(size, version, 64, 0.0, 0.0, gate, 0, 0, 148)
        assert B.lib.augtree_block_create(C.byref(d), -1, C.byref(h)) == -1 and not h.value
    assert B.lib.augtree_block_destroy(None) == -1
    blk = B.Block(64, device=None, n_lanes=148)
    n, p = C.c_size_t(), C.c_int64()
    assert B.lib.augtree_block_workspace_bytes(blk._h, -1, C.byref(n)) == -1
    assert B.lib.augtree_block_workspace_bytes(blk._h, 1 << 31, C.byref(n)) == -2
    assert B.lib.augtree_block_workspace_bytes(blk._h, 1, None) == -1
    assert B.lib.augtree_ckpt_pitch(0, C.byref(p)) == -1 and B.lib.augtree_ckpt_pitch(12, C.byref(p)) == -2
    assert B.lib.augtree_ckpt_pitch((1 << 20) + 8, C.byref(p)) == -2 and B.lib.augtree_ckpt_pitch(8, None) == -1
    assert B.lib.augtree_ckpt_wgrad_bytes(blk._h, 10, 60, 64, C.byref(n)) == -2
    assert B.lib.augtree_ckpt_wgrad_bytes(blk._h, 10, 64, 0, C.byref(n)) == -1
    # launches on a host-only handle are refused before anything is touched
    z = None
    assert B.lib.augtree_block_fwd(blk._h, z, 0, z, 0, z, 0, z, z, 0, 1, z, z, 0, z, z, z, z, z) == -1
    assert B.lib.augtree_block_bwd(blk._h, z, 0, z, 0, z, 0, z, 0, z, 0, z, z, 0, z, z, 1, z, z, 0, z, z, z, 0, z, 0, z) == -1
    assert B.lib.augtree_ckpt_pack(blk._h, z, 0, 0, 1, 8, z, z) == -1
    assert B.lib.augtree_ckpt_unpack(blk._h, z, 1, 8, z, z, 0, z, 0, 0, z) == -1
    assert B.lib.augtree_glu_fwd(blk._h, z, z, 0, 0, 1, 8, z, z, z, z) == -1
    assert B.lib.augtree_glu_bwd(blk._h, z, 0, z, z, 0, 0, 1, 8, z, z, 0, z, z) == -1
    assert B.lib.augtree_ckpt_wgrad(blk._h, z, 1, 8, z, 8, z, z, 0, z, 0, 0, z, 0, z) == -1
    s = C.c_int()
    assert B.lib.augtree_block_last_device_status(blk._h, C.byref(s), None) == -1


@pytest.mark.parametrize("cols,pitch", [(8, 32), (16, 32), (24, 48), (512, 528), (520, 560), (3584, 3696), (18944, 19536)])
def test_pitch(B, cols, pitch):
    assert B.ckpt_pitch(cols) == pitch and pitch % 16 == 0 and pitch >= cols + -(-cols // 32)


def test_workspaces(B):
    blk = B.Block(3584, device=None, n_lanes=148)
    assert blk.workspace_bytes(0) == blk.workspace_bytes(1 << 20) == 148 * 2 * 3584 * 4
    x = 16384 * 3584 * 2
    assert x <= blk.wgrad_workspace_bytes(16384, 18944, 3584) <= x + 512       # many tiles: no shares, X once in bf16
    few = blk.wgrad_workspace_bytes(16384, 512, 512)                           # four tiles: shares of whole tiles in fp32
    assert few >= 2 * 512 * 512 * 4
    assert 0 < blk.wgrad_workspace_bytes(0, 64, 64) <= 512


def test_tensors_that_do_not_fit_are_named(B):
    blk = B.Block(64, device=None, n_lanes=148)
    x, one = torch.zeros(3, 64), torch.zeros(3)
    k = torch.zeros(3, B.ckpt_pitch(64), dtype=U8)
    for call in (lambda: blk.fwd(x, None, None, None, one, None, x, None, one), lambda: blk.fwd(None, None, None, None, None, None, None, None, None),
                 lambda: blk.fwd(3, None, None, None, None, None, None, None, None), lambda: blk.bwd(x, x, x, None, None, None, one, None, one, x, None, None, None, one, k),
                 lambda: blk.bwd(None, None, x, None, None, None, one, None, one, x, None, None, None, one, k), lambda: blk.pack(x, k), lambda: blk.unpack(k, x),
                 lambda: blk.pack(torch.zeros(3, 60), k), lambda: blk.glu_fwd(x, x, x), lambda: blk.glu_fwd(x, x, None), lambda: blk.glu_bwd(x, k, k, x, x),
                 lambda: blk.glu_bwd(x, None, None, x, x), lambda: blk.wgrad(x, k, x, k), lambda: blk.wgrad(x, k, None, k)):
        with pytest.raises(ValueError):
            call()


def test_the_plain_form_of_8_bits():
    """The border at which a group's exponent grows, ties, the smallest exponent, and the bound that the format promises."""
    x = torch.zeros(7, 32)
    x[0, :3] = torch.tensor([127.0, 0.5, 1.5])           # e = 0: ties to even
    x[1, 0] = 127.5                                       # one more
    x[2, 0] = torch.nextafter(torch.tensor(127.5), torch.tensor(0.0))
    x[3] = 1e-42
    x[4, 0], x[4, 1] = float("nan"), 3.0
    x[5, 31] = float("-inf")
    x[6] = torch.linspace(-1, 1, 32) * 3e38
    q, byte = bu.encode(x)
    assert byte[:, 0].tolist()[:4] == [127, 128, 127, 1] and byte[4, 0] == 255 and byte[5, 0] == 255
    assert q[0, :3].tolist() == [127, 0, 2] and q[1, 0] == 64 and q[2, 0] == 127 and q[3].abs().max() == 0
    v = bu.decode(q, byte, 32)
    assert v[4].isnan().all() and v[5].isnan().all()
    fine = [0, 1, 2, 3, 6]
    assert (q.abs().max(1).values[[0, 1, 2, 6]] >= 64).all() and q.abs().max() <= 127
    assert ((v - x.double()).abs() <= torch.exp2(byte - 128))[fine].all()
    # what it stands for fits bf16
    assert torch.equal(v[fine].to(F32).to(BF16).double(), v[fine])


def test_the_bounds_see_planted_mistakes():
    """A norm without eps, a swapped gate, a missing mean, a rounding too many, a dropped token: each is beyond the bounds of the plain form."""
    g = torch.Generator().manual_seed(3)
    n, c = 40, 72
    r = lambda *s: torch.randn(*s, generator=g)
    x, o, w_out, w_in, gate = r(n, c), (0.01 * r(n, c)).to(BF16), 1 + 0.2 * r(c), 1 + 0.2 * r(c), r(n)
    kw = dict(kind="token", sigmoid=True, scale=0.7, y_type=F32, h_type=F32)
    ref = bu.block_fwd(x, o, gate, w_out, w_in, eps=1e-5, **kw)
    for other in (bu.block_fwd(x, o, gate, w_out, w_in, eps=1e-6, **kw), bu.block_fwd(x, o, gate.flip(0), w_out, w_in, eps=1e-5, **kw),
                  bu.block_fwd(x.to(BF16), o, gate, w_out, w_in, eps=1e-5, **kw), bu.block_fwd(x, o, gate, w_in, w_out, eps=1e-5, **kw)):
        for k in ("y", "h"):
            with pytest.raises(AssertionError):
                bu.check(other[k][0], ref[k])
    y, r_i = ref["y"][0], ref["r_in"][0]
    r_o = ref["r_out"][0]
    dy, dh = r(n, c), r(n, c)
    kw = dict(kind="token", sigmoid=True, scale=0.7, types={"x": F32, "o": F32, "w": F32, "gate": F32})
    bw = bu.block_bwd(dy, dh, y, o, gate, w_out, w_in, r_o, r_i, **kw)
    for k, other in (("dx", bu.block_bwd(dy, dh, y, o, gate, w_out, w_in, r_o, 1.001 * r_i, **kw)), ("dx", bu.block_bwd(dy, dh.to(BF16), y, o, gate, w_out, w_in, r_o, r_i, **kw)),
                     ("d_o", bu.block_bwd(dy, dh, y, o.flip(1), gate, w_out, w_in, r_o, r_i, **kw)), ("d_gate", bu.block_bwd(dy, dh, y, o, 1.01 * gate, w_out, w_in, r_o, r_i, **kw)),
                     ("dw_in", bu.block_bwd(dy[1:], dh[1:], y[1:], o[1:], gate[1:], w_out, w_in, r_o[1:], r_i[1:], **kw))):
        with pytest.raises(AssertionError):
            bu.check(other[k][0], bw[k])
    a, b = r(100, 8).to(BF16), bu.in_8_bits(r(100, 16).to(BF16))
    want = bu.wgrad(a, b, None, None, F32)
    for off in (bu.wgrad(a[1:], b[1:], None, None, F32), bu.wgrad(a.flip(0), b, None, None, F32)):
        with pytest.raises(AssertionError):
            bu.check(off[0], want)
    u = bu.glu(r(n, c), r(n, c), dy, F32)
    with pytest.raises(AssertionError):
        bu.check(u["dg"][0] * 1.0001, u["dg"])

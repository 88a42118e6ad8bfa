"""Decoder block ends, 8-bit checkpoints, gated MLP and weight gradient against 64-bit plain forms."""
import pytest
import torch

from tests import block_util as bu

pytestmark = pytest.mark.gpu
F64, F32, BF16, F16, U8 = torch.float64, torch.float32, torch.bfloat16, torch.float16, torch.uint8
SCALE, EPS = 0.7, 1e-5


@pytest.fixture(scope="module")
def B():
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import binding
    return binding


def rand(shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    chan = torch.exp(0.5 * torch.randn(shape[-1:], generator=g))
    return (torch.randn(shape, generator=g) * chan * scale).to(dtype)


def cu(t):
    return None if t is None else t.cuda()


def e(shape, dtype):
    """An output that holds what no result leaves there."""
    t = torch.empty(shape, device="cuda", dtype=dtype)
    return t.fill_(173) if dtype is U8 else t.fill_(float("nan"))


class Case:
    """Inputs of one block end and the handle for it."""

    def __init__(self, B, n, c, *, x=F32, o=BF16, h=BF16, w=F32, kind="none", sigmoid=False, post=True, branch=True, gate=None, seed=0, flags=0):
        self.n, self.c, self.kind, self.sigmoid, self.branch = n, c, kind if branch else "none", sigmoid, branch
        self.x_t, self.o_t, self.h_t, self.w_t, self.g_t = x, o, h, w, gate or (w if kind == "channel" else o)
        self.x, self.w_in = rand((n, c), seed, x, 2.0), (1 + rand((c,), seed + 1, F32, 0.2)).to(w)
        self.o = rand((n, c), seed + 2, o) if branch else None
        self.w_out = (1 + rand((c,), seed + 3, F32, 0.2)).to(w) if branch and post else None
        shape = {"token": (n,), "channel": (c,), "full": (n, c)}.get(self.kind)
        self.g = None if shape is None else rand(shape, seed + 4, F32).clamp(-6, 6).to(self.g_t)
        self.dy, self.dh = rand((n, c), seed + 5, x, 0.3), rand((n, c), seed + 6, h, 0.3)
        self.blk = B.Block(c, device=0, eps=EPS, residual_scale=SCALE, gate=self.kind, gate_sigmoid=sigmoid, flags=flags)
        self.pitch = B.ckpt_pitch(c)

    def forward(self, ckpt=False):
        n, c = self.n, self.c
        out = {"h": e((n, c), self.h_t), "r_in": e((n,), F32)}
        if self.branch:
            out["y"] = e((n, c), self.x_t)
            if self.w_out is not None:
                out["r_out"] = e((n,), F32)
        if ckpt:
            out["ckpt_y"] = e((n, self.pitch), U8)
            out["ckpt_o"] = e((n, self.pitch), U8) if self.branch else None
        self.blk.fwd(cu(self.x), cu(self.o), cu(self.g), cu(self.w_out), cu(self.w_in), out.get("y"), out["h"], out.get("r_out"), out["r_in"],
                     out.get("ckpt_y"), out.get("ckpt_o"))
        return out

    def forward_ref(self):
        ref = bu.block_fwd(self.x, self.o, self.g, self.w_out, self.w_in, kind=self.kind, sigmoid=self.sigmoid, scale=SCALE, eps=EPS,
                           y_type=self.x_t, h_type=self.h_t)
        if self.w_out is None:
            ref.pop("r_out", None)
        return ref

    def backward(self, fw, y=None, o=None, accumulate=None, dy=True, dh=True):
        """y, o: what is handed over as saved tensors (default: in full)."""
        n, c = self.n, self.c
        y = (fw["y"] if self.branch else cu(self.x)) if y is None else y
        o = cu(self.o) if o is None else o
        out = {"dx": e((n, c), self.x_t)}
        if dh:
            out["dw_in"] = e((c,), self.w_t) if accumulate is None else accumulate["dw_in"].clone()
        if self.branch:
            out["d_o"] = e((n, c), self.o_t)
            if self.w_out is not None:
                out["dw_out"] = e((c,), self.w_t) if accumulate is None else accumulate["dw_out"].clone()
            if self.g is not None:
                out["d_gate"] = e(self.g.shape, self.g_t) if accumulate is None or self.kind != "channel" else accumulate["d_gate"].clone()
        ws = e((self.blk.workspace_bytes(n),), U8)
        self.blk.bwd(cu(self.dy) if dy else None, cu(self.dh) if dh else None, y if dh else None, o, cu(self.g), cu(self.w_out), cu(self.w_in) if dh else None,
                     fw.get("r_out"), fw["r_in"] if dh else None, out["dx"], out.get("d_o"), out.get("d_gate"), out.get("dw_out"), out.get("dw_in"), ws,
                     accumulate=accumulate is not None)
        return out

    def backward_ref(self, fw, y, o, dy=True, dh=True):
        c = lambda t: None if t is None else t.cpu()
        return bu.block_bwd(self.dy if dy else None, self.dh if dh else None, c(y), c(o), self.g, self.w_out, self.w_in, c(fw.get("r_out")),
                            c(fw["r_in"]), kind=self.kind, sigmoid=self.sigmoid, scale=SCALE,
                            types={"x": self.x_t, "o": self.o_t, "w": self.w_t, "gate": self.g_t})

    def check_all(self, ckpt):
        fw = self.forward(ckpt)
        for k, want in self.forward_ref().items():
            bu.check(fw[k], want, k)
        y, o = fw["y"] if self.branch else self.x, self.o
        if ckpt:
            # the 8-bit forms are those of the delivered y and of o, to the bit
            for name, t in (("ckpt_y", y), ("ckpt_o", o)):
                if t is None:
                    continue
                q, byte = bu.split(fw[name].cpu(), self.c)
                q0, byte0 = bu.encode(t.cpu())
                assert torch.equal(byte, byte0) and torch.equal(q, q0), name
            bw = self.backward(fw, fw["ckpt_y"], fw["ckpt_o"])
            ref = self.backward_ref(fw, bu.in_8_bits(y.cpu()), bu.in_8_bits(o) if o is not None else None)
        else:
            bw = self.backward(fw)
            ref = self.backward_ref(fw, y, o)
        assert set(ref) == set(bw)
        for k, want in ref.items():
            bu.check(bw[k], want, k)
        assert self.blk.device_status() == (0, 0)


# ------------------------------------------------------------------------------------------------ block ends
@pytest.mark.parametrize("n,c", [(1, 8), (3, 64), (37, 248), (743, 256), (5, 264), (300, 520), (149, 1032), (64, 2000), (200, 3584), (2, 7680),
                                 (9, 7688), (33, 8192), (2183, 72), (5001, 256)])
@pytest.mark.parametrize("ckpt", [False, True])
def test_sizes(B, n, c, ckpt):
    Case(B, n, c, kind="token", sigmoid=True, seed=n + c).check_all(ckpt)


@pytest.mark.parametrize("kind,sigmoid", [("none", False)] + [(k, s) for k in ("token", "channel", "full") for s in (False, True)])
@pytest.mark.parametrize("post", [False, True])
def test_gates(B, kind, sigmoid, post):
    for ckpt in (False, True):
        Case(B, 77, 1032, kind=kind, sigmoid=sigmoid, post=post, seed=7).check_all(ckpt)


@pytest.mark.parametrize("x,o,h,w,gate", [(F32, F32, F32, F32, F32), (BF16, BF16, BF16, BF16, BF16), (F16, F16, F16, F16, F16), (F32, F16, BF16, BF16, F32),
                                          (BF16, F32, F16, F32, F16), (F16, BF16, F32, BF16, BF16)])
@pytest.mark.parametrize("kind", ["full", "channel"])
def test_types(B, x, o, h, w, gate, kind):
    for ckpt in (False, True):
        Case(B, 65, 328, x=x, o=o, h=h, w=w, gate=gate, kind=kind, sigmoid=True, seed=3).check_all(ckpt)


@pytest.mark.parametrize("n,c", [(1, 3584), (129, 256), (300, 1032)])
@pytest.mark.parametrize("ckpt", [False, True])
def test_norm_before_a_block_alone(B, n, c, ckpt):
    Case(B, n, c, branch=False, seed=11).check_all(ckpt)


def test_block_end_without_a_norm_before_the_next(B):
    s = Case(B, 50, 264, kind="full", seed=5)
    y, r = e((50, 264), F32), e((50,), F32)
    s.blk.fwd(cu(s.x), cu(s.o), cu(s.g), cu(s.w_out), None, y, None, r, None)
    ref = s.forward_ref()
    bu.check(y, ref["y"], "y")
    fw = {"y": y, "r_out": r, "r_in": None}
    bw = s.backward(fw, dh=False)
    want = bu.block_bwd(s.dy, None, None, s.o, s.g, s.w_out, None, r.cpu(), None, kind="full", sigmoid=False, scale=SCALE,
                        types={"x": F32, "o": BF16, "w": F32, "gate": BF16})
    assert set(want) == set(bw)
    for k in want:
        bu.check(bw[k], want[k], k)


def test_gradient_of_h_alone(B):
    s = Case(B, 50, 264, seed=6)
    fw = s.forward()
    bw = s.backward(fw, dy=False)
    for k, want in s.backward_ref(fw, fw["y"], s.o, dy=False).items():
        bu.check(bw[k], want, k)


# ------------------------------------------------------------------------------------------------ 8 bits
def odd_values():
    """Groups at the format's borders: zeros, subnormal and largest numbers, halves of a step, the border 127.5, NaN and infinities."""
    rows = [torch.zeros(32), torch.full((32,), 1e-45), torch.full((32,), 3e38), torch.arange(32) - 15.5, torch.full((32,), 127.5),
            torch.tensor([127.49999] + [0.5] * 31), torch.tensor([63.75] + [0.25, 0.75, -0.25, -0.75] * 7 + [1.0] * 3),
            torch.tensor([float("nan")] + [1.0] * 31), torch.tensor([1.0] * 31 + [float("inf")]), torch.tensor([-float("inf")] + [0.0] * 31),
            torch.tensor([2.0 ** -126] * 32), torch.tensor([2.0 ** -120 * 127.5] + [2.0 ** -127] * 31), torch.tensor([1e-30, -1e-30] * 16)]
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,c", [(1, 8), (13, 32), (3, 40), (129, 1032), (1000, 256), (7, 3584)])
def test_pack_and_unpack(B, dtype, n, c):
    blk = B.Block(64, device=0)
    x = (rand((n, c), n + c, F32) * torch.exp(3 * torch.randn(n, 1, generator=torch.Generator().manual_seed(n)))).to(dtype)
    if (n, c) == (13, 32):
        x = odd_values().to(dtype)
    ckpt = e((n, B.ckpt_pitch(c)), U8)
    blk.pack(cu(x), ckpt)
    q, byte = bu.split(ckpt.cpu(), c)
    q0, byte0 = bu.encode(x)
    fine = (byte0 != 255).repeat_interleave(32, 1)[:, :c]
    assert torch.equal(byte, byte0) and torch.equal(q[fine], q0[fine])
    for out_t in (F32, BF16, F16):
        out = e((n, c), out_t)
        blk.unpack(ckpt, out)
        want = bu.decode(q0, byte0, c).to(F32).to(out_t)      # (fp32 holds the values)
        assert torch.equal(out.cpu().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0)), out_t
    fin = torch.isfinite(x.double()) & fine
    half = torch.exp2(byte0 - 128).repeat_interleave(32, 1)[:, :c]
    assert ((bu.decode(q0, byte0, c) - x.double()).abs() <= half)[fin].all()


def test_pack_and_unpack_with_leading_sizes_and_factors(B):
    blk = B.Block(64, device=0)
    n, c = 61, 200
    wide = rand((n, 3 * c), 1, BF16).cuda()
    ckpt, flat = e((n, B.ckpt_pitch(c)), U8), e((n, B.ckpt_pitch(c)), U8)
    blk.pack(wide[:, c:2 * c], ckpt)
    blk.pack(wide[:, c:2 * c].contiguous(), flat)
    q, byte = bu.split(ckpt.cpu(), c)
    q0, byte0 = bu.split(flat.cpu(), c)
    assert torch.equal(q, q0) and torch.equal(byte, byte0)
    row, col = rand((n,), 2), rand((c,), 3, BF16)
    out = e((n, 3 * c), F32)
    blk.unpack(ckpt, out[:, c:2 * c], cu(row), cu(col))
    want = bu.decode(q, byte, c) * row.double()[:, None] * col.double()
    bu.check(out[:, c:2 * c], (want, 3 * bu.U * want.abs()))
    assert out[:, :c].isnan().all() and out[:, 2 * c:].isnan().all()


# ------------------------------------------------------------------------------------------------ gated MLP
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n,c", [(1, 8), (5, 40), (743, 512), (33, 1032), (3, 18944)])
@pytest.mark.parametrize("ckpt", [False, True])
def test_glu(B, dtype, n, c, ckpt):
    blk = B.Block(64, device=0)
    g, u, da = rand((n, c), 1, F32, 2.0).to(dtype), rand((n, c), 2, dtype), rand((n, c), 3, dtype)
    a, again, dg, du = (e((n, c), dtype) for _ in range(4))
    boxes = [e((n, B.ckpt_pitch(c)), U8) for _ in range(2)] if ckpt else [None, None]
    blk.glu_fwd(cu(g), cu(u), a, *boxes)
    bu.check(a, bu.glu(g, u, da, dtype)["a"], "a")
    if ckpt:
        for box, t in zip(boxes, (g, u)):
            q, byte = bu.split(box.cpu(), c)
            q0, byte0 = bu.encode(t)
            assert torch.equal(q, q0) and torch.equal(byte, byte0)
        blk.glu_bwd(cu(da), *boxes, dg, du, again)
        g, u = bu.in_8_bits(g), bu.in_8_bits(u)
    else:
        blk.glu_bwd(cu(da), cu(g), cu(u), dg, du, again)
    ref = bu.glu(g, u, da, dtype)
    bu.check(again, ref["a"], "a again")
    bu.check(dg, ref["dg"], "dg")
    bu.check(du, ref["du"], "du")


def test_glu_halves_of_one_product(B):
    blk = B.Block(64, device=0)
    n, c = 37, 136
    gu, da = rand((n, 2 * c), 1, BF16).cuda(), rand((n, c), 3, BF16).cuda()
    a, d_gu = e((n, c), BF16), e((n, 2 * c), BF16)
    blk.glu_fwd(gu[:, :c], gu[:, c:], a)
    blk.glu_bwd(da, gu[:, :c], gu[:, c:], d_gu[:, :c], d_gu[:, c:])
    ref = bu.glu(gu[:, :c].cpu(), gu[:, c:].cpu(), da.cpu(), BF16)
    bu.check(a, ref["a"])
    bu.check(d_gu[:, :c], ref["dg"])
    bu.check(d_gu[:, c:], ref["du"])


# ------------------------------------------------------------------------------------------------ weight gradient
@pytest.mark.parametrize("n,out,c,lanes", [(1, 8, 8, 0), (63, 64, 64, 0), (64, 256, 256, 0), (65, 264, 200, 0), (129, 256, 512, 0), (743, 520, 1032, 0), (2183, 512, 136, 0),
                                           (5000, 72, 328, 0), (4160, 640, 576, 0), (700, 520, 328, 2), (1000, 328, 520, 4), (2200, 72, 264, 2), (2049, 512, 512, 4)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("factors", [False, True])
def test_wgrad(B, n, out, c, lanes, dtype, factors):
    """Few lanes: many tiles a CTA pair, the operand by way of bf16 scratch; all lanes: from the bits."""
    blk = B.Block(64, device=0, n_lanes=lanes)
    if lanes:
        assert blk.wgrad_workspace_bytes(n, out, c) == -(-n * -(-c // 64) * 128 // 256) * 256 + 256      # a bf16 copy, no shares
    dy, x = rand((n, out), 1, BF16), rand((n, c), 2, BF16, 2.0)
    row, col = (rand((n,), 3).abs() + 0.1, rand((c,), 4, F32)) if factors else (None, None)
    ckpt, dw = e((n, B.ckpt_pitch(c)), U8), e((out, c), dtype)
    ws = e((blk.wgrad_workspace_bytes(n, out, c),), U8)
    blk.pack(cu(x), ckpt)
    blk.wgrad(cu(dy), ckpt, dw, ws, cu(row), cu(col))
    want = bu.wgrad(dy, bu.in_8_bits(x), row, col, dtype)
    bu.check(dw, want)
    if dtype is F32:
        before = rand((out, c), 5).cuda()
        acc = before.clone()
        blk.wgrad(cu(dy), ckpt, acc, ws, cu(row), cu(col), accumulate=True)
        bu.check(acc, (want[0] + before.cpu().double(), want[1] + bu.U * (want[0] + before.cpu().double()).abs()))
    assert blk.device_status() == (0, 0)

"""Block ends, checkpoints, gated MLP and weight gradient where calls go wrong: no tokens, rows that hold NaN, what lies behind the last row, aliases,
alignment, streams, captured graphs, large offsets, refusals, waits that run out."""
import pytest
import torch

from tests import block_util as bu
from tests.test_gpu_block import Case, cu, e, rand

pytestmark = pytest.mark.gpu
F64, F32, BF16, F16, U8 = torch.float64, torch.float32, torch.bfloat16, torch.float16, torch.uint8


@pytest.fixture(scope="module")
def B():
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import binding
    return binding


def same(a, b):
    """Equal bits (NaN like NaN)."""
    assert set(a) == set(b)
    for k in a:
        if a[k] is not None:
            assert torch.equal(a[k].view(U8), b[k].view(U8)), k


def known(out, s):
    """Forward outputs without the bytes of a checkpoint that are not defined."""
    return {k: v if v is None or v.dtype is not U8 else torch.cat([t for t in bu.split(v.cpu(), s.c)], 1) for k, v in out.items()}


# ------------------------------------------------------------------------------------------------ sizes
@pytest.mark.parametrize("kind", ["none", "channel"])
def test_no_tokens(B, kind):
    s = Case(B, 0, 264, kind=kind, seed=1)
    fw = s.forward(ckpt=True)
    assert fw["h"].shape == (0, 264)
    bw = s.backward(fw)
    assert (bw["dw_in"] == 0).all() and (bw["dw_out"] == 0).all() and (kind == "none" or (bw["d_gate"] == 0).all())
    before = {k: rand((264,), 2).cuda() for k in ("dw_in", "dw_out", "d_gate")}
    after = s.backward(fw, accumulate=before)
    assert all(torch.equal(after[k], before[k]) for k in ("dw_in", "dw_out"))
    k, x = e((0, B.ckpt_pitch(264)), U8), e((0, 264), BF16)
    s.blk.pack(x, k), s.blk.unpack(k, x), s.blk.glu_fwd(x, x, x), s.blk.glu_bwd(x, k, k, x, x, x)
    dw, ws = e((40, 264), F32), e((s.blk.wgrad_workspace_bytes(0, 40, 264) + 1,), U8)
    s.blk.wgrad(e((0, 40), BF16), k, dw, ws)
    assert (dw == 0).all()
    s.blk.wgrad(e((0, 40), BF16), k, dw.fill_(3.0), ws, accumulate=True)
    assert (dw == 3).all()


@pytest.mark.parametrize("lanes", [1, 3, 1000])
@pytest.mark.parametrize("n,c", [(70, 264), (1000, 72)])
def test_lane_counts(B, lanes, n, c):
    """Few persistent CTAs, or more than the device has: the same rows; sums over tokens within their bounds (chains of n / lanes)."""
    s = Case(B, n, c, kind="channel", sigmoid=True, seed=4)
    want = s.forward(ckpt=True)
    s.blk = B.Block(c, device=0, eps=1e-5, residual_scale=0.7, gate="channel", gate_sigmoid=True, n_lanes=lanes)
    fw = s.forward(ckpt=True)
    same(known(fw, s), known(want, s))
    bw = s.backward(fw)
    c_ = lambda t: t.cpu()
    ref = bu.block_bwd(s.dy, s.dh, c_(fw["y"]), s.o, s.g, s.w_out, s.w_in, c_(fw["r_out"]), c_(fw["r_in"]), kind="channel", sigmoid=True, scale=0.7,
                       types={"x": F32, "o": BF16, "w": F32, "gate": F32}, lanes=min(lanes, 148))
    for k, v in ref.items():
        bu.check(bw[k], v, k)


def test_more_than_two_to_the_31_elements(B):
    """Offsets beyond 32 bits, forward and backward: the last rows are those of a small call on them."""
    n, c, tail = 600_000, 3584, 64
    assert n * c > 1 << 31
    blk = B.Block(c, device=0)
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda: torch.randn(4096, c, device="cuda", generator=g).to(BF16).repeat(n // 4096 + 1, 1)[:n]
    x, o, w = r(), r(), (1 + 0.2 * torch.randn(c, device="cuda", generator=g)).to(BF16)
    ky, ko = torch.empty(n, B.ckpt_pitch(c), device="cuda", dtype=U8), torch.empty(n, B.ckpt_pitch(c), device="cuda", dtype=U8)
    y, h, r_o, r_i = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    blk.fwd(x, o, None, w, w, y, h, r_o, r_i, ky, ko)
    t = slice(n - tail, n)
    small = [torch.empty_like(z[t]) for z in (y, h, r_o, r_i, ky, ko)]
    blk.fwd(x[t].clone(), o[t].clone(), None, w, w, *small)
    for a, b in zip((y, h, r_o, r_i), small):
        assert torch.equal(a[t], b)
    for a, b in zip((ky, ko), small[4:]):
        assert all(torch.equal(p, q) for p, q in zip(bu.split(a[t].cpu(), c), bu.split(b.cpu(), c)))
    dw, ws = torch.empty_like(w), torch.empty(blk.workspace_bytes(n), device="cuda", dtype=U8)
    dx, d_o, more = torch.empty_like(x), torch.empty_like(x), [torch.empty_like(x[t]) for _ in range(2)]
    blk.bwd(x, o, ky, ko, None, w, w, r_o, r_i, dx, d_o, None, dw.clone(), dw, ws)
    blk.bwd(x[t].clone(), o[t].clone(), ky[t].clone(), ko[t].clone(), None, w, w, r_o[t].clone(), r_i[t].clone(), *more, None, dw.clone(), dw.clone(), ws)
    assert torch.equal(dx[t], more[0]) and torch.equal(d_o[t], more[1])
    blk.glu_fwd(x, o, y, ky, ko)
    blk.glu_fwd(x[t].clone(), o[t].clone(), small[0], small[4], small[5])
    assert torch.equal(y[t], small[0]) and all(torch.equal(p, q) for p, q in zip(bu.split(ko[t].cpu(), c), bu.split(small[5].cpu(), c)))
    blk.glu_bwd(h, ky, ko, dx, d_o)
    blk.glu_bwd(h[t].clone(), small[4], small[5], *more)
    assert torch.equal(dx[t], more[0]) and torch.equal(d_o[t], more[1])
    blk.unpack(ky, y)
    blk.unpack(small[4], small[0])
    assert torch.equal(y[t], small[0])
    # the weight gradient: nothing but the last tokens count, and n is a multiple of a stage's 64, so they meet in the same order
    x[: n - tail] = 0
    k, dw = torch.empty(n, B.ckpt_pitch(64), device="cuda", dtype=U8), [torch.empty(c, 64, device="cuda") for _ in range(2)]
    blk.pack(o[:, :64], k)
    for m, out in ((n, dw[0]), (tail, dw[1])):
        blk.wgrad(x[n - m:].clone(), k[n - m:].clone(), out, torch.empty(blk.wgrad_workspace_bytes(m, c, 64), device="cuda", dtype=U8))
    assert (dw[1] != 0).any() and torch.equal(*dw)
    assert blk.device_status() == (0, 0)


# ------------------------------------------------------------------------------------------------ values
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
def test_rows_do_not_touch_each_other(B, ckpt, bad):
    """A row that overflows or holds NaN spoils its own results and the sums over tokens, no other row."""
    s = Case(B, 75, 520, kind="full", seed=8)
    clean_f = s.forward(ckpt)
    saved = (lambda f: (f["ckpt_y"], f["ckpt_o"])) if ckpt else (lambda f: (None, None))
    clean_b = s.backward(clean_f, *saved(clean_f))
    s.x[31, 100], s.dh[40, 3] = bad, float("nan")
    fw = s.forward(ckpt)
    bw = s.backward(fw, *saved(fw))
    rows = [i for i in range(75) if i not in (31, 40)]
    for k in ("y", "h", "r_in", "r_out"):
        assert torch.equal(fw[k][rows], clean_f[k][rows]), k
    for k in ("dx", "d_o", "d_gate"):
        assert torch.equal(bw[k][rows], clean_b[k][rows]), k
    assert not torch.isfinite(bw["dx"][40]).all()
    if ckpt and bad != 3e38:
        q, byte = bu.split(fw["ckpt_y"].cpu(), 520)
        assert byte[31, 3] == 255 and (byte[31] != 255).sum() == 16     # the group that holds it, and that one alone


def test_zero_and_constant_rows(B):
    """A row of zeros has the reciprocal root of eps; gradients stay finite."""
    s = Case(B, 20, 264, kind="token", seed=9)
    s.x[3], s.o[3], s.o[5], s.g[7], s.dy[9], s.dh[9] = 0.0, 0.0, 0.0, 0.0, 0.0, 0.0
    s.check_all(False)
    s.check_all(True)


# ------------------------------------------------------------------------------------------------ memory
def guarded(shape, dtype, rows=3):
    """A buffer with rows behind it, filled with a pattern."""
    t = torch.empty((shape[0] + rows, *shape[1:]), device="cuda", dtype=dtype)
    t.view(U8).fill_(0x5a)
    return t


@pytest.mark.parametrize("n,c", [(61, 264), (150, 1032), (1, 72)])
def test_rows_behind_the_last_one_stay(B, n, c):
    s = Case(B, n, c, kind="full", seed=10)
    big = {k: guarded(sh, dt) for k, sh, dt in (("y", (n, c), F32), ("h", (n, c), BF16), ("r_o", (n,), F32), ("r_i", (n,), F32), ("ky", (n, s.pitch), U8),
                                               ("ko", (n, s.pitch), U8), ("dx", (n, c), F32), ("do", (n, c), BF16), ("dg", (n, c), BF16), ("a", (n, c), BF16),
                                               ("dwo", (c,), F32), ("dwi", (c,), F32), ("dw", (c, c), F32))}
    v = {k: t[: t.shape[0] - 3] for k, t in big.items()}
    x, o, g, wo, wi, dy, dh = (cu(t) for t in (s.x, s.o, s.g, s.w_out, s.w_in, s.dy, s.dh))
    s.blk.fwd(x, o, g, wo, wi, v["y"], v["h"], v["r_o"], v["r_i"], v["ky"], v["ko"])
    ws = guarded((s.blk.workspace_bytes(n),), U8, 64)
    s.blk.bwd(dy, dh, v["ky"], v["ko"], g, wo, wi, v["r_o"], v["r_i"], v["dx"], v["do"], v["dg"], v["dwo"], v["dwi"], ws[:-64])
    ws2 = guarded((s.blk.wgrad_workspace_bytes(n, c, c),), U8, 64)
    s.blk.wgrad(dh, v["ky"], v["dw"], ws2[:-64], v["r_i"], wi)
    s.blk.glu_fwd(o, dh, v["a"], v["ky"], v["ko"])
    s.blk.glu_bwd(v["a"], v["ky"], v["ko"], v["h"], v["do"])
    s.blk.pack(x, v["ky"]), s.blk.unpack(v["ky"], v["h"])
    for k, t in big.items():
        assert (t[t.shape[0] - 3:].view(U8) == 0x5a).all(), k
    assert (ws[-64:] == 0x5a).all() and (ws2[-64:] == 0x5a).all()


@pytest.mark.parametrize("x", [F32, BF16])
def test_streams_in_place(B, x):
    """y may be x and dx may be dy."""
    s = Case(B, 300, 1032, x=x, w=x, kind="token", seed=11)
    fw = s.forward(True)
    bw = s.backward(fw, fw["ckpt_y"], fw["ckpt_o"])
    t, o, g, wo, wi, dy, dh = (cu(t) for t in (s.x, s.o, s.g, s.w_out, s.w_in, s.dy, s.dh))
    h, r_o, r_i, ky, ko = e((300, 1032), BF16), e((300,), F32), e((300,), F32), e((300, s.pitch), U8), e((300, s.pitch), U8)
    s.blk.fwd(t, o, g, wo, wi, t, h, r_o, r_i, ky, ko)
    assert torch.equal(t, fw["y"]) and torch.equal(h, fw["h"])
    d_o, dg, dwo, dwi, ws = e((300, 1032), BF16), e((300,), BF16), e((1032,), x), e((1032,), x), e((s.blk.workspace_bytes(300),), U8)
    s.blk.bwd(dy, dh, ky, ko, g, wo, wi, r_o, r_i, dy, d_o, dg, dwo, dwi, ws)
    same({"dx": dy, "d_o": d_o, "d_gate": dg, "dw_out": dwo, "dw_in": dwi}, bw)


def shifted(t, by=16):
    """The same values `by` bytes behind a 512-byte boundary."""
    if t is None:
        return None
    raw = torch.zeros(t.nbytes + 512, device="cuda", dtype=U8)
    v = raw[by:by + t.nbytes].view(t.dtype).view(t.shape)
    return v.copy_(t)


@pytest.mark.parametrize("c", [256, 1040])
def test_sixteen_byte_boundaries(B, c):
    """Base pointers on 16 bytes, not on the 32 of the widest accesses: the same bits."""
    s = Case(B, 90, c, kind="full", seed=12)
    fw = s.forward(True)
    bw = s.backward(fw, fw["ckpt_y"], fw["ckpt_o"])
    at = {k: shifted(cu(v)) for k, v in dict(x=s.x, o=s.o, g=s.g, wo=s.w_out, wi=s.w_in, dy=s.dy, dh=s.dh).items()}
    out = {k: None if v is None else shifted(torch.empty_like(v)) for k, v in fw.items()}
    s.blk.fwd(at["x"], at["o"], at["g"], at["wo"], at["wi"], out["y"], out["h"], out["r_out"], out["r_in"], out["ckpt_y"], out["ckpt_o"])
    same(known(out, s), known(fw, s))
    back = {k: shifted(torch.empty_like(v)) for k, v in bw.items()}
    ws = shifted(e((s.blk.workspace_bytes(90),), U8))
    s.blk.bwd(at["dy"], at["dh"], out["ckpt_y"], out["ckpt_o"], at["g"], at["wo"], at["wi"], out["r_out"], out["r_in"], back["dx"], back["d_o"], back["d_gate"],
              back["dw_out"], back["dw_in"], ws)
    same(back, bw)
    n = 90
    for dtype in (F32, BF16):
        g, u = rand((n, c), 5, dtype).cuda(), rand((n, c), 6, dtype).cuda()
        a, k1, k2 = e((n, c), dtype), e((n, s.pitch), U8), e((n, s.pitch), U8)
        s.blk.glu_fwd(g, u, a, k1, k2)
        a2, k3, k4 = shifted(a), shifted(k1), shifted(k2)
        s.blk.glu_fwd(shifted(g), shifted(u), a2.zero_(), k3, k4)
        d1, d2, d3, d4 = (torch.empty_like(a) for _ in range(4))
        s.blk.glu_bwd(a, k1, k2, d1, d2)
        d3, d4 = shifted(d3), shifted(d4)
        s.blk.glu_bwd(a2, k3, k4, d3, d4)
        assert torch.equal(a, a2) and torch.equal(d1, d3) and torch.equal(d2, d4)
        back = shifted(torch.empty_like(a))
        s.blk.unpack(k1, a), s.blk.unpack(k3, back)
        assert torch.equal(a, back)


def test_halves_with_odd_leading_sizes(B):
    """Leading sizes that break the 32-byte boundaries of every other row."""
    blk = B.Block(64, device=0)
    n, c = 45, 1040
    wide = rand((n, 2 * c + 8), 7, BF16).cuda()
    g, u, da = wide[:, :c], wide[:, c:2 * c], rand((n, c), 8, BF16).cuda()
    a, a2, k = e((n, c), BF16), e((n, c), BF16), [e((n, B.ckpt_pitch(c)), U8) for _ in range(4)]
    blk.glu_fwd(g, u, a, k[0], k[1])
    blk.glu_fwd(g.contiguous(), u.contiguous(), a2, k[2], k[3])
    assert torch.equal(a, a2) and all(torch.equal(p, q) for p, q in zip(bu.split(k[1].cpu(), c), bu.split(k[3].cpu(), c)))
    out, d1, d2 = e((n, 2 * c + 8), BF16), e((n, c), BF16), e((n, c), BF16)
    blk.glu_bwd(da, g, u, out[:, :c], out[:, c + 8:])
    blk.glu_bwd(da, g.contiguous(), u.contiguous(), d1, d2)
    assert torch.equal(out[:, :c], d1) and torch.equal(out[:, c + 8:], d2) and out[:, c:c + 8].isnan().all()


# ------------------------------------------------------------------------------------------------ order
def everything(B, blk, s, x, o, g, wo, wi, dy, dh, out):
    """Forward, backward, gated MLP and weight gradient on the current stream."""
    blk.fwd(x, o, g, wo, wi, out["y"], out["h"], out["r_o"], out["r_i"], out["ky"], out["ko"])
    blk.bwd(dy, dh, out["ky"], out["ko"], g, wo, wi, out["r_o"], out["r_i"], out["dx"], out["do"], out["dg"], out["dwo"], out["dwi"], out["ws"])
    blk.glu_fwd(out["h"], out["do"], out["a"], out["ky"], out["ko"])
    blk.glu_bwd(dh, out["ky"], out["ko"], out["da"], out["db"], out["a"])
    blk.pack(x, out["ky"])
    blk.wgrad(dh, out["ky"], out["dw"], out["ws"], out["r_i"], wi)
    blk.unpack(out["ky"], out["b"])


def buffers(s):
    n, c, p = s.n, s.c, s.pitch
    size = max(s.blk.workspace_bytes(n), s.blk.wgrad_workspace_bytes(n, c, c))
    return {k: e(sh, dt) for k, sh, dt in (("y", (n, c), F32), ("h", (n, c), BF16), ("r_o", (n,), F32), ("r_i", (n,), F32), ("ky", (n, p), U8), ("ko", (n, p), U8),
                                           ("dx", (n, c), F32), ("do", (n, c), BF16), ("dg", (n,), BF16), ("dwo", (c,), F32), ("dwi", (c,), F32), ("ws", (size,), U8),
                                           ("a", (n, c), BF16), ("da", (n, c), BF16), ("db", (n, c), BF16), ("dw", (c, c), F32), ("b", (n, c), BF16))}


RESULTS = ("y", "h", "r_o", "r_i", "dx", "do", "dg", "dwo", "dwi", "a", "da", "db", "dw", "b")


def test_repeatable_on_streams_in_graphs_and_with_a_shared_workspace(B):
    s = Case(B, 333, 520, kind="token", seed=13)
    args = [cu(t) for t in (s.x, s.o, s.g, s.w_out, s.w_in, s.dy, s.dh)]
    one = buffers(s)
    everything(B, s.blk, s, *args, one)
    torch.cuda.synchronize()
    want = {k: one[k].clone() for k in RESULTS}
    # two streams at once, a workspace each
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [buffers(s), buffers(s)]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for st, out in zip(streams, outs):
            with torch.cuda.stream(st):
                everything(B, s.blk, s, *args, out)
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(out[k], want[k]) for k in RESULTS)
    # two graphs on one workspace, replayed in turn with other inputs between
    s2 = Case(B, 333, 520, kind="token", seed=14)
    args2 = [cu(t) for t in (s2.x, s2.o, s2.g, s2.w_out, s2.w_in, s2.dy, s2.dh)]
    other = buffers(s)
    other["ws"] = one["ws"]
    everything(B, s.blk, s, *args2, other)
    torch.cuda.synchronize()
    want2 = {k: other[k].clone() for k in RESULTS}
    graphs = []
    st = torch.cuda.Stream()
    for a, out in ((args, one), (args2, other)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            everything(B, s.blk, s, *a, out)
        graphs.append(g)
    for k in RESULTS:
        one[k].fill_(float("nan")), other[k].fill_(float("nan"))
    for _ in range(5):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(one[k], want[k]) for k in RESULTS) and all(torch.equal(other[k], want2[k]) for k in RESULTS)
    assert s.blk.device_status() == (0, 0)


@pytest.mark.parametrize("c", [256, 1032, 8192])
def test_one_saved_in_full_and_one_in_8_bits(B, c):
    """y and o are saved independently of each other, in any of the types."""
    s = Case(B, 40, c, kind="token", seed=21)
    fw = s.forward(True)
    q = lambda t: bu.in_8_bits(t.cpu())
    for y, o, yr, orr in ((fw["ckpt_y"], cu(s.o), q(fw["y"]), s.o), (fw["y"], fw["ckpt_o"], fw["y"], q(s.o)), (fw["y"].to(BF16), cu(s.o).float(), fw["y"].to(BF16), s.o)):
        bw = s.backward(fw, y, o)
        for k, want in s.backward_ref(fw, yr, orr).items():
            bu.check(bw[k], want, k)


@pytest.mark.parametrize("kind", ["channel", "none"])
def test_gradients_added_to_what_is_there(B, kind):
    s = Case(B, 200, 264, kind=kind, seed=15)
    fw = s.forward()
    before = {k: rand((264,), 20 + i).cuda() for i, k in enumerate(("dw_in", "dw_out", "d_gate"))}
    plain, added = s.backward(fw), s.backward(fw, accumulate=before)
    for k in plain:
        if k in ("dw_in", "dw_out") or (k == "d_gate" and kind == "channel"):
            want = plain[k].double() + before[k].double()
            assert ((added[k].double() - want).abs() <= 2.0 ** -23 * (want.abs() + plain[k].double().abs())).all(), k
        else:
            assert torch.equal(plain[k], added[k]), k


def test_outputs_that_nobody_asks_for(B):
    """Each output alone.  (Such calls run kernels with the call's form looked up, where the compiler may fuse a product with a sum that it keeps apart in
    the others: not the same bits, but the same bounds, which hold for either.)"""
    s = Case(B, 120, 520, kind="full", seed=16)
    fw = s.forward()
    whole, ref = s.backward(fw), s.backward_ref(fw, fw["y"], s.o)
    order = ("dx", "d_o", "d_gate", "dw_out", "dw_in")
    args = [cu(t) for t in (s.dy, s.dh)], [cu(t) for t in (s.o, s.g, s.w_out, s.w_in)]
    ws = e((s.blk.workspace_bytes(120),), U8)
    for k in order:
        out = [torch.empty_like(whole[q]) if q == k else None for q in order]
        s.blk.bwd(*args[0], fw["y"], *args[1], fw["r_out"], fw["r_in"], *out, ws)
        bu.check(out[order.index(k)], ref[k], k)


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals(B):
    n, c = 10, 264
    s = Case(B, n, c, kind="token", seed=17)
    x, o, g, wo, wi, dy, dh = (cu(t) for t in (s.x, s.o, s.g, s.w_out, s.w_in, s.dy, s.dh))
    fw = s.forward(True)
    y, h, r_o, r_i, ky, ko = (fw[k] for k in ("y", "h", "r_out", "r_in", "ckpt_y", "ckpt_o"))
    ws = e((s.blk.workspace_bytes(n),), U8)
    fwd = lambda **k: s.blk.fwd(*[k.get(a, b) for a, b in dict(x=x, o=o, g=g, wo=wo, wi=wi, y=y, h=h, r_o=r_o, r_i=r_i, ky=ky, ko=ko).items()])
    bwd = lambda **k: s.blk.bwd(*[k.get(a, b) for a, b in dict(dy=dy, dh=dh, y=y, o=o, g=g, wo=wo, wi=wi, r_o=r_o, r_i=r_i, dx=e((n, c), F32), do=e((n, c), BF16),
                                                                 dg=e((n,), BF16), dwo=e((c,), F32), dwi=e((c,), F32), ws=ws, acc=False).items()])
    fwd(), bwd()
    odd = lambda t: torch.empty(t.nbytes + 16, device="cuda", dtype=U8)[t.element_size():t.element_size() + t.nbytes].view(t.dtype).view(t.shape)
    for bad in (dict(x=x[:, :256]), dict(x=x.double()), dict(y=y.to(BF16)), dict(h=h[:5]), dict(o=o.t()), dict(g=g[:5]), dict(wo=wo.to(BF16)), dict(r_i=r_i.to(BF16)),
                dict(ky=ky[:, :-16]), dict(ko=ko.to(F32)), dict(x=x.cpu()), dict(x=x.expand(n, c)[:, ::1].t().contiguous().t())):
        with pytest.raises(ValueError):
            fwd(**bad)
    for bad, code in ((dict(y=None), -1), (dict(h=None), -1), (dict(wi=None), -1), (dict(g=None), -1), (dict(o=None), -1), (dict(x=odd(x)), -1), (dict(h=odd(h)), -1),
                      (dict(ky=odd(ky)), -1)):
        with pytest.raises(B.AugtreeError) as err:
            fwd(**bad)
        assert err.value.code == code, bad
    for bad, code in ((dict(ws=ws[:-16]), -3), (dict(ws=odd(ws)), -3), (dict(r_i=None), -1), (dict(r_o=None), -1), (dict(y=None), -1), (dict(o=None, do=None, dg=None, g=None), -1),
                      (dict(wi=None, dwi=None), -1), (dict(dh=None), -1), (dict(do=odd(o)), -1)):
        with pytest.raises(B.AugtreeError) as err:
            bwd(**bad)
        assert err.value.code == code, bad
    for bad in (dict(dx=e((n, c), BF16)), dict(wi=None), dict(wo=None), dict(dy=None, dh=None), dict(y=y[:5]), dict(dg=None, g=g.float(), dwo=e((c,), BF16))):
        with pytest.raises(ValueError):
            bwd(**bad)
    low = Case(B, n, c, w=BF16, kind="none", seed=18)
    fl = low.forward()
    with pytest.raises(B.AugtreeError) as err:       # sums in bf16 are not added to
        low.backward(fl, accumulate={"dw_in": e((c,), BF16), "dw_out": e((c,), BF16)})
    assert err.value.code == -2
    none = B.Block(c, device=0)
    with pytest.raises(ValueError):                  # a gate for a handle without one
        none.fwd(x, o, g, wo, wi, y, h, r_o, r_i)
    k = e((n, B.ckpt_pitch(c)), U8)
    dw, ws2 = e((16, c), BF16), e((none.wgrad_workspace_bytes(n, 16, c),), U8)
    dz = e((n, 16), BF16)
    for call, code in ((lambda: none.wgrad(dz, k, dw, ws2, accumulate=True), -2), (lambda: none.wgrad(dz, k, dw, ws2[:-256]), -3), (lambda: none.wgrad(odd(dz), k, dw, ws2), -1),
                       (lambda: none.pack(odd(x), k), -1), (lambda: none.pack(e((n, c + 4), F32)[:, :c], k), -1), (lambda: none.glu_fwd(o, dh, h, k, None), -1)):
        with pytest.raises(B.AugtreeError) as err:
            call()
        assert err.value.code == code
    for call in (lambda: none.wgrad(dz, k, e((16, c), F16), ws2), lambda: none.wgrad(dz.to(F16), k, dw, ws2), lambda: none.pack(x.t(), k), lambda: none.glu_fwd(o, dh.to(F16), h),
                 lambda: none.glu_fwd(o, e((n, c + 8), BF16)[:, :c], h), lambda: none.glu_bwd(o, k, o, h, h), lambda: none.unpack(k, e((n, c), torch.float64)),
                 lambda: none.pack(x[:1].expand(n, c), k)):
        with pytest.raises(ValueError):
            call()
    wide = B.Block(8192, device=0, gate="full")
    z = lambda: torch.zeros(2, 8192, device="cuda")
    v, w8 = torch.zeros(2, device="cuda"), torch.ones(8192, device="cuda")
    with pytest.raises(B.AugtreeError) as err:       # five fp32 rows of 8192 do not fit a CTA
        wide.bwd(z(), z(), z(), z(), z(), w8, w8, v, v, z(), z(), z(), w8.clone(), w8.clone(), e((wide.workspace_bytes(2),), U8))
    assert err.value.code == -2
    assert s.blk.device_status() == (0, 0) and none.device_status() == (0, 0)
    fwd(), bwd()                                     # nothing of the refusals is left behind
    torch.cuda.synchronize()


def test_a_wait_that_runs_out_is_reported(B):
    """A stage that is never loaded: the calls return, the status word names the wait, the next call is right."""
    flags = B.FLAG_TEST_SHORT_WAIT | B.FLAG_TEST_SKIP_FWD_LOAD
    s = Case(B, 700, 520, kind="none", seed=19, flags=flags)
    fw = s.forward(True)
    status, site = s.blk.device_status()
    assert status == -5 and site == 90
    s.backward(fw)
    status, site = s.blk.device_status()
    assert status == -5 and site == 90
    dy, k, dw = rand((700, 256), 1, BF16).cuda(), fw["ckpt_o"], e((256, 520), F32)
    s.blk.pack(cu(s.o), k)
    for lanes, end in ((0, 108), (2, 104)):      # from the bits, by way of bf16 scratch (whichever of the waits on one another is the first to give up)
        blk = B.Block(64, device=0, flags=flags, n_lanes=lanes)
        blk.wgrad(dy, k, dw, e((blk.wgrad_workspace_bytes(700, 256, 520),), U8))
        status, site = blk.device_status()
        assert status == -5 and 100 <= site < end, site
    Case(B, 700, 520, kind="none", seed=19).check_all(True)


def test_a_handle_that_dies_during_a_capture(B):
    blk, old = B.Block(64, device=0), B.Block(128, device=0)
    x, k, out = rand((40, 64), 1, BF16).cuda(), e((40, B.ckpt_pitch(64)), U8), e((40, 64), BF16)
    blk.pack(x, k)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            blk.pack(x, k)
            del old
            blk.unpack(k, out)
    out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().double(), bu.in_8_bits(x.cpu()))

"""Host side of the vocabulary operators: descriptor checks and workspace sizes, no GPU."""
import ctypes as C

import pytest
import torch

from tests import lm_util as lu


@pytest.fixture(scope="module")
def B():
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import binding
    return binding


@pytest.mark.parametrize("kw,code", [
    (dict(vocab=0, hidden=64), -1), (dict(vocab=10, hidden=0), -1), (dict(vocab=10, hidden=-8), -1), (dict(vocab=10, hidden=60), -2),
    (dict(vocab=10, hidden=64, n_lanes=0), -1), (dict(vocab=10, hidden=64, n_lanes=-1), -1), (dict(vocab=10, hidden=64, piece_bytes=-1), -1),
    (dict(vocab=10, hidden=64, embed_scale=float("nan")), -1), (dict(vocab=10, hidden=64, logit_scale=float("inf")), -1),
    (dict(vocab=(1 << 27) + 1, hidden=64), -2), (dict(vocab=10, hidden=(1 << 20) + 8), -2)])
def test_descriptor_checks(B, kw, code):
    with pytest.raises(B.AugtreeError) as e:
        B.LM(**{"device": None, "n_lanes": 148, **kw})
    assert e.value.code == code


def test_bad_pointers_and_struct(B):
    h = C.c_void_p()
    assert B.lib.augtree_lm_create(None, -1, C.byref(h)) == -1 and not h.value
    d = B.LmDescC(4, 1, 10, 64, 0.0, 0.0, 0, 148, 0)
    assert B.lib.augtree_lm_create(C.byref(d), -1, C.byref(h)) == -1 and not h.value
    d = B.LmDescC(C.sizeof(B.LmDescC), 99, 10, 64, 0.0, 0.0, 0, 148, 0)
    assert B.lib.augtree_lm_create(C.byref(d), -1, C.byref(h)) == -1 and not h.value
    assert B.lib.augtree_lm_destroy(None) == -1
    lm = B.LM(10, 64, device=None, n_lanes=148)
    n = C.c_size_t()
    assert B.lib.augtree_lm_workspace_bytes(lm._h, -1, C.byref(n), None, None) == -1
    assert B.lib.augtree_lm_workspace_bytes(lm._h, 1 << 31, C.byref(n), None, None) == -2
    # launches on a host-only handle are refused before anything is touched
    assert B.lib.augtree_embed_fwd(lm._h, None, 0, None, 8, 1, None, 0, None) == -1
    assert B.lib.augtree_embed_bwd(lm._h, None, 0, None, 8, 1, None, 0, 0, None, 0, None) == -1
    assert B.lib.augtree_lm_loss_fwd(lm._h, None, None, None, 8, 1, None, None, None, 0, None) == -1
    assert B.lib.augtree_lm_loss_bwd(lm._h, None, None, None, 8, None, None, 1, None, None, 0, 0, None, 0, None) == -1
    s = C.c_int()
    assert B.lib.augtree_lm_last_device_status(lm._h, C.byref(s), None) == -1


def test_workspace_stays_far_below_the_logits(B):
    """The point of the operator: at 16384 rows x 152064 words the logits alone would be 10 GB in fp32."""
    lm = B.LM(152064, 3584, device=None, n_lanes=148)
    fwd, bwd, emb = lm.workspace_parts(16384)
    assert fwd < 0.05 * 16384 * 152064 * 4 and bwd < 0.2 * 16384 * 152064 * 4
    assert lm.workspace_bytes(16384) == max(fwd, bwd, emb)
    assert lm.workspace_bytes(0) > 0


def test_workspace_grows_with_the_piece_bound(B):
    small = B.LM(50000, 512, device=None, n_lanes=148, piece_bytes=1).workspace_parts(4096)[1]
    large = B.LM(50000, 512, device=None, n_lanes=148, piece_bytes=256 << 20).workspace_parts(4096)[1]
    assert small < large <= small + (256 << 20) + (64 << 20) * 64
    # sizes beyond 32 bits do not wrap
    assert B.LM(152064, 8192, device=None, n_lanes=148).workspace_parts(2_000_000)[1] > 2_000_000 * 8192 * 2


@pytest.mark.parametrize("vocab,hidden,lanes,piece", [(152064, 3584, 148, 0), (503, 256, 148, 0), (50257, 1032, 148, 1 << 24), (700, 64, 3, 1), (40000, 8, 1000, 0)])
def test_workspace_for_more_tokens_is_enough_for_fewer(B, vocab, hidden, lanes, piece):
    """Pieces, shares and the few-row kernels change with the number of tokens; the size that is told never shrinks with it."""
    lm = B.LM(vocab, hidden, device=None, n_lanes=lanes, piece_bytes=piece)
    last = (0, 0, 0)
    for n in sorted({*range(0, 700, 3), *range(700, 20000, 397), 127, 128, 129, 256, 257, 4096, 4097, 8192, 8193, 303104, 303105, 1000000}):
        now = lm.workspace_parts(n)
        assert all(a >= b for a, b in zip(now, last)), (n, now, last)
        last = now


def test_no_more_lanes_than_index_arithmetic_holds(B):
    """Grids are multiples of the lanes (32 of them for the lookup), and a partial sum is kept for each: a plan's limit holds here too."""
    assert B.LM(500, 64, device=None, n_lanes=1 << 20).workspace_bytes(100) > 0
    for lanes in ((1 << 20) + 1, (1 << 31) - 1):
        with pytest.raises(B.AugtreeError) as e:
            B.LM(500, 64, device=None, n_lanes=lanes)
        assert e.value.code == -2


@pytest.mark.parametrize("kw", [dict(vocab=(1 << 32) + 503), dict(hidden=(1 << 32) + 64), dict(n_lanes=(1 << 32) + 1), dict(vocab=-(1 << 32) + 503),
                                dict(piece_bytes=(1 << 64) + 1), dict(flags=1 << 32), dict(flags=-1),
                                dict(embed_scale=1e-50), dict(logit_scale=-1e-50)])
def test_numbers_beyond_the_descriptors_fields_are_refused(B, kw):
    """A field of 32 or 64 bits takes what fits of a number: a handle of other sizes than those that were asked for."""
    with pytest.raises(ValueError):
        B.LM(**{"vocab": 503, "hidden": 64, "device": None, "n_lanes": 148, **kw})


def test_token_counts_beyond_the_interface_are_refused(B):
    lm = B.LM(503, 64, device=None, n_lanes=148)
    for n in ((1 << 64) + 5, -(1 << 64) + 5):
        with pytest.raises(ValueError):
            lm.workspace_parts(n)


@pytest.mark.parametrize("t", [3, 128, 129, 256])
def test_bounds_of_two_halves_see_a_missing_half(t):
    """G rounded to bf16 once, in the plain form: outside the bounds that the kernels' two halves are held to; hi + lo is inside."""
    v, k = 257, 64
    h, w, y, a = lu.make_loss(t, v, k, seed=t, push=4.0)
    ref = lu.loss_reference(h, w, y, a)
    bound = lu.gradient_bounds_two_halves(ref, v, k, t)
    hd, wd = h.double(), w.double()
    x = hd @ wd.T
    g = a.double()[:, None] * (torch.softmax(x, 1) - torch.nn.functional.one_hot(y, v))
    hi = g.to(torch.bfloat16).double()
    lo = (g - hi).to(torch.bfloat16).double()
    bf = lambda z: z.to(torch.bfloat16).double()
    for name, one, two in (("d_hidden", hi @ wd, (hi + lo) @ wd), ("d_weight", hi.T @ hd, (hi + lo).T @ hd)):
        allowed = lu.delivered_bf16(ref[name], bound[name])
        assert ((bf(two) - ref[name]).abs() <= allowed).all(), name
        assert ((bf(one) - ref[name]).abs() > allowed).double().mean() > 0.02, name
    assert ((hi.T @ hd - ref["d_weight"]).abs() > bound["d_weight"] + 2.0 ** -24 * ref["d_weight"].abs()).double().mean() > 0.2
    assert ((hi + lo).T @ hd - ref["d_weight"]).abs().le(bound["d_weight"]).all()


@pytest.mark.parametrize("t,v,k", lu.LONG_CASES)
def test_bounds_of_long_contractions_see_wrong_results(t, v, k):
    h, w, y, a = lu.make_long(t, v, k, seed=t)
    ref = lu.loss_reference(h, w, y, a)
    bound = lu.loss_bounds(ref, v, k, t)
    # (rows of dW without a target are all sum_t a_t h_t / vocab but for the spread of p: only the targets' rows tell where they stand)
    rows = {"d_hidden": torch.arange(t), "d_weight": torch.unique(y), "loss": torch.arange(t), "lse": torch.arange(t)}
    out = lambda name, x: ((x - ref[name]).abs() > bound[name])[rows[name]].double().mean()
    for name in ("d_hidden", "d_weight"):
        assert out(name, torch.zeros_like(ref[name])) > 0.9                                   # nothing written
        assert out(name, ref[name].roll(1, 0)) > 0.9                                          # rows one off
        assert out(name, torch.cat([ref[name][:, 256:], ref[name][:, :256]], 1)) > 0.9        # column tiles one off
    assert out("d_weight", ref["d_weight"].roll(256, 0)) > 0.9                                # row tiles one off
    if t > 256:
        assert out("d_hidden", ref["d_hidden"].roll(256, 0)) > 0.9
    for name in ("loss", "lse"):
        assert out(name, torch.zeros_like(ref[name])) == 1
    assert out("loss", ref["loss"].roll(1)) > 0.8


def test_workspace_follows_the_piece_bound_and_no_more(B):
    """From a piece of one tile of columns (256, and 256 that equal pieces may be rounded up by) to one of 256 MiB: G grows by the bound less
    a tile, 16 a row of everything else is as before."""
    rows, mib = 4096, 1 << 20
    small = B.LM(50000, 512, device=None, n_lanes=148, piece_bytes=1).workspace_parts(rows)[1]
    large = B.LM(50000, 512, device=None, n_lanes=148, piece_bytes=256 * mib).workspace_parts(rows)[1]
    assert 250 * mib < large - small <= 256 * mib
    # the rest: packed hidden states, partial sums of dH (at most 16384 rows of them, or twice the rows), a few numbers a row
    assert small <= rows * 512 * 2 + max(16384, 2 * rows) * 512 * 4 + rows * 512 * 2 + 64 * rows + (1 << 14)

"""Host side of the block ends and checkpoints, continued: what can be seen without a GPU."""
import gc
import os
import re
import shutil
import subprocess
import sys
import weakref

import pytest
import torch

from tests import block_util as bu

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_33133_b200", "csrc")


@pytest.fixture(scope="module")
def B():
    from paper_2609_33133_b200 import build
    build.build()
    from paper_2609_33133_b200 import binding
    return binding


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_shared_memory_for_the_other_cta_is_handed_over_at_cluster_scope():
    """The arrival without release at cluster scope is for TMEM that has been read (the accumulators' barriers) and for nothing else; operands that warps
    have written for the pair's MMA are released, and waited for, at cluster scope."""
    plain, released, waited = set(), set(), set()
    for name in (n for n in os.listdir(CSRC) if n.endswith(".cuh") and n != "ptx.cuh"):
        text = source(name)
        plain |= set(re.findall(r"mbar_arrive_cluster\(map_to_rank\((\w+)", text))
        released |= set(re.findall(r"mbar_arrive_cluster_release\(map_to_rank\((\w+)", text))
        waited |= set(re.findall(r"mbar_wait_cluster\((\w+)", text))
    assert plain == {"acc_empty", "bar_acc_empty"} and released == waited == {"x_full"}
    ptx = source("ptx.cuh")
    body = lambda name: re.search(r"\b" + name + r"\([^{]*\{(.*?)\n?\}\n", ptx, re.S).group(1)
    assert re.search(r"fence\.release\.sync_restrict::shared::cta\.cluster;.*mbarrier\.arrive\.relaxed\.cluster\.shared::cluster", body("mbar_arrive_cluster_release"))
    assert "mbarrier.try_wait.parity.relaxed.cluster.shared::cta" in body("mbar_try_wait_cluster")
    assert "fence.acquire.sync_restrict::shared::cluster.cluster;" in body("acquire_cluster_shared") and "acquire_cluster_shared();" in body("mbar_wait_cluster")


# ------------------------------------------------------------------------------------------------ autograd, with a handle that does no arithmetic
class Still:
    """A handle whose calls do nothing: what autograd keeps, releases and refuses does not depend on the numbers."""

    def __init__(self, hidden):
        self.hidden, self.calls = hidden, []

    def __getattr__(self, name):
        return lambda *a, **k: self.calls.append((name, a, k))

    def workspace_bytes(self, n):
        return 16

    def wgrad_workspace_bytes(self, *a):
        return 16


def chain(A, blk, ckpt):
    """(loss, checkpoints) of a block end, a product of its norm and a gated MLP."""
    leaf = lambda *s, dtype=torch.float32: torch.ones(s, dtype=dtype, requires_grad=True)
    x, o, w = leaf(6, 64), leaf(6, 64, dtype=torch.bfloat16), leaf(64)
    _, h, kept = A.block(blk, x, o, None, w, w, ckpt=ckpt)
    z = A.linear(blk, h, leaf(72, 64, dtype=torch.bfloat16), kept)
    return A.glu_linear(blk, z, z * 2, leaf(64, 72, dtype=torch.bfloat16), ckpt=ckpt).float().sum(), kept


def test_checkpoints_are_saved_tensors(B):
    """Released as the backward pass goes by even if the loss is held, seen by hooks, and a change in place is an error."""
    from paper_2609_33133_b200 import autograd as A
    blk, live = Still(64), []
    alive = lambda: sum(r() is not None for r in live)

    def pack(t):
        if t.dtype is torch.uint8:
            live.append(weakref.ref(t))
        return t
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
        loss, kept = chain(A, blk, True)
    assert len(live) == 5 and kept.ckpt.shape == (6, B.ckpt_pitch(64))     # y and o of the block end, y again for the product, g and u
    blk.calls.clear()
    del kept
    gc.collect()
    assert alive() == 5
    loss.backward()
    blk.calls.clear()
    gc.collect()
    assert loss is not None and alive() == 0
    for change in ("ckpt", "row"):
        loss, kept = chain(A, Still(64), True)
        getattr(kept, change).zero_()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


def test_a_product_whose_gradient_cannot_be_made_is_refused_at_once(B):
    from paper_2609_33133_b200 import autograd as A
    BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
    blk = Still(64)

    def product(n=6, out=72, h=BF16, weight=BF16, shape=None, rows=None, wanted=True, device="cpu"):
        kept = A.Kept(torch.zeros(rows or n, B.ckpt_pitch(64), dtype=torch.uint8), torch.ones(rows or n), torch.ones(64))
        return A.linear(blk, torch.ones(shape or (n, 64), dtype=h, device=device), torch.ones(out, 64, dtype=weight, requires_grad=wanted, device=device), kept)
    product().float().sum().backward()
    assert [name for name, _, _ in blk.calls] == ["wgrad"]
    for bad in (dict(h=F16, weight=F16), dict(h=F32, weight=F32), dict(out=60), dict(shape=(2, 3, 64)), dict(shape=(64,)), dict(rows=5)):
        with pytest.raises(ValueError, match="linear"):
            product(**bad)
        product(**bad, wanted=False)       # (nobody wants the weight's gradient)
        with torch.no_grad():
            product(**bad)
    blk = B.Block(64, device=None, n_lanes=4)
    with pytest.raises(B.AugtreeError) as err:      # more features than the product takes
        product(out=(1 << 20) + 8, device="meta")
    assert err.value.code == B.ERR_UNSUPPORTED
    with torch.autocast("cpu", BF16):      # the product's type counts, not its operands'
        assert product(weight=F32).dtype is BF16


# ------------------------------------------------------------------------------------------------ the extension that checks arguments
@pytest.mark.parametrize("broken", [False, True])
def test_only_the_block_handle_needs_the_argument_checks(B, tmp_path, broken):
    """Without csrc/marshal.cpp's extension, or with one that does not load, plans and vocabulary handles work and a block handle says what to do."""
    from paper_2609_33133_b200 import build
    package = os.path.basename(build.HERE)
    shutil.copytree(build.HERE, tmp_path / package, ignore=shutil.ignore_patterns("_marshal*", "__pycache__"))
    if broken:
        (tmp_path / package / os.path.basename(build.marshal_path())).write_bytes(b"not a library")
    code = ("from paper_2609_33133_b200 import binding as B\n"
            "plan, lm = B.Plan([5], [[3]], 2, 1, 64, device=None, n_lanes=4), B.LM(503, 64, device=None, n_lanes=4)\n"
            "try:\n    B.Block(64, device=None, n_lanes=4)\n"
            "except ImportError as err:\n    print(plan.total_p, lm.vocab, err)\n")
    run = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env={**os.environ, "PYTHONPATH": str(tmp_path)}, capture_output=True, text=True)
    assert run.returncode == 0 and run.stdout.startswith("5 503 "), run.stdout + run.stderr
    assert ("does not load" if broken else "is missing") in run.stdout and "paper_2609_33133_b200.build" in run.stdout


def test_another_torch_gets_an_extension_of_its_own(B, monkeypatch):
    from paper_2609_33133_b200 import build
    here = build.marshal_path()
    assert os.path.exists(here) and not build._stale(here, build.MARSHAL_SOURCES)
    monkeypatch.setattr(torch, "__version__", "99.0")
    assert build.marshal_path() != here and build._stale(build.marshal_path(), build.MARSHAL_SOURCES)


# ------------------------------------------------------------------------------------------------ the weight gradient's bounds
@pytest.mark.parametrize("n", [65, 743, 2183, 5000])
def test_the_bounds_see_mistakes_in_the_tokens_factors(n):
    """A rounding too many of the factors, a scale, the last token with its neighbour's factor, two tokens swapped, the last token left out."""
    gen = torch.Generator().manual_seed(n)
    randn = lambda *s: torch.randn(*s, generator=gen)
    dy, x, row, col = randn(n, 72).to(torch.bfloat16), bu.in_8_bits(2 * randn(n, 64)), randn(n).abs() + 0.1, 1 + 0.2 * randn(64)
    want = bu.wgrad_exact_operand(dy, x, row, col, torch.float32)
    bu.check_delivered(want[0].float(), want)
    last, swapped = row.clone(), row.clone()
    last[-1], swapped[3], swapped[17] = row[-2], row[17], row[3]
    for other in ((dy, x, row.to(torch.bfloat16).float(), col), (dy, x, 1.003 * row, col), (dy, x, last, col), (dy, x, swapped, col), (dy[:-1], x[:-1], row[:-1], col),
                  (dy, x * row[:, None], None, col)):
        with pytest.raises(AssertionError):
            bu.check_delivered(bu.wgrad_exact_operand(*other, torch.float32)[0].float(), want)

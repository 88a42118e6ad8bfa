"""Host side of the block ends and checkpoints, continued: what can be seen without a GPU."""
import os
import re

import pytest
import torch

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

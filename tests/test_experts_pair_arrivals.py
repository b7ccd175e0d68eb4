"""Arrivals of threads on a barrier in the other CTA of a pair name the cluster as their scope, and the waits for them too: an
arrival of CTA scope and a wait in another CTA are no pair in the memory model. Read from the sources (what a narrower scope gives
is wrong now and then at most)."""
import os
import re

import pytest

from paper_2604_23996_gb300.build import CSRC


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_arrivals_by_a_cluster_address_have_cluster_scope():
    arrivals = re.findall(r"mbarrier\.arrive[\w.:]*shared::cluster[\w.:]*", source("ptx.cuh"))
    assert len(arrivals) >= 3
    for a in arrivals:
        assert ".cluster.shared::cluster" in a and (".relaxed." in a or ".release." in a), a


@pytest.mark.parametrize("name,barriers", [("expert_gemm.cu", {"acc_empty"}), ("expert_gemm_f32.cu", {"acc_empty", "split_peer"}),
                                           ("expert_mx.cu", {"acc_empty", "full"})])
def test_waits_for_them_have_cluster_scope(name, barriers):
    text = source(name)
    given = set(re.findall(r"mbar_arrive_peer(?:_release)?\(peer_smem\(&bars\.(\w+)\[", text))
    assert barriers <= given
    for b in barriers:
        waits = re.findall(rf"(warp_wait(?:<true>)?)\(&bars\.{b}\[", text)
        assert waits and all(w == "warp_wait<true>" for w in waits), (b, waits)


@pytest.mark.parametrize("name", ["expert_gemm.cu", "expert_gemm_f32.cu", "expert_mx.cu"])
def test_a_relaxed_arrival_follows_the_fence_of_tensor_memory(name):
    """It orders nothing but what tc_fence_before does: tensor memory that the warp has read or written."""
    text = source(name)
    for m in re.finditer(r"mbar_arrive_peer\(", text):
        before = text[:m.start()]
        if re.search(r"if \(chunks <= g && lane == 0\) $", before):
            continue                                    # a warp without a chunk: it has touched nothing
        last = before[before.rindex("tc_fence_before();"):]
        assert "__syncwarp();" in last and not re.search(r"st\.shared|stmatrix|\*reinterpret_cast|tmem_ld|tmem_st\d", last), last

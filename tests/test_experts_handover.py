"""What a CTA's threads write to its shared memory for the tensor cores of both CTAs of a pair is handed to the CTA that issues the
products: with a release at cluster scope where it lives in the other CTA, and a wait that acquires at that scope. Read from the
sources (a narrower arrival gives wrong results now and then at most): between a kernel's fence of such writes for the tensor
cores and the arrival that hands them over there is no arrival of CTA scope on a barrier of the pair."""
import os
import re

import pytest

from paper_2604_23996_gb300.build import CSRC


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["expert_gemm.cu", "expert_gemm_f32.cu"])
def test_writes_for_the_pairs_tensor_cores_are_released_to_the_pair(name):
    text = source(name)
    fences = [m.end() for m in re.finditer(r"fence_proxy_async_smem\(\);", text)]
    assert fences
    for at in fences:
        after = text[at:at + 500].split("fence_proxy_async_smem();")[0].split("tc_fence_before();")[0]
        assert "mbar_arrive_peer(" not in after, after
    assert "mbar_arrive_peer_release(" in text and "warp_wait<true>(" in text


def test_the_pairs_forms_have_cluster_scope():
    text = source("ptx.cuh")
    body = lambda f: text[text.index(f):].split("}\n")[0]  # noqa: E731
    assert "mbarrier.arrive.release.cluster.shared::cluster" in body("void mbar_arrive_peer_release(")
    assert "mbarrier.try_wait.parity.acquire.cluster" in text[text.index("bool mbar_try_wait_cluster("):][:500]

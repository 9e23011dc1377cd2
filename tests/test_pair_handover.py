"""CTA pairs: what one CTA hands to the other through a barrier in its shared memory is released and acquired at cluster scope (an arrive
or a wait without a qualifier reaches the threads of one CTA only)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09821_b200", "csrc")


def code(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


@pytest.mark.parametrize("name", ["act8_gemm.cu", "mlp_tc.cu", "tc_ptx.cuh"])
def test_remote_arrives_release_at_cluster_scope(name):
    text = code(name)
    for arrive in re.finditer(r"mbarrier\.arrive[\w.:]*shared::cluster[\w.:]*", text):
        body = text[text.rindex("{", 0, arrive.start()):arrive.start()]
        fenced = ".relaxed.cluster" in arrive.group() and "fence.release.sync_restrict::shared::cta.cluster" in body
        assert ".release.cluster" in arrive.group() or fenced, arrive.group()


def test_the_leader_acquires_at_cluster_scope():
    text = code("act8_gemm.cu")
    assert "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64" in text
    # the barriers that the other CTA arrives on, acc_empty and the leader's full, are waited for by the warp that issues MMAs
    issuer = text[text.index("} else if (warp == 1) {"):text.index("} else if (warp < kFirstDecode) {")]
    assert len(re.findall(r"warp_wait<PAIR>\(", issuer)) == len(re.findall(r"warp_wait", issuer)) == 2
    assert re.search(r"template <bool FROM_PEER = false>\s*__device__ __forceinline__ bool warp_wait", text)
    assert len(re.findall(r"acc_empty\[acc\]\), acc_phase \^ 1u", text)) == 1

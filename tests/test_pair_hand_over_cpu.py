"""What a CTA of a pair hands over to the other one is released to it: read from the source, since on the GPU a missing order shows rarely or never."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_02495_b200", "csrc")


def test_words_in_shared_memory_are_released_to_the_other_cta():
    """An arrival without release hands over TMEM only (tempty, behind the fences of tcgen05), or follows a release of shared memory; and the
    issuer's wait for a stage acquires at cluster scope."""
    text = open(os.path.join(CSRC, "fp8_gemm_tcgen05.cu")).read()
    lines = text.splitlines()
    relaxed = [i for i, s in enumerate(lines) if "mbar_arrive_cluster_relaxed(" in s]
    assert relaxed
    for i in relaxed:
        if "->tempty" in lines[i]:
            assert re.search(r"tmem_ld_wait\(\);\s*tc_fence_before\(\);\s*__syncwarp\(\);", "\n".join(lines[i - 8:i]))
        else:
            assert "fence_release_smem();" in lines[i - 1], lines[i]
    assert re.search(r"PAIR \? mbar_wait_warp_cluster\(&ctl->full\[stage\]", text)
    tc = open(os.path.join(CSRC, "tc.cuh")).read()
    assert "fence.release.sync_restrict::shared::cta.cluster;" in tc and "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64" in tc

"""Host-side check of the hand-over of scale words inside a pair of CTAs: compiled with g++ and run, and what the kernel arrives on."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2503_02495_b200", "csrc")


def test_every_order_ends_with_every_block_passed_on(tmp_path):
    exe = str(tmp_path / "pair_scales_check")
    src = os.path.join(ROOT, "tests", "host", "pair_scales_check.cpp")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, src, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.strip().endswith("ok")


def test_words_in_shared_memory_are_released_to_the_other_cta():
    """An arrival without release hands over TMEM only (tempty, behind the fences of tcgen05), or follows a fence of cluster scope."""
    lines = open(os.path.join(CSRC, "fp8_gemm_tcgen05.cu")).read().splitlines()
    relaxed = [i for i, s in enumerate(lines) if "mbar_arrive_cluster_relaxed(" in s]
    assert relaxed
    for i in relaxed:
        before = "\n".join(lines[i - 8:i])
        if "->tempty" in lines[i]:
            assert re.search(r"tmem_ld_wait\(\);\s*tc_fence_before\(\);\s*__syncwarp\(\);", before)
        else:
            assert re.search(r"fence_cluster\(\);[^\n]*$", before), lines[i]

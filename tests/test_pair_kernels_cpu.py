"""Rules that the kernels on CTA pairs keep, read off their sources: what breaks them shows once in thousands of calls or not at all, and then
as a GPU that waits for ever, so no run is made to show it."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_01703_b200", "csrc")


def _source(path):
    text = open(path).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


PAIRS = sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*.cu")) if "tmem_alloc_pair" in _source(p))


def test_the_files_with_kernels_on_pairs_are_found():
    assert {"lm_loss.cu", "project_tc.cu", "score_tc.cu"} <= set(PAIRS)


@pytest.mark.parametrize("name", PAIRS)
def test_no_kernel_beside_one_on_pairs_begins_early_or_lets_another_begin(name):
    text = _source(os.path.join(CSRC, name))
    for word in ("ahead_release", "ahead_wait", "launch_ahead", "griddepcontrol", "ProgrammaticStreamSerialization"):
        assert word not in text, word


def _kernels(text):
    """Bodies of the kernels of a source that allocate tensor memory for a pair."""
    parts = re.split(r"(?=__global__)", text)
    return [part for part in parts if "tmem_alloc_pair(" in part]


@pytest.mark.parametrize("name", PAIRS)
def test_both_blocks_of_a_pair_wait_for_the_commits_that_arrive_in_them(name):
    # a commit of the leader arrives in the shared memory of both; the last one is waited for behind the roles, by both, before the pair parts
    seen = 0
    for body in _kernels(_source(os.path.join(CSRC, name))):
        if "mma_commit_pair(" not in body:
            continue
        seen += 1
        end = body[body.rindex("__syncthreads();"):body.index("tmem_dealloc_pair(")]
        wait = re.search(r"if \((?:warp == \d|threadIdx\.x == 0)\) (?:pair_drained\(&bars->(\w+)\)|mbar_wait\(smem_u32\(&bars->(\w+)\), 0,)", end)
        assert wait is not None and end.index("cluster_sync_all();") > wait.start()
        last = wait.group(1) or wait.group(2)
        assert re.findall(r"mma_commit_pair\(smem_u32\(&bars->(\w+)", body)[-1] == last
        # rings that a producer or generator waits for are waited for once more behind their last use
        for ring in set(re.findall(r"mma_commit_pair\(smem_u32\(&bars->(\w*empty)", body)):
            assert re.search(r"ring_drained\(bars->%s|mbar_wait_cluster\(smem_u32\(&bars->%s\[grp\]" % (ring, ring), body) or last == "done", ring
    assert seen >= (2 if name == "microbench.cu" else 1)

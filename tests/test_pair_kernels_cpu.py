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

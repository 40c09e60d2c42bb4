"""Rules about tensor memory that the kernels keep, read off their sources: what breaks them depends on how blocks happen to meet on an SM, or on how the compiler
happens to lay out a loop, and would show as a GPU that waits for ever. So no run is made to show it."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_01703_b200", "csrc")


def _source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def _kernels(name):
    """(name, body) of each kernel of a source."""
    for part in re.split(r"(?=__global__)", _source(name))[1:]:
        at = part.index("{")
        found = re.search(r"(\w+)\s*\([^{]*$", part[:at])
        depth = 0
        for i in range(at, len(part)):
            depth += (part[i] == "{") - (part[i] == "}")
            if depth == 0:
                break
        yield re.findall(r"(\w+_kernel)\b", part[:at])[0] if "_kernel" in part[:at] else found.group(1), part[at:i + 1]


FILES = sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*.cu")))
HOLDERS = [(f, k, body) for f in FILES for k, body in _kernels(f) if re.search(r"\btmem_alloc\(", body) and "ahead_release();" in body]


def test_the_kernels_that_are_launched_ahead_and_hold_tensor_memory_are_found():
    assert {k for _, k, _ in HOLDERS} == {"attention_kernel", "attention_dq_kernel", "attention_dkv_kernel", "few_gemm_kernel", "lora_factors_kernel", "lora_outer_kernel"}


@pytest.mark.parametrize("name,kernel,body", HOLDERS, ids=[k for _, k, _ in HOLDERS])
def test_no_kernel_lets_the_next_one_in_before_it_has_its_tensor_memory(name, kernel, body):
    """A block of the next kernel may share an SM with one of this kernel's. Had it taken tensor memory first, it would hold it until this kernel has ended
    (griddepcontrol.wait), and this kernel's block would wait for tensor memory for ever. One thread's release is the block's, so the barrier behind the
    allocation has to lie between."""
    alloc = re.search(r"\btmem_alloc\(", body).start()
    barrier = body.index("__syncthreads();", alloc)
    assert body.count("ahead_release();") == 1 and body.index("ahead_release();") > barrier

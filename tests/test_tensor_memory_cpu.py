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


# ---- accesses by whole warps ---------------------------------------------------------------------------------------------

ACCESS = re.compile(r"\btmem_(?:ld|st)_x\d+\(")
TOGETHER = re.compile(r"__syncwarp\(\);|__(?:all|any|shfl_xor|shfl)_sync\(|__syncthreads\(\);|\btmem_(?:ld|st)_x\d+\(")      # a warp's lanes are together behind these
APART = re.compile(r"lane == 0|lane <|\bcontinue;|>= feats|at < w\.t\.len|store_rows32\(|\bput\(|\bdst\[|nullptr\)")      # and may part at these
LAYER = ["attention.cu", "attention_backward.cu", "ffn.cu", "ffn_few.cu", "ffn_common.cuh"]


def _blocks(text):
    """(start, end) of every braced block."""
    stack, got = [], []
    for i, c in enumerate(text):
        if c == "{":
            stack.append(i)
        elif c == "}":
            got.append((stack.pop(), i))
    return got


@pytest.mark.parametrize("name", LAYER)
def test_lanes_are_together_at_every_access_to_tensor_memory(name):
    """tcgen05.ld and tcgen05.st are instructions of a whole warp (.sync.aligned). Between a statement at which lanes may part (a store by some of them, an arrival by
    one) and the next such access stands one that brings them together: in a function, behind its beginning; in a loop, inside the loop, for its last statements
    come before its first."""
    text = _source(name)
    blocks = _blocks(text)
    looked_at = 0
    for m in ACCESS.finditer(text):
        looked_at += 1
        before, line = text[:m.start()], text[m.start():m.start() + 60]
        together = [t.start() for t in TOGETHER.finditer(before)]
        apart = [t.start() for t in APART.finditer(before)]
        assert together and (not apart or max(together) > max(apart)), line
        for lo, hi in blocks:
            if not lo < m.start() < hi:
                continue
            head = before[max(before.rfind(c, 0, lo) for c in ";}") + 1:lo]
            loop = re.search(r"for \(int c0? = [^;]*;[^;]*;[^;]*\)\s*$", before[:lo])
            if (loop and APART.search(text[lo:hi])) or re.search(r"__device__ __forceinline__ void", head):
                assert any(t > lo for t in together), line
    assert looked_at or name in ("ffn.cu", "ffn_few.cu")      # (all of theirs are load_acc's)

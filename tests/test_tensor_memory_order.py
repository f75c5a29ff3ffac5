"""A kernel that lets the next one of its stream start early (chain_next) does so behind its own allocation of tensor memory and a barrier
of the warps that say so: the next one's blocks may find their place beside this kernel's, and if they took the columns first they would hold them
until this kernel ends, which waits for the columns."""
import glob
import os
import re

import pytest

from paper_1905_10830_b200 import build

SOURCES = sorted(p for p in glob.glob(os.path.join(build.CSRC, "*.cu")) if "tmem_alloc" in open(p).read())


def _functions(path):
    """The bodies of a source's functions: from a brace in column 0 to the one that closes it."""
    code = re.sub(r"//[^\n]*", "", open(path).read())
    return re.findall(r"^\{$(.*?)^\}", code, re.M | re.S)


def test_sources_are_found():
    names = {os.path.basename(p) for p in SOURCES}
    assert {"block_matmul.cu", "decode_runs.cu", "encode_tc.cu", "wide_gemm.cu"} <= names
    for path in SOURCES:
        inside = sum(f.count("tmem_alloc") for f in _functions(path))
        assert inside == open(path).read().count("tmem_alloc") > 0, path


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_the_next_kernel_starts_behind_the_allocation(path):
    for body in _functions(path):
        alloc, start = body.find("tmem_alloc"), body.find("chain_next()")
        if alloc < 0 or start < 0:
            continue
        between = body[alloc:start]
        assert start > alloc, "chain_next ahead of the allocation"
        assert re.search(r"__syncthreads\(\)|named_bar_sync\(|cluster_sync\(\)", between), "no barrier between the allocation and chain_next"

"""Order of cluster barriers and accesses to another CTA's shared memory (peer_*, pair_*) in the
low-precision and block-attention kernels, from their source: between the first and the last
barrier only."""

import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_09231_gb300", "csrc")
REMOTE = r"\b(peer_\w+|pair_\w+)\("
BARRIER = r"\bcluster_sync_all\("


def kernels():
    for f in ("gemm_fp8.cu", "attn_blocks.cu", "lowbit.cu"):
        src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, f)).read())
        for m in re.finditer(r"__global__[^;{]*?(\w+_kernel)\(", src):
            i = src.index("{", m.end())
            depth, j = 1, i + 1
            while depth:
                depth += {"{": 1, "}": -1}.get(src[j], 0)
                j += 1
            if re.search(REMOTE, src[i:j]):
                yield m.group(1), src[i:j]


def test_the_kernels_are_found():
    assert {"gemm_fp8_few_kernel", "gemm_fp8_pair_kernel", "attn_blocks_kernel", "attn_token_kernel"} == {n for n, _ in kernels()}


@pytest.mark.parametrize("name,body", list(kernels()), ids=lambda v: v if v.endswith("_kernel") else "")
def test_remote_accesses_lie_between_cluster_barriers(name, body):
    remote = [m.start() for m in re.finditer(REMOTE, body)]
    barriers = [m.start() for m in re.finditer(BARRIER, body)]
    assert barriers and barriers[0] < remote[0] and barriers[-1] > remote[-1]

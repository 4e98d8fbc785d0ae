"""Another block's shared memory is only defined once that block is known to have started: a kernel that stores or signals there has a cluster barrier before its first such access, not only
behind it. Nothing shows on a GPU when it is missing, as long as the blocks of a cluster happen to start together, so the sources are read."""
import os
import re

import pytest

from paper_1701_06538_b200 import build as moe_build

REMOTE = r"st\.shared::cluster|st_cluster_v4\(|mbar_arrive_cluster_addr\(|mbar_arrive_leader"
BARRIER = r"barrier\.cluster\.wait|cluster_sync_all\(\)|cluster_wait\(\)"


def kernels(text):
    """(name, body) of every __global__ function."""
    for m in re.finditer(r"__global__\s+void\s+(?:__\w+__\((?:[^()]|\([^()]*\))*\)\s*)*(\w+)\([^{;]*\)\s*\{", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield m.group(1), text[m.end():at]


@pytest.mark.parametrize("source,kernel", [("few_tokens.cu", "few_logits_kernel"), ("ffn_tc.cu", "grouped_gemm2_kernel"), ("products.cu", "expert_products_kernel")])
def test_a_barrier_before_the_first_remote_store(source, kernel):
    with open(os.path.join(moe_build.CSRC, source)) as f:
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    bodies = {name: body for name, body in kernels(text) if re.search(REMOTE, body)}
    assert kernel in bodies, sorted(bodies)
    for name, body in bodies.items():
        first = re.search(REMOTE, body).start()
        assert re.search(BARRIER, body[:first]), f"{name} reaches into another block's shared memory before any cluster barrier"

"""The second launch of the layer for a few tokens begins before the first has ended, and the first before what made its inputs has. Non-coherent loads (__ldg, pointers to const that are
__restrict__) are defined for memory that nothing writes while the kernel runs, so the kernels that start early have none of them. Only the sources can show it: what is wrong about them depends on
where the compiler puts the load."""
import os
import re

from paper_1701_06538_b200 import build as moe_build


def source():
    with open(os.path.join(moe_build.CSRC, "few_tokens.cu")) as f:
        return re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)


def test_no_non_coherent_loads():
    text = source()
    assert "__ldg(" not in text and "ld.global.nc" not in text
    assert not re.search(r"__global__[^;{]*few_select_kernel\([^)]*__restrict__", text)


def test_the_lanes_loads_come_behind_the_look_at_the_counter():
    """One lane waits for a token's parts, all lanes load them: between the two stand a fence and a warp barrier. A vote makes the lanes meet but orders no memory."""
    text = source()
    body = text[text.index("bool complete("):]
    body = body[:body.index("return __all_sync")]
    assert 0 < body.index("load_relaxed") < body.index("__threadfence()") < body.index("__syncwarp()")

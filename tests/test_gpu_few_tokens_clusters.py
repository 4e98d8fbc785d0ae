"""The routing of a few tokens by clusters of one to eight blocks, over chains so short that the blocks hand over their logits as soon as they start."""
import pytest
import torch

import test_gpu_few_tokens as F
from paper_1701_06538_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,act", [(4, "f32"), (8, "bf16")])
@pytest.mark.parametrize("n", [20, 40, 96, 100, 130, 192, 200, 256])
def test_short_chains(n, d, act):
    for T in (1, 6, 64):
        t, cfg = F.layer(T, d, 8, n, 2, act), B.make_config(T, d, 8, n, 2, act)
        want = F.routed_by_moe_gate(cfg, t)
        for _ in range(5):
            got = F.run(cfg, t)[1:]
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

"""The block for up to eight tokens on both sides of the weights' size at which it changes kernels."""
import pytest
import torch

import paper_2604_03446_b200 as mm
import test_gpu_gated_ffn as block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(block.TYPES))
@pytest.mark.parametrize("sizes", [(1, 4096, 8192, 4096), (7, 2048, 20480, 1024), (2, 4096, 16384, 4096), (8, 16384, 2048, 16384 + 8)],
                         ids=lambda s: "x".join(map(str, s)))
def test_few_tokens_through_weights_of_a_hundred_megabytes_and_more(sizes, dtype):
    t = block.make(*sizes, block.TYPES[dtype], seed=61)
    y, saved = mm.mmee_gated_ffn(*t[:4], save=True)
    want = block.formulas(*t, "silu", torch.finfo(block.TYPES[dtype]).eps / 2)
    block.inside("y", y, want["y"])
    block.inside("hidden", saved[0], want["hidden"])
    mm.mmee_chain_status()

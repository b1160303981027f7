"""Calls of the chains through the C interface that are refused before anything is launched (no GPU)."""
import math

import numpy as np
import pytest

import paper_2604_03446_b200 as mm
import test_gpu_attention as attention
from test_gpu_attention import _Case


def both(c):
    lib = mm.library()
    return lib.mmee_attention(c.w, c.a, None), lib.mmee_attention_backward(c.w, c.a, c.g, None)


@pytest.mark.parametrize("field", ["lse", "kv_len"])
@pytest.mark.parametrize("address", [4097, 4098, 4099])
def test_words_of_32_bits_at_odd_addresses_are_refused(field, address):
    """(A kernel that reads or writes one there faults.)"""
    c = _Case()
    setattr(c.a, field, address)
    assert both(c) == (mm.ERR_ARG, mm.ERR_ARG)


@pytest.mark.parametrize("scale", [1e-45, 2.0 ** -127, float(np.nextafter(np.float32(2.0 ** -126), np.float32(0))),
                                   float(np.nextafter(np.float32(2.0 ** 127), np.float32(math.inf))), 3.4e38])
def test_scales_whose_powers_of_two_leave_32_bits_are_refused(scale):
    """scale log2(e) would be flushed to zero or infinite, and a masked score (-infinity times zero) no number."""
    c = _Case()
    c.a.scale = scale
    assert both(c) == (mm.ERR_ARG, mm.ERR_ARG)


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** 127])
@pytest.mark.parametrize("seq_q", [1, 140])
def test_the_ends_of_the_scales_are_taken(scale, seq_q):
    """Scores of nothing beside masked keys: the mean of the valid values."""
    import torch
    q, k, v, _ = attention.make((3, 2, 1, seq_q, 300, 64, 64), torch.bfloat16, seed=41)
    if scale > 1:
        q = q * 0
    n = torch.tensor([300, 77, 0], dtype=torch.int32, device="cuda")
    attention.check_forward(q, k, v, n, scale)


@pytest.mark.parametrize("ns", [1 << 62, (1 << 64) - 1])
def test_limits_that_pass_the_clock_are_refused(ns):
    assert mm.library().mmee_chain_wait_limit(ns) == mm.ERR_ARG


@pytest.mark.parametrize("seconds", [-1.0, float("nan"), float("inf"), 2.0 ** 32])
def test_limits_that_are_no_time_are_refused(seconds):
    with pytest.raises(mm.MmeeError) as e:
        mm.mmee_chain_wait_limit(seconds)
    assert e.value.code == mm.ERR_ARG

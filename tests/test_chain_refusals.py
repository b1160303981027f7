"""Calls of the chains through the C interface that are refused before anything is launched (no GPU)."""
import pytest

import paper_2604_03446_b200 as mm
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

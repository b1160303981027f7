"""Gradients in fp16 far from one: what one sequence, head or row holds takes no bits from another's, and what fits the
type neither overflows nor vanishes on the way."""
import math

import pytest
import torch

import paper_2604_03446_b200 as mm
import test_gpu_attention as attention

pytestmark = pytest.mark.gpu


def attention_case(size, seed):
    q, k, v, do = attention.make(size, torch.float16, seed=seed)
    return q, k, v, do


def backward(q, k, v, do, kv_len=None):
    o, saved = mm.mmee_attention(q, k, v, kv_len=kv_len)
    return mm.mmee_attention_backward(do, q, k, v, o, saved, kv_len=kv_len)


@pytest.mark.parametrize("size", [(3, 4, 2, 70, 512, 64, 64), (3, 6, 2, 200, 300, 128, 40), (3, 2, 2, 1, 1000, 72, 128)])
def test_attention_gradients_of_sequences_and_heads_far_apart(size):
    """Every sequence and key head within the bound that its own largest dO and V allow: 2^19 between sequences, 2^4 between heads,
    and a sequence without keys whose dO counts nothing."""
    b, hq, hkv, n, m, dk, dv = size
    q, k, v, do = attention_case(size, 21)
    for i, s in enumerate((2.0 ** 9, 2.0 ** -6, 2.0 ** 11)):
        do[i] *= s
    v[0] *= 2.0 ** 4
    do[:, :, :hq // hkv] *= 2.0 ** -2
    do[:, :, hq // hkv:] *= 2.0 ** 2
    kv_len = torch.tensor([m, m - 5, 0], dtype=torch.int32, device="cuda")
    got = backward(q, k, v, do, kv_len)
    g = hq // hkv
    for i in range(b):
        for h in range(hkv):
            own = (q[i:i + 1, :, h * g:h * g + g], k[i:i + 1, :, h:h + 1], v[i:i + 1, :, h:h + 1])
            want = attention.formulas(*own, kv_len[i:i + 1], 2.0 ** -11, None, do[i:i + 1, :, h * g:h * g + g])
            attention.inside("dq %d %d" % (i, h), got[0][i:i + 1, :, h * g:h * g + g], want["dq"])
            attention.inside("dk %d %d" % (i, h), got[1][i:i + 1, :, h:h + 1], want["dk"])
            attention.inside("dv %d %d" % (i, h), got[2][i:i + 1, :, h:h + 1], want["dv"])


@pytest.mark.parametrize("what", [2.0 ** 13, math.inf])
def test_attention_gradients_depend_on_no_other_sequence_or_head(what):
    q, k, v, do = attention_case((2, 4, 2, 70, 300, 64, 64), 22)
    do *= 2.0 ** -10
    o, saved = mm.mmee_attention(q, k, v)
    want = mm.mmee_attention_backward(do, q, k, v, o, saved)
    other = do.clone()
    other[0, 3] = what                                 # a row of another sequence
    got = mm.mmee_attention_backward(other, q, k, v, o, saved)
    for a, c in zip(got, want):
        assert torch.equal(a[1], c[1])
    other = do.clone()
    other[1, 5, 1] = what                              # a row of another key head's query head
    got = mm.mmee_attention_backward(other, q, k, v, o, saved)
    assert torch.equal(got[0][:, :, 2:], want[0][:, :, 2:])
    for a, c in zip(got[1:], want[1:]):
        assert torch.equal(a[:, :, 1], c[:, :, 1])


def test_an_infinite_row_leaves_the_other_rows_of_its_head():
    """dQ of the other rows is as with zeros in that row's place; its own is no number."""
    q, k, v, do = attention_case((1, 2, 1, 70, 300, 64, 64), 23)
    do *= 2.0 ** -10
    o, saved = mm.mmee_attention(q, k, v)
    do[0, 7, 1] = 0
    want = mm.mmee_attention_backward(do, q, k, v, o, saved)
    do[0, 7, 1] = math.inf
    got = mm.mmee_attention_backward(do, q, k, v, o, saved)
    assert not torch.isfinite(got[0][0, 7, 1]).any()
    assert torch.equal(got[0][0, :, 0], want[0][0, :, 0])
    assert torch.equal(got[0][0, :7], want[0][0, :7]) and torch.equal(got[0][0, 8:], want[0][0, 8:])

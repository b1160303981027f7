"""Waits inside the chains' kernels that run out: every role leaves, what is in flight ends, the status tells, and the next call is a
sound one.  A limit of nothing ends a wait at its first look at the clock, after some 0.35 ms; reductions of millions of values make
the warps that wait for a tile's sums wait longer, while loads and matrix instructions are under way."""
import pytest
import torch

import paper_2604_03446_b200 as mm
import test_gpu_gated_ffn as block

pytestmark = pytest.mark.gpu

# tokens, in, inner, out: which of the kernels has the long reduction
LONG = {
    "pairs of CTAs, parts of the reduction": (130, 8, 1 << 22, 8),
    "single CTAs, gate and up": (130, 1 << 22, 8, 8),
    "few tokens, gate and up": (16, 1 << 22, 128, 8),
    "few tokens, down": (16, 8, 1 << 22, 128),
}


@pytest.fixture
def no_patience():
    mm.mmee_chain_wait_limit(0.0)
    try:
        yield
    finally:
        mm.mmee_chain_wait_limit()


def ran_out():
    with pytest.raises(mm.MmeeError) as e:
        mm.mmee_chain_status()
    assert e.value.code == mm.ERR_TIMEOUT
    mm.mmee_chain_status()                             # (once)


def small_call():
    t = block.make(300, 264, 520, 136, torch.bfloat16, seed=4)
    return block.run(*t, mm.ACT_SILU)


@pytest.mark.parametrize("sizes", LONG.values(), ids=list(LONG))
def test_a_wait_that_runs_out_in_the_block(sizes, no_patience):
    mm.mmee_chain_status()
    want = small_call()
    torch.cuda.synchronize()
    tokens, d_in, d_ff, d_out = sizes
    mk = lambda r, c: torch.zeros(r, c, dtype=torch.bfloat16, device="cuda")
    t = mk(tokens, d_in), mk(d_ff, d_in), mk(d_ff, d_in), mk(d_out, d_ff)
    mm.mmee_gated_ffn(*t)
    ran_out()
    got = small_call()
    for n in want:
        assert torch.equal(got[n], want[n]), n
    mm.mmee_chain_status()
    mm.mmee_chain_wait_limit()
    y, _ = mm.mmee_gated_ffn(*t)                       # with patience
    mm.mmee_chain_status()
    assert (y == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
def test_a_wait_that_runs_out_in_the_gradients(dtype, no_patience):
    """The gradient of hidden, whose kernel has asked for gate and up when its sums do not come."""
    mm.mmee_chain_status()
    tokens, d_in, d_ff, d_out = 130, 8, 8, 1 << 22
    mk = lambda r, c: torch.zeros(r, c, dtype=dtype, device="cuda")
    t = mk(tokens, d_in), mk(d_ff, d_in), mk(d_ff, d_in), mk(d_out, d_ff)
    _, saved = mm.mmee_gated_ffn(*t, save=True)
    mm.mmee_chain_status()
    mm.mmee_gated_ffn_backward(mk(tokens, d_out), *t, saved)
    ran_out()
    small_call()
    mm.mmee_chain_status()
    mm.mmee_chain_wait_limit()
    grads = mm.mmee_gated_ffn_backward(mk(tokens, d_out), *t, saved)
    mm.mmee_chain_status()
    assert all((g == 0).all() for g in grads)


def test_a_short_limit_ends_no_wait_of_ordinary_calls(no_patience):
    """Waits of ordinary sizes take microseconds."""
    want = small_call()
    q, k, v = (torch.randn(2, 300, 4, 64, device="cuda").bfloat16() for _ in range(3))
    o, saved = mm.mmee_attention(q, k, v)
    grads = mm.mmee_attention_backward(o, q, k, v, o, saved)
    mm.mmee_chain_status()
    mm.mmee_chain_wait_limit()
    again = small_call()
    assert all(torch.equal(again[n], want[n]) for n in want)
    for a, b in zip(grads, mm.mmee_attention_backward(o, q, k, v, o, saved)):
        assert torch.equal(a, b)

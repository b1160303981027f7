"""Calls that take what the call before them in the stream writes, with no other kernel between: kernels that start early must not
have read it before."""
import pytest
import torch

import paper_2604_03446_b200 as mm

pytestmark = pytest.mark.gpu


def block_inputs(tokens, d_in, d_ff, d_out, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda r, c, s: (torch.randn(r, c, generator=gen, device="cuda") * s).bfloat16()
    return mk(tokens, d_in, 1.0), mk(d_ff, d_in, d_in ** -0.5), mk(d_ff, d_in, d_in ** -0.5), mk(d_out, d_ff, 4 * d_ff ** -0.5)


def settle(on):
    if on:
        torch.cuda.synchronize()


@pytest.mark.parametrize("tokens", [1, 7, 100, 600])
def test_single_token_attention_reads_what_the_block_has_just_written(tokens):
    heads, d = 4, 64
    cases = [(block_inputs(tokens, 256, 512, heads * d, s), block_inputs(1, 256, 512, 2 * heads * d, s + 50)) for s in range(6)]

    def chain(case, wait):
        kv, q = case
        y, _ = mm.mmee_gated_ffn(*kv)
        settle(wait)
        few, _ = mm.mmee_gated_ffn(*q)
        settle(wait)
        k = y.view(1, tokens, heads, d)
        o, saved = mm.mmee_attention(few.view(1, 1, 2 * heads, d), k, k)
        settle(wait)
        again, _ = mm.mmee_attention(o, o[:, :, :heads], o[:, :, heads:])
        settle(wait)
        return o, saved, again
    want = [chain(c, True) for c in cases]
    for _ in range(5):
        got = [chain(c, False) for c in cases]         # (the same memory again and again)
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


@pytest.mark.parametrize("tokens", [1, 5, 40, 300])
def test_the_block_takes_weights_that_a_call_has_just_written(tokens):
    """Rows of attention's result as the gate's and the down product's weights."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    mk = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    cases = [(mk(1, 128, 2, 64), mk(1, 50, 2, 64), mk(1, 50, 2, 64), mk(tokens, 128)) for _ in range(6)]

    def chain(case, wait):
        q, k, v, x = case
        o, _ = mm.mmee_attention(q, k, v)
        settle(wait)
        w = o.view(128, 128)
        y, saved = mm.mmee_gated_ffn(x, w, w, w, save=True)
        settle(wait)
        return (o, y) + mm.mmee_gated_ffn_backward(y, x, w, w, w, saved)
    want = [chain(c, True) for c in cases]
    for _ in range(5):
        got = [chain(c, False) for c in cases]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(a, b) for a, b in zip(g, w))


def training(x, ws, q, k, v, n):
    """The block on tokens, attention of its rows, both backwards, weights changed in place, twice over."""
    ws = [w.clone() for w in ws]
    out = []
    for _ in range(2):
        y, kept = mm.mmee_gated_ffn(x, *ws, save=True)
        o, saved = mm.mmee_attention(y.view(q.shape), k, v, kv_len=n)
        dq, dk, dv = mm.mmee_attention_backward(q, y.view(q.shape), k, v, o, saved, kv_len=n)
        grads = mm.mmee_gated_ffn_backward(dq.view(y.shape), x, *ws, kept)
        for w, g in zip(ws, grads[1:]):
            w.add_(g, alpha=-2.0 ** -6)
        out += [y, o, dq, dk, dv, *grads]
    return out + ws


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["fp16", "bf16"])
@pytest.mark.parametrize("tokens", [3, 64, 450])
def test_training_steps_without_a_pause_on_streams_and_replayed(tokens, dtype):
    """The same bits as with a pause after every step: eager, on two streams at once, and captured."""
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    mk = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device="cuda") * std).to(dtype)

    def case():
        return (mk(2 * tokens, 192), [mk(520, 192, std=0.07), mk(520, 192, std=0.07), mk(256, 520, std=0.04)],
                mk(2, tokens, 4, 64, std=2.0 ** -8), mk(2, 200, 2, 64), mk(2, 200, 2, 64), torch.tensor([200, 31], dtype=torch.int32, device="cuda"))
    cases = [case() for _ in range(3)]
    want = []
    for c in cases:
        want.append(training(*c))
        torch.cuda.synchronize()
    for _ in range(3):
        got = [training(*c) for c in cases]
        streams = [torch.cuda.Stream() for _ in cases]
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(training(*c))
        torch.cuda.synchronize()
        for i, g in enumerate(got):
            assert all(torch.equal(a, b) for a, b in zip(g, want[i % 3]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = training(*cases[0])
    for _ in range(2):
        for t in out:
            t.zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[0]))
    mm.mmee_chain_status()

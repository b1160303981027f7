"""Gradients in fp16 far from one: what one sequence, head or row holds takes no bits from another's, and what fits the
type neither overflows nor vanishes on the way."""
import math

import pytest
import torch

import paper_2604_03446_b200 as mm
import test_gpu_attention as attention
import test_gpu_gated_ffn as block

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


# --- the gated feed-forward block -----------------------------------------------------------------------------------

U = 2.0 ** -11                             # fp16: half a step, relative


def block_formulas(x, wg, wu, wd, dy, name):
    """The gradients in 64 bits with bounds as in the block's own tests, but for what fp16 loses below its smallest normal value: dg and
    du are kept 2^s larger, where 2^s takes a bound B on them to 2^14 at least (half of that allowed for B's own arithmetic), so
    that they are off by 2^-25 of 2^-s <= 2 B 2^-14; 2^s is at most 2^60.  hidden and the results are off by 2^-25."""
    x, wg, wu, wd, dy = (t.double() for t in (x, wg, wu, wd, dy))
    f = lambda n: n * 2.0 ** -23 + 2.0 ** -22
    n_tok, n_in, n_ff, n_out = x.shape[0], x.shape[1], wg.shape[0], wd.shape[0]
    g, up = x @ wg.T, x @ wu.T
    eg, eu = f(n_in) * (x.abs() @ wg.abs().T), f(n_in) * (x.abs() @ wu.abs().T)
    a, da = block.act64(name, g)
    ea = 1.13 * eg + block.ACT32 * (a.abs() + g.abs() * 2.0 ** -6)
    eda = eg + block.ACT32 * (1 + g.abs())
    if name == "relu":
        eda = torch.where(g.abs() <= eg, torch.ones_like(g), torch.zeros_like(g))
    h = a * up
    eh = ea * (up.abs() + eu) + a.abs() * eu + 2.0 ** -22 * h.abs()
    eh = eh + U * (h.abs() + eh) + 2.0 ** -25
    dh = dy @ wd
    edh = f(n_out) * (dy.abs() @ wd.abs())
    dg, du = dh * up * da, dh * a
    edg = edh * (up * da).abs() + (dh.abs() + edh) * (eu * (da.abs() + eda) + up.abs() * eda)
    edu = edh * (a.abs() + ea) + dh.abs() * ea
    meets = torch.maximum(1.13 * up.abs().amax(1), torch.ones_like(g[:, 0]) if name == "sigmoid" else g.abs().amax(1))
    b = n_out ** 0.5 * float(wd.abs().max()) * float((dy.norm(dim=1) * meets).max())
    lost = 2.0 ** -25 * max(2 * b * 2.0 ** -14, 2.0 ** -60)
    rdg, rdu = (e + U * (t.abs() + e) + lost for t, e in ((dg, edg), (du, edu)))

    def out(value, err, sizes, n):
        err = err + f(n) * sizes
        return value, err + U * (value.abs() + err) + 2.0 ** -25

    return dict(
        d_x=out(dg @ wg + du @ wu, rdg @ wg.abs() + rdu @ wu.abs(), (dg.abs() + rdg) @ wg.abs() + (du.abs() + rdu) @ wu.abs(), 2 * n_ff),
        d_w_gate=out(dg.T @ x, rdg.T @ x.abs(), (dg.abs() + rdg).T @ x.abs(), n_tok),
        d_w_up=out(du.T @ x, rdu.T @ x.abs(), (du.abs() + rdu).T @ x.abs(), n_tok),
        d_w_down=out(dy.T @ h, dy.abs().T @ eh, dy.abs().T @ (h.abs() + eh), n_tok))


def check_block(t, name):
    got = block.run(*t, block.ACTS[name])
    for n, want in block_formulas(*t, name).items():
        block.inside(n, got[n], want)
    mm.mmee_chain_status()


BLOCKS = [(1, 64, 64, 64), (5, 72, 136, 40), (130, 64, 256, 1032), (300, 328, 1000, 520), (200, 2048, 4104, 520), (2100, 264, 1032, 136)]


@pytest.mark.parametrize("size_of_dy", [2.0 ** -20, 2.0 ** -14, 2.0 ** -8, 1.0])
@pytest.mark.parametrize("sizes", BLOCKS, ids=lambda s: "x".join(map(str, s)))
def test_small_gradients_of_the_block(sizes, size_of_dy):
    t = list(block.make(*sizes, torch.float16, seed=31))
    t[4] = (t[4] * size_of_dy).half()
    check_block(t, "silu")


@pytest.mark.parametrize("act", list(block.ACTS))
def test_small_gradients_of_the_block_for_every_activation(act):
    t = list(block.make(300, 72, 200, 136, torch.float16, seed=32, spread=3.0))
    t[4] = (t[4] * 2.0 ** -14).half()
    check_block(t, act)


@pytest.mark.parametrize("sizes", [(5, 72, 136, 40), (300, 72, 200, 136)])
def test_gradients_that_fit_while_those_of_the_gate_do_not(sizes):
    """up of 2^8 under a d_y of 2^8: dg passes 65504, the results do not."""
    x, wg, wu, wd, dy = block.make(*sizes, torch.float16, seed=33)
    t = ((x * 2.0 ** -7).half(), (wg * 2.0 ** -4).half(), (wu * 2.0 ** 15).half(), wd, (dy * 2.0 ** 8).half())
    g = t[4].double() @ wd.double() * (t[0].double() @ t[2].double().T) * 0.5
    most = float(g.abs().max())
    assert most > 65504
    check_block(t, "silu")


def test_what_is_no_number_in_a_token_takes_no_bits_from_the_others():
    t = list(block.make(200, 72, 200, 136, torch.float16, seed=34))
    t[4] = (t[4] * 2.0 ** -14).half()
    rest = [i for i in range(200) if i != 9]
    for which in (0, 4):                               # x, d_y
        bad, none = list(t), list(t)
        bad[which], none[which] = t[which].clone(), t[which].clone()
        bad[which][9], none[which][9] = math.inf, 0
        got, want = (block.run(*v, mm.ACT_SILU)["d_x"] for v in (bad, none))
        assert torch.equal(got[rest], want[rest]) and not torch.isfinite(got[9]).any()

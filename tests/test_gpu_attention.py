"""Attention over states of another length against its formulas in 64 bits, element by element.

Bounds: u = eps / 2 of the type is the most that a rounding is off, relative to the value.  Probabilities are rounded once
before they meet the values and o once: |o_err| <= u P |V| + u |o|.  A score, a 32-bit sum of d products, is off by at most
e = (d + 2) 2^-23 of scale |q| |k| (2^-23: the tensor cores may cut off), its probability by twice the largest e of its row
(numerator and sum) and by 2^-20 of the approximate exponential."""
import math

import pytest
import torch

import paper_2604_03446_b200 as mm

gpu = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

# batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v
SIZES = [
    (1, 1, 1, 1, 1, 8, 8), (1, 1, 1, 1, 2, 64, 64), (2, 2, 1, 1, 17, 16, 24), (1, 12, 12, 1, 512, 64, 64), (3, 8, 2, 1, 300, 128, 128),
    (2, 8, 1, 2, 777, 72, 40), (1, 16, 1, 1, 1000, 128, 64), (1, 2, 2, 16, 65, 40, 128), (1, 1, 1, 8, 5000, 128, 128),
    (1, 4, 4, 17, 128, 64, 64), (2, 4, 2, 64, 129, 64, 128), (1, 2, 1, 100, 127, 128, 64), (1, 1, 1, 127, 1, 96, 96),
    (3, 5, 1, 77, 1501, 72, 40), (1, 3, 3, 128, 128, 128, 128), (2, 2, 2, 129, 255, 64, 64), (1, 2, 2, 255, 256, 128, 128),
    (1, 4, 1, 256, 257, 120, 8), (2, 4, 2, 300, 640, 64, 64), (1, 2, 1, 513, 1025, 128, 128), (1, 1, 1, 200, 9000, 64, 64), (5, 16, 4, 260, 2700, 128, 64),
    (1, 31, 31, 700, 1300, 64, 64),
]


def make(size, dtype, seed=0, spread=1.5):
    b, hq, hkv, n, m, dk, dv = size
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return ((mk(b, n, hq, dk) * spread).to(dtype), mk(b, m, hkv, dk).to(dtype), mk(b, m, hkv, dv).to(dtype), mk(b, n, hq, dv).to(dtype))


def f(n):
    return (n + 2) * 2.0 ** -23


def heads(x, hq):
    """[b, n, h, d] as [b, hq, n, d] in 64 bits, key heads repeated."""
    x = x.double().permute(0, 2, 1, 3)
    return x.repeat_interleave(hq // x.shape[1], dim=1)


def formulas(q, k, v, kv_len, u, scale=None, do=None):
    """name -> (value, bound) in the layouts of the calls."""
    b, n, hq, dk = q.shape
    m, hkv, dv = k.shape[1], k.shape[2], v.shape[3]
    scale = dk ** -0.5 if scale is None else scale
    valid = torch.ones(b, m, dtype=torch.bool, device=q.device) if kv_len is None else torch.arange(m, device=q.device) < kv_len.clamp(0, m)[:, None]
    k, v = (torch.where(valid[:, :, None, None], t, torch.zeros((), dtype=t.dtype, device=t.device)) for t in (k, v))
    Q, K, V = heads(q, hq), heads(k, hq), heads(v, hq)
    ok = valid[:, None, None, :]
    S = (scale * Q @ K.transpose(-1, -2)).masked_fill(~ok, -math.inf)
    top = S.amax(-1, keepdim=True)
    E = torch.exp(S - torch.where(top == -math.inf, 0.0, top))
    L = E.sum(-1, keepdim=True)
    P = E / torch.where(L == 0, 1.0, L)
    lse = torch.where(L == 0, -math.inf, top + torch.log(L))
    es = (f(dk) * scale * Q.abs() @ K.abs().transpose(-1, -2) + 2.0 ** -22 * torch.where(ok, S.abs(), 0.0)) * ok
    worst = es.amax(-1, keepdim=True)
    rel = 2 * worst + 2.0 ** -20 + f(m) * 0.5            # relative error of a probability before its rounding
    O = P @ V
    tiny = 2.0 ** -24
    spread = P @ V.abs()
    eo = (u + rel + f(m)) * spread + tiny
    back = lambda x: x.permute(0, 2, 1, 3)
    out = dict(o=(back(O), back(eo + u * (O.abs() + eo))), lse=(lse[..., 0], (worst + 2.0 ** -20 * (2 + top.abs().nan_to_num(0, 0, 0)))[..., 0]))
    if do is None:
        return out
    D = heads(do, hq)
    dP = D @ V.transpose(-1, -2)
    delta = (D * O).sum(-1, keepdim=True)
    dS = P * (dP - delta) * ok
    edp = f(dv) * (D.abs() @ V.abs().transpose(-1, -2))
    # (delta from o and the rest of its rounding, which is rounded itself: u^2, and 2^-25 in fp16)
    ed = (D.abs() * (eo + u * u * (O.abs() + eo) + 2.0 ** -25)).sum(-1, keepdim=True) + f(dv) * (D.abs() * O.abs()).sum(-1, keepdim=True)
    relp = 2 * worst + 2.0 ** -19 + 2.0 ** -20 * (lse.nan_to_num(0, 0, 0).abs())     # here P = exp(S - lse)
    eds = P * (1 + relp) * (edp + ed + 2.0 ** -22 * (dP.abs() + delta.abs())) + relp * dS.abs()
    # Rounded once to the type; in fp16 what is below the smallest normal value of the scaled dS (2^-14 of at most 2^15) is off by
    # 2^-25 of 2^15 / 2 of the largest dS that the tensors allow.
    biggest = 2 * dv * D.abs().max() * V.abs().max() * 2
    eds = (eds + u * (dS.abs() + eds) + (2.0 ** -39 * biggest if u < 2.0 ** -9 else 0)) * ok
    dQ, edq = scale * dS @ K, scale * (eds @ K.abs() + f(m) * ((dS.abs() + eds) @ K.abs()))
    t = lambda x: x.transpose(-1, -2)
    fold = lambda x: back(x.reshape(b, hkv, hq // hkv, *x.shape[2:]).sum(2))
    N = n * (hq // hkv)
    dK, edk = fold(scale * t(dS) @ Q), fold(scale * (t(eds) @ Q.abs() + f(N) * (t(dS.abs() + eds) @ Q.abs())))
    ep = P * (relp + u) + 2.0 ** -37
    dV, edv = fold(t(P) @ D), fold(t(ep) @ D.abs() + f(N) * (t(P + ep) @ D.abs()))
    rounded = lambda x, e: (x, e + u * (x.abs() + e) + tiny)
    out.update(dq=rounded(back(dQ), back(edq)), dk=rounded(dK, edk), dv=rounded(dV, edv))
    return out


def inside(name, got, want):
    value, bound = want
    same = got.double() == value                          # (infinities)
    off = torch.where(same, 0.0, (got.double() - value).abs() - bound)
    assert not torch.isnan(got).any(), name
    assert float(off.max()) <= 0, "%s: %.3g over the bound" % (name, float(off.max()))


def forward(*args, **kw):
    o, saved = mm.mmee_attention(*args, **kw)
    return o, mm.attention_lse(saved, o)


def check_forward(q, k, v, kv_len=None, scale=None):
    o, lse = forward(q, k, v, kv_len=kv_len, scale=scale)
    want = formulas(q, k, v, kv_len, torch.finfo(q.dtype).eps / 2, scale)
    inside("o", o, want["o"])
    inside("lse", lse, want["lse"])
    return o, lse


@gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward_against_64_bits(size, dtype):
    q, k, v, _ = make(size, TYPES[dtype])
    check_forward(q, k, v)
    mm.mmee_chain_status()


def lengths(b, m, seed):
    edge = [0, 1, m, m // 2, 15, 16, 17, 127, 128, 129, m - 1, -3, m + 5]
    return torch.tensor([edge[(i + seed) % len(edge)] for i in range(b)], dtype=torch.int32, device="cuda")


@gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", [(13, 4, 2, 1, 300, 64, 64), (13, 2, 1, 3, 1000, 128, 40), (13, 2, 2, 40, 260, 72, 128), (13, 4, 2, 140, 300, 128, 128)])
def test_lengths_and_what_lies_behind_them(size, dtype):
    q, k, v, _ = make(size, TYPES[dtype], seed=1)
    n = lengths(size[0], size[4], 0)
    o, lse = check_forward(q, k, v, n)
    behind = torch.arange(size[4], device="cuda") >= n[:, None]
    for junk in (float("nan"), float("inf"), float("-inf")):
        k2, v2 = k.clone(), v.clone()
        k2[behind], v2[behind] = junk, junk
        o2, lse2 = forward(q, k2, v2, kv_len=n)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    empty = (n <= 0).nonzero()[:, 0]
    assert (o[empty] == 0).all() and (lse[empty] == -math.inf).all()


@gpu
@pytest.mark.parametrize("seq_q", [1, 5, 200])
def test_layouts_with_strides(seq_q):
    """Heads before tokens, keys and values side by side, sequences in a larger buffer."""
    b, hq, hkv, m, d = 2, 4, 2, 333, 64
    q, k, v, _ = make((b, hq, hkv, seq_q, m, d, d), torch.bfloat16, seed=2)
    want = forward(q, k, v)
    q2 = q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    both = torch.full((b, m + 3, hkv, 2, d + 8), float("nan"), dtype=q.dtype, device="cuda")
    both[:, :m, :, 0, :d], both[:, :m, :, 1, 8:] = k, v
    got = forward(q2, both[:, :m, :, 0, :d], both[:, :m, :, 1, 8:])
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_scores_far_apart_and_far_from_zero(dtype):
    """Large scores (the running maximum moves often, up and by much), in both directions along the keys, and flat ones."""
    for size in ((1, 2, 1, 3, 2000, 64, 64), (1, 2, 1, 200, 2000, 64, 64)):
        q, k, v, _ = make(size, TYPES[dtype], seed=3)
        ramp = torch.linspace(0.05, 6.0, size[4], device="cuda")[None, :, None, None]
        for s in (ramp, ramp.flip(1)):
            check_forward((q * 3).to(q.dtype), (k * s).to(q.dtype), v)
        check_forward(q * 0, k, v)
        check_forward(q, k, v, scale=0.001)
        check_forward(q, k, v, scale=3.0)


@gpu
def test_infinite_scores_of_valid_keys():
    """A key whose score is -infinity counts nothing; where all are, the row is as one without keys; NaN goes through."""
    for n in (1, 140):
        q = torch.ones(1, n, 1, 64, dtype=torch.bfloat16, device="cuda")
        k = torch.ones(1, 300, 1, 64, dtype=torch.bfloat16, device="cuda")
        v = torch.randn(1, 300, 1, 64, device="cuda").bfloat16()
        k[:, :150] = float("-inf")
        o, lse = forward(q, k, v)
        inside("o", o, formulas(q, k[:, 150:], v[:, 150:], None, 2.0 ** -8)["o"])
        k[:] = float("-inf")
        o, lse = forward(q, k, v)
        assert (o == 0).all() and (lse == -math.inf).all()
        k[:] = 1
        k[0, 77, 0, 3] = float("nan")
        o, lse = forward(q, k, v)
        assert torch.isnan(o).all() and torch.isnan(lse).all()


@gpu
def test_an_offset_beyond_32_bits():
    """Keys of the last sequence lie more than 2^31 elements into their buffer."""
    m, d = 4096, 128
    big = torch.empty(5, 1 << 29, dtype=torch.float16, device="cuda")
    big[4].normal_(generator=torch.Generator(device="cuda").manual_seed(0))
    kv = big[:, :m * 2 * d].view(5, m, 1, 2 * d)
    k, v = kv[..., :d], kv[..., d:]
    k[:4], v[:4] = 0, 0
    assert k.stride(0) * 4 > 2 ** 31 - 1
    for n in (1, 130):
        q = torch.randn(5, n, 2, d, device="cuda").half()
        o, _ = mm.mmee_attention(q, k, v)
        inside("o", o[4:], formulas(q[4:], k[4:], v[4:], None, 2.0 ** -11)["o"])


@gpu
@pytest.mark.parametrize("size", [(2, 8, 2, 1, 3000, 128, 128), (1, 4, 2, 130, 3000, 64, 64)])
def test_same_bits_every_time_on_any_stream_and_replayed(size):
    q, k, v, _ = make(size, torch.bfloat16, seed=4)
    n = torch.tensor([2999, 700][:size[0]], dtype=torch.int32, device="cuda")
    want = forward(q, k, v, kv_len=n)
    torch.cuda.synchronize()
    got = [forward(q, k, v, kv_len=n, stream=torch.cuda.Stream()) for _ in range(4)]
    torch.cuda.synchronize()
    for o, lse in got:
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = forward(q, k, v, kv_len=n)
        graphs.append((graph, out))
    n.copy_(torch.tensor([1234, 2999][:size[0]], dtype=torch.int32))   # read when it is replayed
    want = forward(q, k, v, kv_len=n)
    for graph, out in graphs * 2:
        out[0].zero_()
        graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


# --- gradients ------------------------------------------------------------------------------------------------------

def check_backward(q, k, v, do, kv_len=None, scale=None):
    o, saved = mm.mmee_attention(q, k, v, kv_len=kv_len, scale=scale)
    grads = mm.mmee_attention_backward(do, q, k, v, o, saved, kv_len=kv_len, scale=scale)
    want = formulas(q, k, v, kv_len, torch.finfo(q.dtype).eps / 2, scale, do)
    for name, got in zip(("dq", "dk", "dv"), grads):
        inside(name, got, want[name])
    return o, saved, grads


@gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", [s for s in SIZES if s[4] <= 5000], ids=lambda s: "x".join(map(str, s)))
def test_gradients_against_64_bits(size, dtype):
    q, k, v, do = make(size, TYPES[dtype], seed=11)
    check_backward(q, k, v, do)
    mm.mmee_chain_status()


@gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", [(13, 4, 2, 1, 300, 64, 64), (13, 2, 2, 40, 260, 72, 128), (13, 4, 2, 140, 300, 128, 40)])
def test_gradients_with_lengths_and_what_lies_behind_them(size, dtype):
    q, k, v, do = make(size, TYPES[dtype], seed=12)
    n = lengths(size[0], size[4], 0)
    o, saved, grads = check_backward(q, k, v, do, n)
    behind = torch.arange(size[4], device="cuda") >= n[:, None]
    assert (grads[1][behind] == 0).all() and (grads[2][behind] == 0).all() and (grads[0][n <= 0] == 0).all()
    for junk in (float("nan"), float("inf"), 6e4):
        k2, v2 = k.clone(), v.clone()
        k2[behind], v2[behind] = junk, junk
        for a, b in zip(grads, mm.mmee_attention_backward(do, q, k2, v2, o, saved, kv_len=n)):
            assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("size_of_do", [2.0 ** -20, 2.0 ** -8, 1.0, 2.0 ** 9])
@pytest.mark.parametrize("size_of_v", [2.0 ** -6, 1.0, 2.0 ** 5])
def test_small_and_large_gradients_in_fp16(size_of_do, size_of_v):
    """Gradients far from one: what fits the type does not overflow on the way, and small ones keep their bits."""
    q, k, v, do = make((1, 2, 1, 150, 400, 64, 64), torch.float16, seed=13)
    o, lse = mm.mmee_attention(q, k, (v * size_of_v).half())
    check_backward(q, k, (v * size_of_v).half(), (do * size_of_do).half())


@gpu
def test_gradients_of_long_flat_rows_in_fp16():
    """16384 keys of equal score: probabilities of 2^-14, the edge of fp16's normal values."""
    q, k, v, do = make((1, 1, 1, 130, 16384, 64, 64), torch.float16, seed=14)
    check_backward(q * 0, k, v, do)
    check_backward((q * 0.1).half(), k, v, do)


@gpu
@pytest.mark.parametrize("group", [1, 4])
def test_gradients_against_differences(group):
    """Against central differences of the formula in 64 bits along random directions: <gradient, v> is the derivative along v.
    The bound on the gradient's entries gives sum |v_i| bound_i; what the step leaves is measured by a second, halved one."""
    t = make((2, 2 * group, 2, 9, 33, 24, 16), torch.float16, seed=15)
    n = torch.tensor([33, 20], dtype=torch.int32, device="cuda")
    grads = check_backward(*t, kv_len=n)[2]
    want = formulas(*t[:3], n, 2.0 ** -11, None, t[3])
    base = [x.double() for x in t[:3]]
    gen = torch.Generator(device="cuda").manual_seed(1)

    def value(q, k, v):
        return float((formulas(q, k, v, n, 0.0)["o"][0] * t[3].double()).sum())

    for i, name in enumerate(("dq", "dk", "dv")):
        d = torch.randn(base[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        at = lambda h: value(*[b + h * d if j == i else b for j, b in enumerate(base)])
        d1, d2 = (at(1e-3) - at(-1e-3)) / 2e-3, (at(5e-4) - at(-5e-4)) / 1e-3
        have = float((grads[i].double() * d).sum())
        assert abs(have - (4 * d2 - d1) / 3) <= float((want[name][1] * d.abs()).sum()) + abs(d1 - d2) + 1e-9, name


@gpu
@pytest.mark.parametrize("dtype", list(TYPES))
def test_gradients_same_bits_every_time_strided_and_replayed(dtype):
    b, hq, hkv, n, m, d = 2, 8, 2, 150, 400, 64
    q, k, v, do = make((b, hq, hkv, n, m, d, d), TYPES[dtype], seed=16)
    lens = torch.tensor([400, 130], dtype=torch.int32, device="cuda")
    o, lse = mm.mmee_attention(q, k, v, kv_len=lens)
    want = mm.mmee_attention_backward(do, q, k, v, o, lse, kv_len=lens)
    both = torch.stack((k, v), dim=3)
    flip = lambda x: x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    torch.cuda.synchronize()
    got = [mm.mmee_attention_backward(do, q, k, v, o, lse, kv_len=lens, stream=torch.cuda.Stream()) for _ in range(3)]
    got.append(mm.mmee_attention_backward(flip(do), flip(q), both[:, :, :, 0], both[:, :, :, 1], flip(o), lse, kv_len=lens))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, lse2 = mm.mmee_attention(q, k, v, kv_len=lens)
        got.append(mm.mmee_attention_backward(do, q, k, v, o2, lse2, kv_len=lens))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for g in got:
        for x, y in zip(g, want):
            assert torch.equal(x, y)


# --- refusals: nothing is launched, so that they need no GPU ---------------------------------------------------------

class _Case:
    """Structs of a sound call, with addresses that are never used."""

    def __init__(self):
        from paper_2604_03446_b200 import binding as b
        self.w = b.Workload(batch=2, q_heads=4, kv_heads=2, seq_q=3, seq_kv=5, d_qk=64, d_v=32, word_bytes=2)
        self.a = b.Attention(dtype=b.BF16, scale=0.125, q=4096, k=4096, v=4096, o=4096, q_stride=(768, 256, 64), k_stride=(640, 128, 64),
                             v_stride=(320, 64, 32), o_stride=(384, 128, 32), lse=4096)
        self.g = b.AttentionGrad(4096, 4096, 4096, 4096, (384, 128, 32), (768, 256, 64), (640, 128, 64), (320, 64, 32), 4096, 4096)


BAD = [("w", "batch", 0), ("w", "q_heads", 0), ("w", "kv_heads", 0), ("w", "kv_heads", 3), ("w", "seq_q", 0), ("w", "seq_kv", 0), ("w", "d_qk", 0),
       ("w", "d_v", 0), ("w", "d_qk", 60), ("w", "d_v", 4), ("w", "word_bytes", 1), ("a", "dtype", 2), ("a", "scale", 0.0), ("a", "scale", -1.0),
       ("a", "scale", math.inf), ("a", "scale", math.nan), ("a", "q", 0), ("a", "k", 4104), ("a", "v", 0), ("a", "o", 0), ("a", "o", 4098), ("a", "o_rest", 4104),
       ("a", "q_stride", (768, 0, 64)), ("a", "k_stride", (0, 128, 64)), ("a", "v_stride", (320, 64, 20)), ("a", "o_stride", (384, -128, 32))]


@pytest.mark.parametrize("where,field,value", BAD)
def test_bad_arguments_are_refused(where, field, value):
    c = _Case()
    if isinstance(value, tuple):
        getattr(c.a, field)[:] = value
    else:
        setattr(getattr(c, where), field, value)
    assert mm.library().mmee_attention(c.w, c.a, None) == mm.ERR_ARG
    assert mm.library().mmee_attention_backward(c.w, c.a, c.g, None) == mm.ERR_ARG


@pytest.mark.parametrize("field,value", [("d_o", 0), ("d_o", 4100), ("d_q", 0), ("d_k", 4104), ("d_v", 0), ("d_o_stride", (384, 0, 32)),
                                         ("d_q_stride", (768, 256, 60)), ("d_k_stride", (0, 128, 64)), ("d_v_stride", (320, -64, 32)),
                                         ("workspace", 0), ("workspace", 4104), ("workspace_bytes", 2 * 4 * 3 * 4 + 15)])
def test_bad_gradient_arguments_are_refused(field, value):
    c = _Case()
    if isinstance(value, tuple):
        getattr(c.g, field)[:] = value
    else:
        setattr(c.g, field, value)
    assert mm.library().mmee_attention_backward(c.w, c.a, c.g, None) == mm.ERR_ARG


def test_a_backward_call_without_its_forward_results_is_refused():
    c, lib = _Case(), mm.library()
    assert lib.mmee_attention_backward(c.w, c.a, None, None) == mm.ERR_ARG
    assert lib.mmee_attention_backward_workspace(None, None) == mm.ERR_ARG
    c.a.lse = None
    assert lib.mmee_attention_backward(c.w, c.a, c.g, None) == mm.ERR_ARG


@pytest.mark.parametrize("field,value", [("d_qk", 136), ("d_v", 256), ("batch", 4096), ("q_heads", 65536 * 2), ("seq_kv", 1 << 30)])
def test_sizes_beyond_the_documented_ones_are_refused(field, value):
    c = _Case()
    setattr(c.w, field, value)
    assert mm.library().mmee_attention(c.w, c.a, None) == mm.ERR_RANGE


def test_null_arguments_are_refused():
    c, lib = _Case(), mm.library()
    assert lib.mmee_attention(None, c.a, None) == mm.ERR_ARG and lib.mmee_attention(c.w, None, None) == mm.ERR_ARG
    assert lib.mmee_attention_workspace(None, None) == mm.ERR_ARG


def test_tensors_that_do_not_fit_are_refused():
    q, k = torch.zeros(2, 3, 4, 64, dtype=torch.float16), torch.zeros(2, 5, 2, 64, dtype=torch.float16)
    for bad in [(q, k, k), (q[0], k, k), (q, k.bfloat16(), k), (q, k, None)]:
        with pytest.raises(mm.MmeeError) as e:
            mm.mmee_attention(*bad)
        assert e.value.code == mm.ERR_ARG


@gpu
def test_shapes_that_do_not_fit_are_refused():
    q, k, v, _ = make((2, 4, 2, 3, 5, 64, 32), torch.float16)
    n = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    for bad in [(q, k[:1], v), (q, k, v[:, :4]), (q[..., :56], k, v), (q, k[..., ::2], v), (q[:, :, :3], k, v), (q[:, :0], k, v), (q, k[:, :0], v[:, :0]),
                (q, k[:, :, :1].expand(-1, -1, 2, -1), v)]:
        with pytest.raises(mm.MmeeError):
            mm.mmee_attention(*bad)
    for bad in (n.long(), n[:1], n.cpu(), [1, 2], torch.zeros(4, dtype=torch.int32, device="cuda")[::2]):
        with pytest.raises(mm.MmeeError):
            mm.mmee_attention(q, k, v, kv_len=bad)
    with pytest.raises(mm.MmeeError):
        mm.mmee_attention(q, k, v, scale=-1.0)
    o, lse = mm.mmee_attention(q, k, v)
    for bad in [(o[:, :2], o, lse), (o, o[..., :24], lse), (o, o, lse.half()), (o, o, lse[:-1]), (o, o, None), (o.bfloat16(), o, lse)]:
        with pytest.raises(mm.MmeeError):
            mm.mmee_attention_backward(bad[0], q, k, v, bad[1], bad[2])

"""The gated feed-forward block against its formulas in 64 bits, element by element.

Bounds: a value rounded to the operands' type is off by at most u = eps / 2 of it.  hidden is rounded once and y once, so
|dy| <= u (|hidden| |Wd|^T + |y|); the gradients of gate and up are rounded once before they enter a product, whose result is
rounded once.  32-bit sums of n products are off by at most n 2^-23 of the sum of their sizes (2^-23, not 2^-24: the tensor
cores may cut off instead of rounding), and the activations, from approximate exponentials, by 2^-18 of their size."""
import ctypes as C
import math

import pytest
import torch

import paper_2604_03446_b200 as mm

gpu = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
ACTS = {"silu": mm.ACT_SILU, "gelu": mm.ACT_GELU, "relu": mm.ACT_RELU, "sigmoid": mm.ACT_SIGMOID}
ACT32 = 2.0 ** -18

SIZES = [                                  # tokens, in, inner, out
    (1, 64, 64, 64), (1, 8, 8, 8), (8, 4096, 8192, 4096), (2, 16, 8, 24), (5, 72, 136, 40), (8, 256, 512, 256), (9, 264, 520, 8), (16, 1024, 2048, 512),
    (17, 64, 384, 64), (33, 200, 264, 712), (64, 512, 128, 1032), (127, 136, 248, 72), (128, 64, 256, 128), (129, 192, 384, 264),
    (300, 328, 1000, 520), (777, 1000, 2728, 712), (768, 64, 384, 64), (2048, 256, 1024, 512), (1500, 520, 4100 - 4, 1000), (4100, 264, 2056, 136), (200, 2048, 4104, 520), (512, 1024, 4096, 1024),
]


def make(tokens, d_in, d_ff, d_out, dtype, seed=0, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda r, c, s: (torch.randn(r, c, generator=gen, device="cuda") * s).to(dtype)
    return (mk(tokens, d_in, spread), mk(d_ff, d_in, d_in ** -0.5), mk(d_ff, d_in, d_in ** -0.5),
            mk(d_out, d_ff, d_ff ** -0.5), mk(tokens, d_out, 1.0))


def act64(name, g):
    if name == "relu":
        return g.clamp_min(0), (g > 0).double()
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if name == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def formulas(x, wg, wu, wd, dy, name, u):
    """Every output in 64 bits with the bound on its error."""
    x, wg, wu, wd, dy = (t.double() for t in (x, wg, wu, wd, dy))
    g, up = x @ wg.T, x @ wu.T
    n_in, n_ff, n_out, n_tok = x.shape[1], wg.shape[0], wd.shape[0], x.shape[0]
    f = lambda n: n * 2.0 ** -23 + 2.0 ** -22
    eg, eu = f(n_in) * (x.abs() @ wg.abs().T), f(n_in) * (x.abs() @ wu.abs().T)     # errors of gate and up
    a, da = act64(name, g)
    # The activations' slopes are at most 1.13, the slopes of their derivatives at most 1 (relu's derivative jumps at 0).
    ea = 1.13 * eg + ACT32 * (a.abs() + g.abs() * 2.0 ** -6)
    eda = eg + ACT32 * (1 + g.abs())
    if name == "relu":
        eda = torch.where(g.abs() <= eg, torch.ones_like(g), torch.zeros_like(g))
    h = a * up
    eh = ea * (up.abs() + eu) + a.abs() * eu + 2.0 ** -22 * h.abs()
    ehr = eh + u * (h.abs() + eh) + 2.0 ** -24                                       # rounded (2^-24: the smallest of fp16)
    y = h @ wd.T
    dh = dy @ wd
    edh = f(n_out) * (dy.abs() @ wd.abs())
    dg, du = dh * up * da, dh * a
    edg = edh * (up * da).abs() + dh.abs() * (eu * (da.abs() + eda) + up.abs() * eda) + edh * (eu * (da.abs() + eda) + up.abs() * eda)
    edu = edh * (a.abs() + ea) + dh.abs() * ea
    rdg, rdu = (e + u * (t.abs() + e) + 2.0 ** -24 for t, e in ((dg, edg), (du, edu)))
    dx = dg @ wg + du @ wu

    def out(value, err, sizes, n):
        err = err + f(n) * sizes
        return value, err + u * (value.abs() + err) + 2.0 ** -24

    return dict(
        hidden=(h, ehr),
        y=out(y, ehr @ wd.abs().T, (h.abs() + ehr) @ wd.abs().T, n_ff),
        d_x=out(dx, rdg @ wg.abs() + rdu @ wu.abs(), (dg.abs() + rdg) @ wg.abs() + (du.abs() + rdu) @ wu.abs(), 2 * n_ff),
        d_w_gate=out(dg.T @ x, rdg.T @ x.abs(), (dg.abs() + rdg).T @ x.abs(), n_tok),
        d_w_up=out(du.T @ x, rdu.T @ x.abs(), (du.abs() + rdu).T @ x.abs(), n_tok),
        d_w_down=out(dy.T @ h, dy.abs().T @ ehr, dy.abs().T @ (h.abs() + ehr), n_tok))


def inside(name, got, want):
    value, bound = want
    off = (got.double() - value).abs() - bound
    assert not torch.isnan(got).any(), name
    assert float(off.max()) <= 0, "%s: %.3g over the bound" % (name, float(off.max()))


def run(x, wg, wu, wd, dy, act):
    y, saved = mm.mmee_gated_ffn(x, wg, wu, wd, activation=act, save=True)
    grads = mm.mmee_gated_ffn_backward(dy, x, wg, wu, wd, saved, activation=act)
    return dict(zip(("y", "hidden", "d_x", "d_w_gate", "d_w_up", "d_w_down"), (y, saved[0]) + grads))


@gpu
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_block_and_gradients_against_64_bits(sizes, dtype):
    t = make(*sizes, TYPES[dtype])
    got = run(*t, mm.ACT_SILU)
    torch.cuda.synchronize()
    for name, want in formulas(*t, "silu", torch.finfo(TYPES[dtype]).eps / 2).items():
        inside(name, got[name], want)
    y, saved = mm.mmee_gated_ffn(*t[:4])
    assert saved is None and torch.equal(y, got["y"])
    mm.mmee_chain_status()


@gpu
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("sizes", [(3, 64, 72, 64), (150, 72, 200, 136)])
def test_activations(sizes, act):
    t = make(*sizes, torch.bfloat16, seed=3, spread=4.0)
    got = run(*t, ACTS[act])
    for name, want in formulas(*t, act, 2.0 ** -8).items():
        inside(name, got[name], want)


def naive(x, wg, wu, wd, act):
    a, _ = act64(act, x @ wg.T)
    return (a * (x @ wu.T)) @ wd.T


@gpu
@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_gradients_against_differences(act):
    """The gradients against central differences of the block in 64 bits along random directions: the derivative along v is
    <gradient, v>.  A gradient of n rounded entries g_i gives at most sum |v_i| bound_i; step h leaves h^2 |f'''| / 6, which a
    second, halved step measures (Richardson)."""
    t = make(40, 64, 72, 48, torch.float16, seed=5)
    got = run(*t, ACTS[act])
    bounds = formulas(*t, act, 2.0 ** -11)
    x, wg, wu, wd, dy = (v.double() for v in t)
    names = ("d_x", "d_w_gate", "d_w_up", "d_w_down")
    base = [x, wg, wu, wd]
    gen = torch.Generator(device="cuda").manual_seed(9)
    for i, name in enumerate(names):
        v = torch.randn(base[i].shape, generator=gen, device="cuda", dtype=torch.float64)

        def at(h):
            return float((naive(*[b + h * v if j == i else b for j, b in enumerate(base)], act) * dy).sum())

        d1, d2 = (at(1e-3) - at(-1e-3)) / 2e-3, (at(5e-4) - at(-5e-4)) / 1e-3
        want, left = (4 * d2 - d1) / 3, abs(d1 - d2)
        have = float((got[name].double() * v).sum())
        assert abs(have - want) <= float((bounds[name][1] * v.abs()).sum()) + left + 1e-9, name


@gpu
def test_rows_with_strides_and_a_window_of_a_larger_buffer():
    """Inputs that are columns of wider buffers; the outputs' surroundings stay as they were (they are tensors of their own)."""
    x, wg, wu, wd, dy = make(77, 136, 200, 72, torch.bfloat16, seed=2)

    def wide(m, left, right):
        buf = torch.full((m.shape[0], left + m.shape[1] + right), float("nan"), dtype=m.dtype, device="cuda")
        buf[:, left:left + m.shape[1]] = m
        return buf[:, left:left + m.shape[1]]

    want = run(x, wg, wu, wd, dy, mm.ACT_SILU)
    got = run(wide(x, 8, 16), wide(wg, 24, 0), wide(wu, 0, 8), wide(wd, 16, 40), wide(dy, 8, 8), mm.ACT_SILU)
    for n in want:
        assert torch.equal(want[n], got[n]), n


@gpu
def test_same_bits_every_time_on_any_stream_and_replayed():
    t = make(300, 264, 520, 136, torch.bfloat16, seed=4)
    want = run(*t, mm.ACT_SILU)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:                                   # at once, each on a stream of its own
        y, saved = mm.mmee_gated_ffn(*t[:4], save=True, stream=s)
        got.append((y, saved, mm.mmee_gated_ffn_backward(t[4], *t[:4], saved, stream=s)))
    torch.cuda.synchronize()
    for y, saved, grads in got:
        assert torch.equal(y, want["y"]) and torch.equal(saved[0], want["hidden"])
        for n, g in zip(("d_x", "d_w_gate", "d_w_up", "d_w_down"), grads):
            assert torch.equal(g, want[n]), n
    graphs = []
    for _ in range(2):                                  # two graphs, whose workspaces are their own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run(*t, mm.ACT_SILU)
        graphs.append((graph, out))
    for _ in range(2):
        for graph, out in graphs:
            for v in out.values():
                v.zero_()
            graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        for n in want:
            assert torch.equal(want[n], out[n]), n


@gpu
def test_infinities_and_nan_stay_in_their_rows():
    t = list(make(40, 64, 128, 64, torch.bfloat16, seed=6))
    want, _ = mm.mmee_gated_ffn(*t[:4])
    x = t[0].clone()
    x[7], x[33, 5] = float("nan"), float("inf")
    got, _ = mm.mmee_gated_ffn(x, *t[1:4])
    rest = [i for i in range(40) if i not in (7, 33)]
    assert torch.equal(got[rest], want[rest])
    assert torch.isnan(got[7]).all() and not torch.isfinite(got[33]).any()


# --- refusals: nothing is launched, so that they need no GPU ---------------------------------------------------------

class _Case:
    """Structs of a sound call, with addresses that are never used."""

    def __init__(self):
        from paper_2604_03446_b200 import binding as b
        self.b = b
        self.w = b.Workload(batch=1, q_heads=1, kv_heads=1, seq_q=4, seq_kv=64, d_qk=32, d_v=16, word_bytes=2)
        self.f = b.GatedFfn(dtype=b.BF16, activation=0, x=4096, w_gate=4096, w_up=4096, w_down=4096, x_stride=32, w_gate_stride=32,
                            w_up_stride=32, w_down_stride=64, hidden=4096, kept=4096, y=4096, workspace=4096, workspace_bytes=4 * 4 * 64)
        self.g = b.GatedFfnGrad(4096, 16, 4096, 4096, 4096, 4096)


BAD = [("w", "batch", 2), ("w", "q_heads", 2), ("w", "kv_heads", 2), ("w", "seq_q", 0), ("w", "seq_kv", 0), ("w", "d_qk", 0),
       ("w", "d_v", 0), ("w", "d_qk", 36), ("w", "seq_kv", 60), ("w", "d_v", 12), ("w", "word_bytes", 4),
       ("f", "dtype", 2), ("f", "activation", 4), ("f", "x", 0), ("f", "x", 4104), ("f", "w_gate", 0), ("f", "w_up", 8),
       ("f", "w_down", 0), ("f", "x_stride", 24), ("f", "x_stride", 36), ("f", "w_down_stride", 56), ("f", "w_gate_stride", -32),
       ("f", "hidden", 0), ("f", "hidden", 4098)]


@pytest.mark.parametrize("where,field,value", BAD)
def test_bad_arguments_are_refused(where, field, value):
    c = _Case()
    setattr(getattr(c, where), field, value)
    lib = mm.library()
    assert lib.mmee_gated_ffn(c.w, c.f, None) == mm.ERR_ARG
    assert lib.mmee_gated_ffn_backward(c.w, c.f, c.g, None) == mm.ERR_ARG


@pytest.mark.parametrize("field,value", [("d_y", 0), ("d_y", 4100), ("d_y_stride", 8), ("d_y_stride", 20), ("d_x", 0), ("d_w_gate", 0),
                                         ("d_w_up", 4100), ("d_w_down", 0), ("kept", 0), ("kept", 4100)])
def test_bad_gradient_arguments_are_refused(field, value):
    c = _Case()
    setattr(c.f if field == "kept" else c.g, field, value)
    assert mm.library().mmee_gated_ffn_backward(c.w, c.f, c.g, None) == mm.ERR_ARG


def test_null_and_missing_arguments_are_refused():
    c, lib = _Case(), mm.library()
    assert lib.mmee_gated_ffn(None, c.f, None) == mm.ERR_ARG and lib.mmee_gated_ffn(c.w, None, None) == mm.ERR_ARG
    assert lib.mmee_gated_ffn_backward(c.w, c.f, None, None) == mm.ERR_ARG
    assert lib.mmee_gated_ffn_workspace(None, 0, None) == mm.ERR_ARG
    c.f.y = None
    assert lib.mmee_gated_ffn(c.w, c.f, None) == mm.ERR_ARG
    c.f.kept = None
    assert lib.mmee_gated_ffn_backward(c.w, c.f, c.g, None) == mm.ERR_ARG
    c = _Case()
    c.w.seq_q = 1 << 28
    assert lib.mmee_gated_ffn(c.w, c.f, None) == mm.ERR_RANGE


def test_tensors_that_do_not_fit_are_refused():
    x, w, d = torch.zeros(4, 32, dtype=torch.bfloat16), torch.zeros(64, 32, dtype=torch.bfloat16), torch.zeros(16, 64, dtype=torch.bfloat16)
    for bad in [(x, w, w, d), (x.float(), w.float(), w.float(), d.float()), (x[0], w, w, d), (x, w.half(), w, d), (x, w, w, None)]:
        with pytest.raises(mm.MmeeError) as e:
            mm.mmee_gated_ffn(*bad)
        assert e.value.code == mm.ERR_ARG


@gpu
def test_a_workspace_that_is_missing_short_or_unaligned_is_refused():
    """(The sizes of workspaces go by the device, so that the check comes after one.)"""
    lib, need = mm.library(), C.c_uint64()
    c = _Case()
    for tokens in (4, 300):
        c.w.seq_q = tokens
        for backward in (0, 1):
            assert lib.mmee_gated_ffn_workspace(c.w, backward, need) == mm.OK
            if not need.value:
                continue
            for at, size in ((0, need.value), (4104, need.value), (4096, need.value - 1)):
                c.f.workspace, c.f.workspace_bytes = at, size
                code = lib.mmee_gated_ffn_backward(c.w, c.f, c.g, None) if backward else lib.mmee_gated_ffn(c.w, c.f, None)
                assert code == mm.ERR_ARG
    assert lib.mmee_gated_ffn_workspace(c.w, 2, need) == mm.ERR_ARG


@gpu
def test_shapes_that_do_not_fit_are_refused():
    x, wg, wu, wd, dy = make(4, 32, 64, 16, torch.bfloat16)
    _, saved = mm.mmee_gated_ffn(x, wg, wu, wd, save=True)
    bad_forward = [(x, wg, wu[:56], wd), (x[:, :24], wg, wu, wd), (x, wg, wu, wd[:, :56]), (x.T, wg, wu, wd), (x[:0], wg, wu, wd),
                   (x, wg.cpu(), wu, wd), (x, wg, wu, wd[::1, ::2])]
    for bad in bad_forward:
        with pytest.raises(mm.MmeeError):
            mm.mmee_gated_ffn(*bad)
    for s in [(saved[0][:3], saved[1]), (saved[0], saved[1][:1]), (saved[0], saved[1].bfloat16()), (saved[0].half(), saved[1])]:
        with pytest.raises(mm.MmeeError):
            mm.mmee_gated_ffn_backward(dy, x, wg, wu, wd, s)
    with pytest.raises(mm.MmeeError):
        mm.mmee_gated_ffn_backward(dy[:, :8], x, wg, wu, wd, saved)

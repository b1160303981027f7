"""The chains run together, as a decoder layer would use them, and beside the search of their mapping."""
import pytest
import torch

import mmee_inputs as mi
import paper_2604_03446_b200 as mm

pytestmark = pytest.mark.gpu
U = 2.0 ** -8                              # bf16: half a step, relative


def inputs(batch=2, tokens=70, states=333, heads=8, kv_heads=2, d=64, d_ff=520, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device="cuda") * std).bfloat16()
    width = heads * d
    return dict(q=mk(batch, tokens, heads, d), k=mk(batch, states, kv_heads, d), v=mk(batch, states, kv_heads, d),
                w_gate=mk(d_ff, width, std=width ** -0.5), w_up=mk(d_ff, width, std=width ** -0.5), w_down=mk(width, d_ff, std=d_ff ** -0.5),
                dy=mk(batch * tokens, width), kv_len=torch.tensor([states, states // 3], dtype=torch.int32, device="cuda"))


def layer(t):
    """Attention over the states, then the block on its output, then both backwards."""
    o, saved = mm.mmee_attention(t["q"], t["k"], t["v"], kv_len=t["kv_len"])
    x = o.view(-1, o.shape[2] * o.shape[3])
    w = t["w_gate"], t["w_up"], t["w_down"]
    y, kept = mm.mmee_gated_ffn(x, *w, save=True)
    dx, dwg, dwu, dwd = mm.mmee_gated_ffn_backward(t["dy"], x, *w, kept)
    dq, dk, dv = mm.mmee_attention_backward(dx.view(o.shape), t["q"], t["k"], t["v"], o, saved, kv_len=t["kv_len"])
    return dict(o=o, y=y, dx=dx, dwg=dwg, dwu=dwu, dwd=dwd, dq=dq, dk=dk, dv=dv)


def layer64(t):
    """The same through autograd in 64 bits."""
    p = {n: t[n].double().requires_grad_() for n in ("q", "k", "v", "w_gate", "w_up", "w_down")}
    b, n, h, d = p["q"].shape
    m, hk = p["k"].shape[1:3]
    ok = torch.arange(m, device="cuda") < t["kv_len"][:, None]
    k, v = (p[i].repeat_interleave(h // hk, dim=2) for i in ("k", "v"))
    s = torch.einsum("bnhd,bmhd->bhnm", p["q"], k) * d ** -0.5
    o = torch.einsum("bhnm,bmhd->bnhd", s.masked_fill(~ok[:, None, None], float("-inf")).softmax(-1), v)
    x = o.reshape(b * n, h * d)
    y = (torch.nn.functional.silu(x @ p["w_gate"].T) * (x @ p["w_up"].T)) @ p["w_down"].T
    names = ("q", "k", "v", "w_gate", "w_up", "w_down")
    grads = torch.autograd.grad(y, [o] + [p[i] for i in names], t["dy"].double())
    return dict(zip(("o", "y", "dx", "dq", "dk", "dv", "dwg", "dwu", "dwd"), (o.detach(), y.detach(), grads[0].reshape(b * n, h * d)) + grads[1:]))


def test_a_layer_and_its_gradients_against_64_bits():
    """Each result passes through at most seven roundings in a row (P, o, hidden, y; or o, hidden, dg, dx, P, dS, the result), each at
    most U of the value it meets, on operands of independent sign: in the 2-norm, seven times U bounds their sum."""
    t = inputs()
    got, want = layer(t), layer64(t)
    for n in want:
        off = float((got[n].double() - want[n]).norm() / want[n].norm())
        assert off <= 7 * U, (n, off)


def test_a_captured_layer_replays_with_other_inputs_beside_eager_calls():
    t = inputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer(t)
    for seed in (1, 2):
        other = inputs(seed=seed)
        want = layer(other)
        for n in t:
            t[n].copy_(other[n])
        graph.replay()
        eager = layer(other)                           # on the same stream, behind the replay
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(out[n], want[n]) and torch.equal(eager[n], want[n]), n


def test_a_capture_in_which_copies_and_fills_come_between():
    """Kernels that start early wait for whatever is before them: copies, fills, other kernels, searches."""
    t, src = inputs(), inputs(seed=7)
    cfg = mi.config1()
    h = mm.mmee_create(cfg["workload"], cfg["arch"], cfg["searches"][0])
    buf = mm.result_buffer(1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for n in t:
            t[n].zero_()
        for n in t:
            t[n].copy_(src[n])
        first = layer(t)
        mm.mmee_search(h, buf)
        t["q"].copy_(first["o"])
        second = layer(t)
        t["q"].fill_(0)
    want = layer(src)
    src2 = dict(src, q=want["o"])
    want2 = layer(src2)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    mm.mmee_destroy(h)
    for n in want:
        assert torch.equal(first[n], want[n]) and torch.equal(second[n], want2[n]), n
    assert float(t["q"].abs().max()) == 0


def test_calls_that_feed_each_other_and_reuse_their_memory():
    """Every call's output is the next one's input, its weights even, in place: none may start to read or write before."""
    t = inputs(heads=4, kv_heads=4, d=64, d_ff=256)    # width 256
    def chain(clone):
        x = t["q"].clone()
        w = [t[n].clone() for n in ("w_gate", "w_up", "w_down")]
        for _ in range(6):
            o, saved = mm.mmee_attention(x, t["k"], t["v"], kv_len=t["kv_len"])
            rows = o.view(-1, 256)
            y, kept = mm.mmee_gated_ffn(rows, *w, save=True)
            few, _ = mm.mmee_gated_ffn(rows[:5], *w)
            grads = mm.mmee_gated_ffn_backward(y, rows, *w, kept)
            x.copy_(y.view(x.shape))
            x[0, :5] = few.view(5, 4, 64)
            for p, g in zip(w, grads[1:]):
                p.add_(g, alpha=-1e-3)
            if clone:
                torch.cuda.synchronize()
        return x, w
    a, b = chain(True), chain(False)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and all(torch.equal(p, q) for p, q in zip(a[1], b[1]))


def test_two_layers_at_once_on_two_streams():
    a, b = inputs(seed=3), inputs(seed=4, tokens=33, states=1000)
    want = layer(a), layer(b)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        for s, t in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(layer(t))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        for n in g:
            assert torch.equal(g[n], want[i % 2][n]), n
    mm.mmee_chain_status()


def test_a_searched_workload_runs():
    """The workload of a search is the shape of the call: BERT-base attention, and a two-GEMM chain as a gated block."""
    import bench
    cfg = mi.config2()
    h = mm.mmee_create(cfg["workload"], cfg["arch"], cfg["searches"][0])
    best, _ = mm.mmee_search_host(h)
    mm.mmee_destroy(h)
    (line,) = bench.run_chains("bert", [(cfg, s) for s in cfg["searches"]], [best, best], steps=1)
    assert line["call"] == "mmee_attention" and line["mapping_idx"] == best.idx and line["ms"] > 0
    chain = [c for c in mi.beyond_attention_configs() if c["name"] == "mlp_768_64_384_64"][0]
    (line,) = bench.run_chains("beyond", [(chain, chain["searches"][0])], [best], steps=1)
    assert line["call"] == "mmee_gated_ffn" and line["ms"] > 0


def test_searches_and_chains_on_one_stream():
    cfg = mi.config1()
    t = inputs(seed=5)
    want = layer(t)
    buf = mm.result_buffer(1)
    h = mm.mmee_create(cfg["workload"], cfg["arch"], cfg["searches"][0])
    try:
        records = []
        for _ in range(4):
            mm.mmee_search(h, buf)
            got = layer(t)
            records.append(buf.clone())
        torch.cuda.synchronize()
    finally:
        mm.mmee_destroy(h)
    for n in want:
        assert torch.equal(got[n], want[n]), n
    assert all(torch.equal(r, records[0]) for r in records)


@pytest.mark.parametrize("device", range(1, 2))
def test_tensors_of_another_device_than_the_current_one(device):
    if torch.cuda.device_count() <= device:
        pytest.skip("one device")
    t = {n: v.to("cuda:%d" % device) for n, v in inputs().items()}
    got, want = layer(t), layer(inputs())
    for n in want:
        assert got[n].device.index == device and torch.equal(got[n].cpu(), want[n].cpu()), n

"""What the C interface of the chains allows and the Python entry points never pass: results in any order of strides within larger
buffers, no lse, no rest of o."""
import ctypes as C

import pytest
import torch

import paper_2604_03446_b200 as mm
import test_gpu_attention as attention
from paper_2604_03446_b200 import binding as b

pytestmark = pytest.mark.gpu
TYPES = attention.TYPES

# batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v: few rows (one cluster, several), tiles (whole, cut up and joined)
SIZES = [(2, 4, 2, 1, 300, 64, 64), (1, 2, 1, 2, 20000, 128, 72), (3, 4, 2, 40, 260, 72, 40), (1, 2, 1, 130, 3000, 128, 128), (2, 2, 2, 300, 640, 64, 64)]


class Window:
    """A tensor of this shape within a larger buffer of a mark, its dimensions but the last in another order."""

    def __init__(self, shape, dtype, order, pad=8):
        n = [s + 1 for s in shape[:3]]
        self.buffer = torch.full([n[i] for i in order] + [shape[3] + 2 * pad], 7.0, dtype=dtype, device="cuda")
        back = [order.index(i) for i in range(3)] + [3]
        self.view = self.buffer.permute(back)[:shape[0], :shape[1], :shape[2], pad:pad + shape[3]]

    def surroundings_untouched(self):
        rest = self.buffer.clone()
        rest.as_strided(self.view.shape, self.view.stride(), self.view.storage_offset()).fill_(7.0)
        return bool((rest == 7.0).all())


def call(q, k, v, o, lse=None, rest=None, kv_len=None):
    """mmee_attention by its C interface; the struct's workspace is kept with it."""
    batch, seq_q, q_heads, d_qk = q.shape
    w = b.Workload(batch=batch, q_heads=q_heads, kv_heads=k.shape[2], seq_q=seq_q, seq_kv=k.shape[1], d_qk=d_qk, d_v=v.shape[3], word_bytes=2)
    need = C.c_uint64()
    assert mm.library().mmee_attention_workspace(w, need) == mm.OK
    space = torch.empty(max(16, need.value), dtype=torch.uint8, device="cuda")
    ptr = lambda t: None if t is None else t.data_ptr()
    s = lambda t: (C.c_int64 * 3)(*t.stride()[:3])
    a = b.Attention(dtype=b.BF16 if q.dtype is torch.bfloat16 else b.F16, scale=d_qk ** -0.5, q=ptr(q), k=ptr(k), v=ptr(v), o=ptr(o),
                    q_stride=s(q), k_stride=s(k), v_stride=s(v), o_stride=s(o), lse=ptr(lse), o_rest=ptr(rest), kv_len=ptr(kv_len),
                    workspace=ptr(space), workspace_bytes=need.value)
    assert mm.library().mmee_attention(w, a, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == mm.OK
    return w, a, space


def lengths(size):
    return torch.tensor([size[4], size[4] // 3, 0][:size[0]], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (2, 1, 0), (1, 0, 2)], ids=str)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_results_in_any_order_of_strides_and_without_the_parts_for_the_backward_pass(size, dtype, order):
    q, k, v, do = attention.make(size, TYPES[dtype], seed=51)
    n = lengths(size)
    want, saved = mm.mmee_attention(q, k, v, kv_len=n)
    o = Window(want.shape, q.dtype, order)
    w, a, _ = call(q, k, v, o.view, kv_len=n)          # no lse, no rest
    torch.cuda.synchronize()
    assert torch.equal(o.view, want) and o.surroundings_untouched()
    lse, rest = torch.zeros_like(mm.attention_lse(saved, want)), torch.zeros_like(want)
    for with_lse, with_rest in ((lse, None), (None, rest), (lse, rest)):
        o.view.zero_()
        call(q, k, v, o.view, with_lse, with_rest, n)
        assert torch.equal(o.view, want)
    assert torch.equal(lse, mm.attention_lse(saved, want))

    # the gradients, with and without what o's rounding took off, into windows
    grads = mm.mmee_attention_backward(do, q, k, v, want, saved, kv_len=n)
    need = C.c_uint64()
    assert mm.library().mmee_attention_backward_workspace(w, need) == mm.OK
    space = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    s = lambda t: (C.c_int64 * 3)(*t.stride()[:3])
    for given in (rest, None):
        outs = [Window(t.shape, t.dtype, order) for t in (q, k, v)]
        a.lse, a.o_rest = lse.data_ptr(), None if given is None else given.data_ptr()
        g = b.AttentionGrad(do.data_ptr(), *[t.view.data_ptr() for t in outs], s(do), *[s(t.view) for t in outs], space.data_ptr(), need.value)
        assert mm.library().mmee_attention_backward(w, a, g, C.c_void_p(torch.cuda.current_stream().cuda_stream)) == mm.OK
        torch.cuda.synchronize()
        assert all(t.surroundings_untouched() for t in outs)
        if given is not None:
            for t, x in zip(outs, grads):
                assert torch.equal(t.view, x)
        else:
            # delta is then from the rounded o: another rounding of o, u |o| at most, in its bound
            u = torch.finfo(q.dtype).eps / 2
            exact = attention.formulas(q, k, v, n, u, None, do)
            D, O = do.double().abs(), want.double().abs()
            ed = (D * u * O).sum(-1).permute(0, 2, 1)[..., None]           # batch, head, token, 1
            valid = torch.arange(size[4], device="cuda") < n.clamp(0)[:, None]
            zero = lambda t: torch.where(valid[:, :, None, None], t, torch.zeros_like(t))
            Q, K = attention.heads(q, size[1]), attention.heads(zero(k), size[1])
            S = (q.shape[3] ** -0.5 * Q @ K.transpose(-1, -2)).masked_fill(~valid[:, None, None, :], float("-inf"))
            P = torch.nan_to_num(S.softmax(-1), 0.0)
            more = P * ed * (1 + 2.0 ** -6) * q.shape[3] ** -0.5           # (1 + 2^-6: its share of dS's own rounding, of P's error)
            group = size[1] // size[2]
            fold = lambda x: x.reshape(size[0], size[2], group, *x.shape[2:]).sum(2).permute(0, 2, 1, 3)
            dq, dk = (more @ K.abs()).permute(0, 2, 1, 3), fold(more.transpose(-1, -2) @ Q.abs())
            attention.inside("dq", outs[0].view, (exact["dq"][0], exact["dq"][1] + dq * (1 + u)))
            attention.inside("dk", outs[1].view, (exact["dk"][0], exact["dk"][1] + dk * (1 + u)))
            assert torch.equal(outs[2].view, grads[2])
    mm.mmee_chain_status()

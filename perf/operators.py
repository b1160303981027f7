"""The chains that a mapping is searched for, run on this GPU: cross attention and the gated feed-forward block, each
forward, with its gradients, and for single tokens.

A case names the call, the sizes in the words of a workload (queries, keys, heads, widths) and the type.  The seed makes
the inputs; which sequences of a batch are short is the seed's choice too, how short they are is the case's.

  attention        one forward pass over a batch of encoder states, some of them padded
  attention_train  the forward pass and the gradients of queries, keys and values
  ffn              down( act(x Wg^T) * (x Wu^T) )
  ffn_train        the same with the gradients of the input and of the three weights
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _attention(name, train, batch, q_heads, kv_heads, seq_q, seq_kv, d_qk, d_v, dtype, lengths="full", packed=False):
    case = dict(call="attention_train" if train else "attention", batch=batch, q_heads=q_heads, kv_heads=kv_heads,
                seq_q=seq_q, seq_kv=seq_kv, d_qk=d_qk, d_v=d_v, dtype=dtype, lengths=lengths, packed=packed)
    return dict(case, name=name) if name else case


def _ffn(name, train, tokens, d_in, d_ff, d_out, dtype, activation="silu"):
    case = dict(call="ffn_train" if train else "ffn", tokens=tokens, d_in=d_in, d_ff=d_ff, d_out=d_out, dtype=dtype,
                activation=activation)
    return dict(case, name=name) if name else case


def listed():
    return [
        # One decoded token over the encoder states of a single short request: the call whose latency a user waits for.
        _attention("attn_token_s512_h12_d64", False, 1, 12, 12, 1, 512, 64, 64, "fp16"),
        # A batch of decoded tokens over long, ragged encoder states, four query heads to a key head: bound by the memory.
        _attention("attn_tokens_b32_gqa_s8192", False, 32, 32, 8, 1, 8192, 128, 128, "bf16", "ragged"),
        # A BERT-sized batch: short queries over padded states.
        _attention("attn_fwd_b16_q128_kv512_d64", False, 16, 12, 12, 128, 512, 64, 64, "fp16", "ragged"),
        # Odd everything: widths that are no power of two, five query heads to a key head, one request without any state.
        _attention("attn_fwd_odd_d72_d40", False, 3, 10, 2, 77, 1501, 72, 40, "bf16", "empty"),
        # A long prompt over a longer context: bound by the tensor cores.
        _attention("attn_fwd_gqa_q4096_kv8192", False, 1, 32, 8, 4096, 8192, 128, 128, "bf16"),
        # A BERT-sized training step over padded states.
        _attention("attn_train_b8_q384_kv512_d64", True, 8, 12, 12, 384, 512, 64, 64, "fp16", "ragged"),
        # A training step with grouped heads, keys and values side by side in one projection's output.
        _attention("attn_train_gqa_q2048_kv4096", True, 2, 32, 8, 2048, 4096, 128, 128, "bf16", "full", True),
        # One token through a large feed-forward block: the weights are read once.
        _ffn("ffn_token_4096_16384", False, 1, 4096, 16384, 4096, "bf16"),
        # A few tokens through a block of ragged widths.
        _ffn("ffn_tokens13_2048_5464", False, 13, 2048, 5464, 2048, "fp16"),
        # A prompt through the large block.
        _ffn("ffn_fwd_4096_16384", False, 4096, 4096, 16384, 4096, "bf16"),
        # A small training step, ragged tokens and widths, another width out than in.
        _ffn("ffn_train_odd_777", True, 777, 1000, 2728, 712, "fp16", "gelu"),
        # A training step of the large block.
        _ffn("ffn_train_4096_16384", True, 4096, 4096, 16384, 4096, "bf16"),
    ]


def _length(rng, lo, hi):
    """A length between lo and hi, even over the logarithm: a power of two, a multiple of 8, or any number."""
    n = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    kind = rng.randrange(3)
    if kind == 0:
        return min(hi, max(lo, 1 << round(math.log2(n))))
    return min(hi, max(lo, round(n / 8) * 8 if kind == 1 else round(n)))


def draw(rng):
    while True:
        dtype = rng.choice(("bf16", "fp16"))
        call = rng.choice(("token", "attention", "attention", "attention_train", "attention_train", "ffn_tokens", "ffn",
                           "ffn_train"))
        if call in ("token", "attention", "attention_train"):
            kv_heads = rng.choice((1, 2, 4, 8, 12))
            group = rng.choice((1, 1, 2, 4, 5, 8))
            d_qk = rng.choice((16, 40, 64, 64, 72, 96, 128, 128))
            train = call == "attention_train"      # (over one key alone, the gradients of queries and keys are nothing)
            case = _attention("", train, _length(rng, 1, 32), kv_heads * group, kv_heads,
                              _length(rng, 1, 4) if call == "token" else _length(rng, 1, 4096),
                              _length(rng, 16 if train else 1, 16384 if call == "token" else 8192), d_qk,
                              d_qk if rng.random() < 0.7 else rng.choice((8, 32, 64, 80, 128)), dtype,
                              rng.choice(("full", "ragged", "empty")), rng.random() < 0.3)
        else:
            widths = [max(64, 8 * round(_length(rng, 64, hi) / 8)) for hi in (4096, 16384, 4096)]
            case = _ffn("", call == "ffn_train", _length(rng, 1, 64 if call == "ffn_tokens" else 4096), *widths, dtype,
                        rng.choice(("silu", "silu", "gelu", "relu", "sigmoid")))
        w = work(case)
        most = 6e11 if case["call"] == "attention" else 1.2e12 if case["call"] == "attention_train" else 5e12
        # the scores of the plain form stay within a few GB
        if w["flops"] <= most and w["bytes"] < 2e9 and (
                "tokens" in case or case["batch"] * case["q_heads"] * case["seq_q"] * case["seq_kv"] <= 1 << 30):
            return case


def _lengths(case):
    """Valid keys of each sequence, in ascending order."""
    b, n = case["batch"], case["seq_kv"]
    if case["lengths"] == "full":
        return [n] * b
    first = 0 if case["lengths"] == "empty" else 1
    return [max(min(first, n), n * (i + first) // (b - 1 + first)) if b > 1 else (n * first + 1) // 2 for i in range(b)]


def prepare(case, seed):
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)

    if case["call"].startswith("attention"):
        b, sq, skv, hq, hkv, dk, dv = (case[n] for n in ("batch", "seq_q", "seq_kv", "q_heads", "kv_heads", "d_qk", "d_v"))
        # Queries a little wider than the keys, so that a row has keys that count and keys that do not.
        state = dict(call=case["call"], q=normal(b, sq, hq, dk, std=2.0), kv_len=None)
        if case["packed"]:
            both = normal(b, skv, hkv, dk + dv)
            state.update(k=both[..., :dk], v=both[..., dk:])
        else:
            state.update(k=normal(b, skv, hkv, dk), v=normal(b, skv, hkv, dv))
        if case["lengths"] != "full":
            lengths = _lengths(case)
            rng.shuffle(lengths)
            state["kv_len"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        if case["call"] == "attention_train":
            state["do"] = normal(b, sq, hq, dv)
        return state
    n, di, df, do = (case[k] for k in ("tokens", "d_in", "d_ff", "d_out"))
    state = dict(call=case["call"], activation=case["activation"], x=normal(n, di),
                 w_gate=normal(df, di, std=di ** -0.5), w_up=normal(df, di, std=di ** -0.5),
                 w_down=normal(do, df, std=df ** -0.5))
    if case["call"] == "ffn_train":
        state["dy"] = normal(n, do)
    return state


# --- the plain forms: 32 bits throughout, rounded once at the end ---------------------------------------------------

def _stacked(x, hkv):
    """[batch, tokens, heads, width] as [batch, key heads, (query heads of that key head, tokens), width] in 32 bits."""
    b, n, h, d = x.shape
    return x.float().reshape(b, n, hkv, h // hkv, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, h // hkv * n, d)


def _unstacked(x, n, dtype):
    b, hkv, rows, d = x.shape
    return x.reshape(b, hkv, rows // n, n, d).permute(0, 3, 1, 2, 4).reshape(b, n, -1, d).to(dtype)


def _plain_attention(s):
    q, k, v = s["q"], s["k"], s["v"]
    (b, n, _, dk), hkv, m = q.shape, k.shape[2], k.shape[1]
    scale = dk ** -0.5
    qs, ks, vs = _stacked(q, hkv), _stacked(k, hkv), _stacked(v, hkv)
    scores = qs @ ks.transpose(-1, -2) * scale
    if s["kv_len"] is not None:
        valid = torch.arange(m, device=q.device) < s["kv_len"][:, None]
        scores = scores.masked_fill(~valid[:, None, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = (scores - torch.where(top == -math.inf, 0.0, top)).exp()
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-30)
    o = p @ vs
    if "do" not in s:
        return _unstacked(o, n, q.dtype)
    do = _stacked(s["do"], hkv)
    ds = p * (do @ vs.transpose(-1, -2) - (do * o).sum(-1, keepdim=True)) * scale
    return dict(o=_unstacked(o, n, q.dtype), dq=_unstacked(ds @ ks, n, q.dtype),
                dk=_unstacked(ds.transpose(-1, -2) @ qs, m, q.dtype), dv=_unstacked(p.transpose(-1, -2) @ do, m, q.dtype))


def _act(name, g):
    """The activation and its derivative."""
    if name == "relu":
        return g.clamp_min(0), (g > 0).to(g.dtype)
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    sig = 1 / (1 + torch.exp(-g))
    return (sig, sig * (1 - sig)) if name == "sigmoid" else (g * sig, sig * (1 + g * (1 - sig)))


def _plain_ffn(s):
    x, wg, wu, wd = (s[n].float() for n in ("x", "w_gate", "w_up", "w_down"))
    dtype = s["x"].dtype
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(s["activation"], g)
    h = a * u
    y = (h @ wd.T).to(dtype)
    if "dy" not in s:
        return y
    dy = s["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    return dict(y=y, dx=(dg @ wg + du @ wu).to(dtype), dw_gate=(dg.T @ x).to(dtype), dw_up=(du.T @ x).to(dtype),
                dw_down=(dy.T @ h).to(dtype))


def run(state):
    if own:
        import paper_2604_03446_b200 as mm
        s = state
        if s["call"] == "attention":
            return mm.mmee_attention(s["q"], s["k"], s["v"], kv_len=s["kv_len"])[0]
        if s["call"] == "attention_train":
            o, lse = mm.mmee_attention(s["q"], s["k"], s["v"], kv_len=s["kv_len"])
            dq, dk, dv = mm.mmee_attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, kv_len=s["kv_len"])
            return dict(o=o, dq=dq, dk=dk, dv=dv)
        w = s["w_gate"], s["w_up"], s["w_down"]
        act = {"silu": mm.ACT_SILU, "gelu": mm.ACT_GELU, "relu": mm.ACT_RELU, "sigmoid": mm.ACT_SIGMOID}[s["activation"]]
        if s["call"] == "ffn":
            return mm.mmee_gated_ffn(s["x"], *w, activation=act)[0]
        y, saved = mm.mmee_gated_ffn(s["x"], *w, activation=act, save=True)
        dx, dwg, dwu, dwd = mm.mmee_gated_ffn_backward(s["dy"], s["x"], *w, saved, activation=act)
        return dict(y=y, dx=dx, dw_gate=dwg, dw_up=dwu, dw_down=dwd)
    return _plain_attention(state) if state["call"].startswith("attention") else _plain_ffn(state)


def work(case):
    train = case["call"].endswith("_train")
    if case["call"].startswith("attention"):
        keys, dk, dv = sum(_lengths(case)), case["d_qk"], case["d_v"]
        rows = case["seq_q"] * case["q_heads"]
        queries, states = rows * case["batch"] * (dk + dv), keys * case["kv_heads"] * (dk + dv)
        # Forward S = Q K^T and P V; the gradients S again (it is not kept), dO V^T, dS K, dS^T Q and P^T dO.  Read q, k, v
        # and write o; with gradients dO in, dq, dk, dv out.
        flops = 2 * rows * keys * ((dk + dv) + (3 * dk + 2 * dv if train else 0))
        return dict(bytes=2 * (queries + states) * (2 if train else 1), flops=flops)
    n, di, df, do = (case[k] for k in ("tokens", "d_in", "d_ff", "d_out"))
    weights = df * (2 * di + do)
    # Three products forward and two for each of them backward.  Read the weights, x, write y; with gradients dy in and dx
    # and the weights' gradients out.
    return dict(bytes=2 * (weights + n * (di + do)) * (2 if train else 1), flops=2 * n * weights * (3 if train else 1))


# --- 64 bits, from the definitions ----------------------------------------------------------------------------------

def _exact_attention(s):
    q, k, v, do = (s[n].double() if n in s else None for n in ("q", "k", "v", "do"))
    b, n, hq, dk = q.shape
    m, hkv = k.shape[1:3]
    grads = do is not None
    o = q.new_zeros(b, n, hq, v.shape[3])
    dq, dkk, dvv = torch.zeros_like(q), torch.zeros(k.shape, dtype=k.dtype, device=k.device), torch.zeros(v.shape, dtype=v.dtype, device=v.device)
    for i in range(b):
        c = m if s["kv_len"] is None else int(s["kv_len"][i])
        if c == 0:
            continue
        for h in range(hq):
            j = h * hkv // hq
            p = torch.softmax(q[i, :, h] @ k[i, :c, j].T / math.sqrt(dk), dim=-1)
            o[i, :, h] = p @ v[i, :c, j]
            if grads:
                dp = do[i, :, h] @ v[i, :c, j].T
                ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(dk)
                dq[i, :, h] = ds @ k[i, :c, j]
                dkk[i, :c, j] += ds.T @ q[i, :, h]
                dvv[i, :c, j] += p.T @ do[i, :, h]
    return dict(o=o, dq=dq, dk=dkk, dv=dvv) if grads else o


def exact(case, seed):
    s = prepare(case, seed)
    if case["call"].startswith("attention"):
        return _exact_attention(s)
    x, wg, wu, wd = (s[n].double().requires_grad_("dy" in s) for n in ("x", "w_gate", "w_up", "w_down"))
    with torch.set_grad_enabled("dy" in s):
        g = torch.nn.functional.linear(x, wg)
        a = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu,
             "sigmoid": torch.sigmoid}[case["activation"]](g)
        y = torch.nn.functional.linear(a * torch.nn.functional.linear(x, wu), wd)
    if "dy" not in s:
        return y
    dx, dwg, dwu, dwd = torch.autograd.grad(y, (x, wg, wu, wd), s["dy"].double())
    return dict(y=y.detach(), dx=dx, dw_gate=dwg, dw_up=dwu, dw_down=dwd)

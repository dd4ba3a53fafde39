"""Operators of a transformer block around the sketched layers: what a program does with them, over the
range of sizes they are used at.

A case is one operator and one pass through it.  ``op`` names the operator:

"attention"   softmax attention of packed heads, q [batch, q_len, heads, head_dim] on k, v [batch, k_len,
              kv_heads, head_dim]; ``ragged`` batches have a length for each sequence
"norm_rope"   RMS norm of every query and key head with the position rotation in the same pass
"embedding"   rows of a table by token, scaled
"dropout"     dropout by a counter-based generator, with a residual added

``train`` is the forward pass and the gradients of every floating input, otherwise the forward pass
alone.  Stored as "bf16" or "f32"; sums are in 32 bits either way.  Where ``own`` is false, ``run`` does
the same with elementary torch operations in 32 bits.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _attention(name, train, batch, q_len, k_len, heads, kv_heads, head_dim, causal=False, ragged=False, dtype="bf16"):
    c = {"op": "attention", "train": train, "batch": batch, "q_len": q_len, "k_len": k_len, "heads": heads,
         "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "ragged": ragged, "dtype": dtype}
    return dict(name=name, **c) if name else c


def _norm_rope(name, train, tokens, heads, kv_heads, head_dim, rotary, interleaved=False, dtype="bf16"):
    c = {"op": "norm_rope", "train": train, "tokens": tokens, "heads": heads, "kv_heads": kv_heads,
         "head_dim": head_dim, "rotary": rotary, "interleaved": interleaved, "dtype": dtype}
    return dict(name=name, **c) if name else c


def _embedding(name, train, tokens, rows, width, dtype="bf16"):
    c = {"op": "embedding", "train": train, "tokens": tokens, "rows": rows, "width": width, "dtype": dtype}
    return dict(name=name, **c) if name else c


def _dropout(name, train, tokens, width, p, residual=True, dtype="bf16"):
    c = {"op": "dropout", "train": train, "tokens": tokens, "width": width, "p": p, "residual": residual, "dtype": dtype}
    return dict(name=name, **c) if name else c


def listed():
    return [
        # a small model in full precision, as in a first experiment or a unit test: latency only
        _attention("attn_train_tiny_f32", True, 4, 16, 16, 4, 4, 64, dtype="f32"),
        # training step of a BERT-base encoder: 32 padded sentences of up to 128 tokens
        _attention("attn_train_sentences", True, 32, 128, 128, 12, 12, 64, ragged=True),
        # the same of a BERT-large encoder on whole passages
        _attention("attn_train_passages", True, 16, 512, 512, 16, 16, 64),
        # training step of an LLM with 4096 features, 16384 tokens, keys shared by four query heads each
        _attention("attn_train_llm", True, 4, 4096, 4096, 32, 8, 128, causal=True),
        # an LLM of 8192 features reads the next piece of a prompt, of odd length, behind what it has cached
        _attention("attn_prompt_odd", False, 1, 1001, 3001, 64, 8, 128, causal=True),
        # it generates: eight sequences of all lengths, an idle one among them, a token each
        _attention("attn_decode", False, 8, 1, 16384, 64, 8, 128, ragged=True),
        # queries and keys of the LLM's training step on their way to attention, and back
        _norm_rope("norm_rope_train_llm", True, 16384, 32, 8, 128, 128),
        # and of its generation: latency only
        _norm_rope("norm_rope_decode", False, 8, 64, 8, 128, 128),
        # token embeddings of ragged sentences packed together, in full precision
        _embedding("embed_train_sentences_f32", True, 4001, 32000, 768, dtype="f32"),
        # an LLM's, whose table is large beside the tokens of a step
        _embedding("embed_train_llm", True, 16384, 65536, 4096),
        # behind a projection of a BERT-base layer
        _dropout("dropout_train_sentences", True, 4096, 768, 0.1),
        # behind one of an LLM, an odd number of tokens
        _dropout("dropout_train_llm", True, 16383, 4096, 0.05),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of ``step`` between lo and hi, spread over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def _draw_attention(rng):
    kind = rng.choice(["sentences", "sentences", "documents", "documents", "f32", "prompt", "decode"])
    kv, group, d = rng.choice([1, 2, 4, 8]), rng.choice([1, 1, 2, 4, 8]), rng.choice([32, 64, 64, 80, 96, 128, 128])
    ragged, dtype, causal, train = rng.random() < 0.5, "bf16", True, True
    if kind == "sentences":
        batch, q, kv, group, causal = _log(rng, 2, 64), _log(rng, 8, 768), rng.choice([4, 8, 12, 16]), 1, False
        k = q
    elif kind == "documents":
        batch, q = _log(rng, 1, 8), _log(rng, 256, 4096)
        k = q
    elif kind == "f32":
        batch, q, dtype, causal = _log(rng, 1, 16), _log(rng, 4, 512), "f32", rng.random() < 0.5
        k = q
    elif kind == "prompt":
        batch, q, train = _log(rng, 1, 4), _log(rng, 2, 2048), False
        k = q + _log(rng, 1, 8192) - 1
    else:
        batch, q, train, ragged = _log(rng, 1, 32), rng.choice([1, 1, 1, 2, 3]), False, True
        k = _log(rng, 16, 32768)
    make = lambda b: _attention(None, train, b, q, k, kv * group, kv, d, causal, ragged, dtype)  # noqa: E731
    most = work(listed()[3])["flops"] / 4   # (the plain form computes masked pairs too)
    while batch > 1 and (2 * q * k * batch * kv * group * d * (7 if train else 2) > most or batch * k * kv * d > 1 << 27):
        batch -= 1
    return make(batch)


def draw(rng):
    op = rng.choice(["attention", "attention", "norm_rope", "embedding", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "attention":
        return _draw_attention(rng)
    if op == "norm_rope":
        train = rng.random() < 0.6
        d = rng.choice([32, 64, 80, 128, 128])
        kv = rng.choice([1, 2, 4, 8])
        return _norm_rope(None, train, _log(rng, 64, 12288) if train else _log(rng, 1, 4096), kv * rng.choice([1, 2, 4]), kv, d,
                          rng.choice([d, d, d // 2]), rng.random() < 0.3, dtype)
    if op == "embedding":
        train = rng.random() < 0.7
        return _embedding(None, train, _log(rng, 1, 32768), _log(rng, 100, 60000), _log(rng, 64, 2048, 8), dtype)
    return _dropout(None, rng.random() < 0.7, _log(rng, 1, 16384), _log(rng, 64, 2048), rng.choice([0.05, 0.1, 0.2, 0.5]),
                    rng.random() < 0.7, dtype)


def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly: which sequence has which goes by the seed."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lengths(c):
    """The queries' and keys' lengths of a case's sequences, in some order."""
    if not c["ragged"]:
        return [c["q_len"]] * c["batch"], [c["k_len"]] * c["batch"]
    if c["train"]:
        n = _spread(c["batch"], max(1, c["q_len"] // 16), c["q_len"])
        return n, n
    # serving: every query counts, on caches filled to various lengths (none at all in an idle slot)
    return [c["q_len"]] * c["batch"], _spread(c["batch"], 0 if c["q_len"] == 1 else c["q_len"], c["k_len"])


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _prepare_attention(c, seed):
    g, dtype = _generator(seed), _TORCH[c["dtype"]]
    B, Tq, Tk, H, Hkv, D = c["batch"], c["q_len"], c["k_len"], c["heads"], c["kv_heads"], c["head_dim"]
    # normed and rotated queries and keys; values come out of the projection beside them, and out of a
    # cache when generating
    q = _normal(g, (B, Tq, H, D), 1.5, dtype)
    kv = _normal(g, (B, Tk, 2, Hkv, D), 1.0, dtype)
    k, v = kv[:, :, 0], kv[:, :, 1]
    s = {"case": c, "q": q, "k": k, "v": v, "q_lengths": None, "k_lengths": None}
    if c["ragged"]:
        order = list(range(B))
        random.Random(seed).shuffle(order)
        ql, kl = (torch.tensor([n[i] for i in order], dtype=torch.int32, device="cuda") for n in _lengths(c))
        s["k_lengths"] = kl
        if c["train"]:
            s["q_lengths"] = ql
    if c["train"]:
        for t in (q, k, v):
            t.requires_grad_()
        s["do"] = _normal(g, (B, Tq, H, D), 1.0, dtype)
    return s


def _prepare_norm_rope(c, seed):
    g, dtype = _generator(seed), _TORCH[c["dtype"]]
    T, H, Hkv, D = c["tokens"], c["heads"], c["kv_heads"], c["head_dim"]
    # slices of one projection's output
    qkv = _normal(g, (T, H + 2 * Hkv, D), 1.0, dtype)
    q, k = qkv[:, :H], qkv[:, H:H + Hkv]
    context = 4096
    angle = torch.arange(context, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, c["rotary"], 2, device="cuda") / c["rotary"])
    s = {"case": c, "q": q, "k": k, "cos": torch.cos(angle), "sin": torch.sin(angle),
         "wq": (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype), "wk": (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype),
         "positions": torch.arange(T, device="cuda") % context if c["train"] else torch.randint(0, context, (T,), generator=g, device="cuda")}
    if c["train"]:
        for n in ("q", "k", "wq", "wk"):
            s[n].requires_grad_()
        s["dq"], s["dk"] = _normal(g, (T, H, D), 1.0, dtype), _normal(g, (T, Hkv, D), 1.0, dtype)
    return s


def _prepare_embedding(c, seed):
    g, dtype = _generator(seed), _TORCH[c["dtype"]]
    # tokens by rank: each about as frequent as its rank's inverse, as words are
    u = torch.rand(c["tokens"], generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(c["rows"] + 1)) - 1).long().clamp_(0, c["rows"] - 1)
    s = {"case": c, "ids": ids, "table": _normal(g, (c["rows"], c["width"]), 0.02, dtype), "scale": math.sqrt(c["width"])}
    if c["train"]:
        s["table"].requires_grad_()
        s["dy"] = _normal(g, (c["tokens"], c["width"]), 1.0, dtype)
    return s


def _prepare_dropout(c, seed):
    g, dtype = _generator(seed), _TORCH[c["dtype"]]
    shape = (c["tokens"], c["width"])
    s = {"case": c, "x": _normal(g, shape, 1.0, dtype), "residual": _normal(g, shape, 1.0, dtype) if c["residual"] else None,
         "seed": (0x9E3779B97F4A7C15 * (seed + 1)) % 2 ** 63, "offset": seed % 1000 + (1 << 33)}
    if c["train"]:
        s["x"].requires_grad_()
        s["dy"] = _normal(g, shape, 1.0, dtype)
    return s


def prepare(case, seed):
    return {"attention": _prepare_attention, "norm_rope": _prepare_norm_rope, "embedding": _prepare_embedding,
            "dropout": _prepare_dropout}[case["op"]](case, seed)


@functools.lru_cache(None)
def _block():
    from paper_2601_15473_amd import block
    return block


def _run_attention(s):
    c = s["case"]
    o = _block().attention(s["q"], s["k"], s["v"], q_lengths=s["q_lengths"], k_lengths=s["k_lengths"], causal=c["causal"])
    if not c["train"]:
        return o
    dq, dk, dv = torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"])
    return {"o": o.detach(), "dq": dq, "dk": dk, "dv": dv}


def _run_norm_rope(s):
    c = s["case"]
    q, k = _block().head_norm_rope(s["q"], s["k"], s["wq"], s["wk"], s["cos"], s["sin"], s["positions"], eps=EPS, interleaved=c["interleaved"])
    if not c["train"]:
        return {"q": q, "k": k}
    dq, dk, dwq, dwk = torch.autograd.grad((q, k), (s["q"], s["k"], s["wq"], s["wk"]), (s["dq"], s["dk"]))
    return {"q": q.detach(), "k": k.detach(), "dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def _run_embedding(s):
    y = _block().embedding(s["ids"], s["table"], scale=s["scale"])
    if not s["case"]["train"]:
        return y
    return {"y": y.detach(), "dtable": torch.autograd.grad(y, s["table"], s["dy"])[0]}


def _run_dropout(s):
    y = _block().dropout(s["x"], s["case"]["p"], s["seed"], s["offset"], residual=s["residual"])
    if not s["case"]["train"]:
        return y
    return {"y": y.detach(), "dx": torch.autograd.grad(y, s["x"], s["dy"])[0]}


# ---- the same in elementary operations ----


def _seen(c, ql, kl):
    """Which key each query sees, [batch or 1, 1, q_len, k_len]: the last query of a sequence stands at its last key."""
    i, j = torch.arange(c["q_len"], device="cuda")[:, None], torch.arange(c["k_len"], device="cuda")
    ql = torch.full((1,), c["q_len"], device="cuda") if ql is None else ql
    kl = torch.full((1,), c["k_len"], device="cuda") if kl is None else kl
    ql, kl = ql.view(-1, 1, 1, 1), kl.view(-1, 1, 1, 1)
    ok = (i < ql) & (j < kl)
    return ok & (j - kl <= i - ql) if c["causal"] else ok


def _plain_attention(s):
    c, dtype = s["case"], s["q"].dtype
    B, Tk, Hkv, D = c["batch"], c["k_len"], c["kv_heads"], c["head_dim"]
    G, scale = c["heads"] // Hkv, c["head_dim"] ** -0.5
    q = s["q"].detach().float().transpose(1, 2)
    k, v = (s[n].detach().float().transpose(1, 2).repeat_interleave(G, 1) for n in "kv")
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    p.masked_fill_(~_seen(c, s["q_lengths"], s["k_lengths"]), -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, 1.0))
    o = torch.matmul(p, v)
    if not c["train"]:
        return o.transpose(1, 2).to(dtype)
    do = s["do"].float().transpose(1, 2)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    shared = [t.view(B, Hkv, G, Tk, D).sum(2).transpose(1, 2).to(dtype) for t in (dk, dv)]
    return {"o": o.transpose(1, 2).to(dtype), "dq": dq.transpose(1, 2).to(dtype), "dk": shared[0], "dv": shared[1]}


def _pairs(c, x):
    """The rotated features' first and second halves, and the rest."""
    n = c["rotary"]
    if c["interleaved"]:
        return x[..., 0:n:2], x[..., 1:n:2], x[..., n:]
    return x[..., :n // 2], x[..., n // 2:n], x[..., n:]


def _unpaired(c, a, b, rest):
    ab = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((ab, rest), -1)


def _plain_norm_rope_one(c, x, w, cos, sin, dy):
    x, w = x.detach().float(), w.detach().float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    a, b, rest = _pairs(c, x * r * w)
    y = _unpaired(c, a * cos - b * sin, b * cos + a * sin, rest)
    if dy is None:
        return y, None, None
    a, b, rest = _pairs(c, dy.float())
    dn = _unpaired(c, a * cos + b * sin, b * cos - a * sin, rest)
    dw = (dn * x * r).sum((0, 1))
    g = dn * w
    return y, r * g - x * r ** 3 * (g * x).mean(-1, keepdim=True), dw


def _plain_norm_rope(s):
    c, dtype = s["case"], s["q"].dtype
    cos, sin = (s[n][s["positions"]][:, None] for n in ("cos", "sin"))
    q, dq, dwq = _plain_norm_rope_one(c, s["q"], s["wq"], cos, sin, s.get("dq"))
    k, dk, dwk = _plain_norm_rope_one(c, s["k"], s["wk"], cos, sin, s.get("dk"))
    out = {"q": q, "k": k}
    if c["train"]:
        out.update(dq=dq, dk=dk, dwq=dwq, dwk=dwk)
    return {n: t.to(dtype) for n, t in out.items()}


def _plain_embedding(s):
    table, dtype = s["table"].detach(), s["table"].dtype
    y = (table[s["ids"]].float() * s["scale"]).to(dtype)
    if not s["case"]["train"]:
        return y
    d = torch.zeros(table.shape, device="cuda").index_add_(0, s["ids"], s["dy"].float())
    return {"y": y, "dtable": (d * s["scale"]).to(dtype)}


_LOW = 0xFFFFFFFF


def _words(n, seed, offset):
    """The first ``n`` of the generator's 16-bit words: Philox 4x32 with ten rounds (Salmon and others, 2011),
    keyed by the seed, on the counters (i, offset), eight words from each, the lowest bits of a number first."""
    i = torch.arange((n + 7) // 8, device="cuda")
    c = [i & _LOW, i >> 32, torch.full_like(i, offset & _LOW), torch.full_like(i, offset >> 32)]
    for r in range(10):
        k0, k1 = (seed + r * 0x9E3779B9) & _LOW, ((seed >> 32) + r * 0xBB67AE85) & _LOW
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57   # (low 64 bits; the sign is cut off below)
        c = [(b >> 32) & _LOW ^ c[1] ^ k0, b & _LOW, (a >> 32) & _LOW ^ c[3] ^ k1, a & _LOW]
    return torch.stack([c[0] & 0xFFFF, c[0] >> 16, c[1] & 0xFFFF, c[1] >> 16, c[2] & 0xFFFF, c[2] >> 16,
                        c[3] & 0xFFFF, c[3] >> 16], 1).flatten()[:n]


def _plain_dropout(s):
    c, x = s["case"], s["x"].detach()
    drop = round(c["p"] * 65536)    # of 65536 words, those below it
    kept = (_words(x.numel(), s["seed"], s["offset"]) >= drop).view(x.shape) * (65536.0 / (65536 - drop))
    y = x.float() * kept
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not c["train"]:
        return y.to(x.dtype)
    return {"y": y.to(x.dtype), "dx": (s["dy"].float() * kept).to(x.dtype)}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"attention": _run_attention, "norm_rope": _run_norm_rope, "embedding": _run_embedding, "dropout": _run_dropout}[op](state)
    return {"attention": _plain_attention, "norm_rope": _plain_norm_rope, "embedding": _plain_embedding, "dropout": _plain_dropout}[op](state)


# ---- the definitions in 64 bits ----


def _exact_attention(c, s):
    B, Tq, Tk, H, Hkv, D = c["batch"], c["q_len"], c["k_len"], c["heads"], c["kv_heads"], c["head_dim"]
    wide = {n: s[n].detach() for n in ("q", "k", "v")}
    o = torch.zeros((B, Tq, H, D), dtype=torch.float64, device="cuda")
    dq, dk, dv = (torch.zeros(wide[n].shape, dtype=torch.float64, device="cuda") for n in ("q", "k", "v"))
    ql = [Tq] * B if s["q_lengths"] is None else s["q_lengths"].tolist()
    kl = [Tk] * B if s["k_lengths"] is None else s["k_lengths"].tolist()
    for b in range(B):
        n, m = ql[b], kl[b]
        first = max(0, n - m) if c["causal"] else 0   # the first query that sees a key
        if m == 0 or first >= n:
            continue
        for h in range(H):
            Q, K, V = wide["q"][b, first:n, h].double(), wide["k"][b, :m, h * Hkv // H].double(), wide["v"][b, :m, h * Hkv // H].double()
            a = (Q @ K.T) / math.sqrt(D)
            if c["causal"]:
                a = torch.where(torch.ones_like(a).tril(m - n + first) > 0, a, -math.inf)
            w = torch.softmax(a, 1)
            o[b, first:n, h] = w @ V
            if c["train"]:
                g = s["do"][b, first:n, h].double()
                e = g @ V.T
                e = w * (e - (w * e).sum(1, keepdim=True)) / math.sqrt(D)
                dq[b, first:n, h] = e @ K
                dk[b, :m, h * Hkv // H] += e.T @ Q
                dv[b, :m, h * Hkv // H] += w.T @ g
    return {"o": o, "dq": dq, "dk": dk, "dv": dv} if c["train"] else o


def _exact_norm_rope(c, s):
    out = {}
    # the rotation as one complex factor for each pair
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"]][:, None]
    n = c["rotary"]
    one = (lambda t: t[..., 0:n:2]) if c["interleaved"] else (lambda t: t[..., :n // 2])
    two = (lambda t: t[..., 1:n:2]) if c["interleaved"] else (lambda t: t[..., n // 2:n])

    def rotated(t, factor):
        z, r = torch.complex(one(t), two(t)) * factor, t.clone()
        one(r).copy_(z.real)
        two(r).copy_(z.imag)
        return r

    for name in ("q", "k"):
        x, w = s[name].detach().double(), s["w" + name].detach().double()
        size = torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
        u = x / size
        out[name] = rotated(u * w, turn)
        if c["train"]:
            dn = rotated(s["d" + name].double(), turn.conj())
            out["dw" + name] = (dn * u).sum((0, 1))
            du = dn * w
            out["d" + name] = (du - u * (du * u).mean(-1, keepdim=True)) / size
    return out


def _exact_embedding(c, s):
    ids, scale = s["ids"], float(s["scale"])
    y = torch.nn.functional.one_hot(ids, c["rows"]).double() @ s["table"].detach().double() * scale if c["tokens"] * c["rows"] < 1 << 20 \
        else s["table"].detach().double().index_select(0, ids) * scale
    if not c["train"]:
        return y
    order = torch.argsort(ids, stable=True)
    sums = torch.zeros((c["rows"], c["width"]), dtype=torch.float64, device="cuda")
    sums.index_put_((ids[order],), s["dy"].double()[order] * scale, accumulate=True)
    return {"y": y, "dtable": sums}


def _exact_dropout(c, s):
    n, seed, offset, low = s["x"].numel(), s["seed"], s["offset"], np.uint64(0xFFFFFFFF)
    at = np.arange((n + 7) // 8, dtype=np.uint64)
    x0, x1 = at & low, at >> np.uint64(32)
    x2, x3 = np.full_like(at, offset & 0xFFFFFFFF), np.full_like(at, offset >> 32)
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (q >> np.uint64(32)) ^ x1 ^ np.uint64(key[0]), q & low, (p >> np.uint64(32)) ^ x3 ^ np.uint64(key[1]), p & low
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    words = np.stack([x0, x1, x2, x3], 1).astype("<u4").view("<u2").reshape(-1)[:n]
    drop = round(c["p"] * 65536)
    keep = torch.from_numpy((words >= drop).astype(np.float64)).cuda().view(s["x"].shape) / (1 - drop / 65536)
    y = s["x"].detach().double() * keep + (0 if s["residual"] is None else s["residual"].double())
    return {"y": y, "dx": s["dy"].double() * keep} if c["train"] else y


def exact(case, seed):
    return {"attention": _exact_attention, "norm_rope": _exact_norm_rope, "embedding": _exact_embedding,
            "dropout": _exact_dropout}[case["op"]](case, prepare(case, seed))


# ---- what a pass cannot do without ----


def _seen_pairs(c):
    """Pairs of a query and a key it sees, over the batch, of one head."""
    total = 0
    for n, m in zip(*_lengths(c)):
        if not c["causal"]:
            total += n * m
            continue
        see = min(n, m)                      # queries that see a key: the last one all m, each before it one fewer
        total += see * m - see * (see - 1) // 2
    return total


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "attention":
        ql, kl = _lengths(c)
        queries, keys = sum(ql) * c["heads"] * c["head_dim"], sum(kl) * c["kv_heads"] * c["head_dim"]
        outside = c["batch"] * c["q_len"] * c["heads"] * c["head_dim"] - queries        # zeros of o and dq, and of dk and dv below
        flops = (14 if c["train"] else 4) * _seen_pairs(c) * c["heads"] * c["head_dim"]    # two products forward, five back
        if not c["train"]:
            return {"bytes": e * (2 * queries + 2 * keys + outside), "flops": flops}
        padding = c["batch"] * c["k_len"] * c["kv_heads"] * c["head_dim"] - keys
        return {"bytes": e * (4 * queries + 4 * keys + 2 * outside + 2 * padding), "flops": flops}
    if c["op"] == "norm_rope":
        values = c["tokens"] * (c["heads"] + c["kv_heads"]) * c["head_dim"]
        table = min(c["tokens"], 4096) * c["rotary"] * 4 + c["tokens"] * 8
        return {"bytes": e * values * (4 if c["train"] else 2) + table, "flops": values * (20 if c["train"] else 8)}
    if c["op"] == "embedding":
        values, rows = c["tokens"] * c["width"], min(c["tokens"], c["rows"])
        # rows of the table looked up (each token its own at most), the result; dY, the whole gradient
        forward = e * (rows * c["width"] + values) + 8 * c["tokens"]
        return {"bytes": forward + (e * (values + c["rows"] * c["width"]) if c["train"] else 0), "flops": values * (2 if c["train"] else 1)}
    values = c["tokens"] * c["width"]
    return {"bytes": e * values * ((3 if c["residual"] else 2) + (2 if c["train"] else 0)), "flops": values * (4 if c["train"] else 2)}

"""Cases of the operators around the linear layers of a decoder block: what produces a layer's calibration activations,
and the gradients with which the parameters that stay in floating point are tuned after the weights are quantized.

A case is a dict of plain values.  `op` says which calls one pass makes:
    attention        attention of packed sequences of different lengths with grouped heads, from whole prompts to one new
                     token per sequence against its cache
    attention_train  the same with log-sum-exps, then the gradients of q, k and v
    norm             h' = r h + gate * norm(y) and the next block's norm(h'), fused
    norm_grad        the gradients of that from those of h' and of the normalised rows
    clip             the global norm of many gradients, and the gradients scaled to at most max_norm
All inputs are made on the GPU from the seed.  Lengths of sequences and of gradients follow from the case alone.
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _api():
    import paper_2603_28845_amd
    return paper_2603_28845_amd


# ---- cases --------------------------------------------------------------------------------------------------------------
def _attention(name=None, op="attention", **kw):
    """seqs sequences of lo .. hi keys (log-uniform by the number `lens`, the first has hi); queries: "all" as many as
    keys, "one" one per sequence, "some" a part of them (the newest).  slack: the keys lie in a cache that has room for
    that many more behind each sequence.  fused: q, k and v are slices of one projection's output."""
    c = {"op": op, "dtype": "bf16", "seqs": 1, "lo": 1, "hi": 1, "lens": 1, "queries": "all", "heads": 32, "kv_heads": 8, "dim": 128,
         "causal": True, "slack": 0, "fused": False}
    c.update(kw)
    return dict(c, name=name) if name else c


def _norm(name=None, op="norm", **kw):
    """rows x width; y: a block's output joins (else h is normalised as it is); post: it is normalised first; gate: "no",
    "channel" (one factor per channel) or "token" (one per entry); kind: "rms" or "layer" (with biases)."""
    c = {"op": op, "dtype": "bf16", "w_dtype": "bf16", "rows": 1, "width": 4096, "y": True, "post": False, "gate": "no", "scale": 1.0,
         "kind": "rms"}
    c.update(kw)
    return dict(c, name=name) if name else c


def _clip(name=None, **kw):
    """shapes: "block" (the linear layers and norms of a decoder block of width `width`) or "small" (`count` tensors of
    lo .. hi entries).  level: their norm over max_norm."""
    c = {"op": "clip", "dtype": "f32", "shapes": "small", "width": 0, "count": 8, "lo": 1, "hi": 1, "lens": 1, "level": 3.0}
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # generation with a quantized model: 32 requests, one new token each, caches of very different lengths
        _attention("attn_tokens_32x16384", seqs=32, lo=100, hi=16384, queries="one", slack=64),
        # a calibration batch: 32 sequences of 2048 tokens through an 8B-class attention
        _attention("attn_calibration_32x2048", seqs=32, lo=2048, hi=2048, fused=True),
        # prompts as they come: odd lengths from one token on, packed; heads of their own, 80 wide
        _attention("attn_ragged_prompts", seqs=40, lo=1, hi=3001, lens=7, heads=20, kv_heads=20, dim=80),
        # one long document
        _attention("attn_prompt_16384", seqs=1, lo=16384, hi=16384),
        # tuning a block on calibration sequences: forward and gradients
        _attention("attn_train_8x2048", op="attention_train", seqs=8, lo=2048, hi=2048, fused=True),
        # the smallest model's block in fp32, odd lengths, every token sees every other
        _attention("attn_train_ragged_f32", op="attention_train", dtype="f32", seqs=6, lo=33, hi=777, lens=5, heads=8, kv_heads=2, dim=64, causal=False),
        # one step of generation: a few rows, launches and latency only
        _norm("norm_8x4096", rows=8),
        # the calibration batch's residual stream: add the block's output, normalise for the next layers
        _norm("norm_65536x4096", rows=65536),
        # gradients with norms on both sides of the block and a learned scale per channel
        _norm("norm_grad_16384x4096", op="norm_grad", rows=16384, post=True, gate="channel"),
        # the same in fp32 with means and biases, an odd number of odd rows and a gate from a branch
        _norm("norm_grad_3001x1359_f32", op="norm_grad", dtype="f32", w_dtype="f32", rows=3001, width=1359, post=True, gate="token",
              scale=0.5, kind="layer"),
        # all gradients of an 8B-class decoder block
        _clip("clip_block_4096_f32", shapes="block", width=4096),
        # only what stays in floating point next to quantized weights: norms, scales, biases
        _clip("clip_60_small_bf16", dtype="bf16", count=60, lo=1, hi=20000, lens=3),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (5e13 if c["dtype"] == "f32" else 5e14)


def _plain_bytes(c):
    """Size of the padded scores, which bounds what the plain form can hold."""
    if not c["op"].startswith("attention"):
        return 0
    q, k = _lengths(c)
    return 4 * c["seqs"] * c["heads"] * max(q) * max(k)


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["attention", "attention", "attention", "attention_train", "attention_train", "norm", "norm_grad", "clip"])
        if op.startswith("attention"):
            kv = rng.choice([1, 2, 4, 5, 8])
            c = _attention(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), seqs=_log_int(rng, 1, 64), lens=rng.randrange(1000),
                           kv_heads=kv, heads=kv * rng.choice([1, 2, 3, 4, 8]), dim=rng.choice([32, 64, 64, 80, 96, 128, 128]),
                           causal=rng.random() < 0.75, fused=rng.random() < 0.3)
            c["queries"] = "all" if op == "attention_train" else rng.choice(["all", "all", "one", "some"])
            c["hi"] = _log_int(rng, 1, 2048 if op == "attention_train" else 16384)
            c["lo"] = _log_int(rng, 1, c["hi"])
            if op == "attention" and c["queries"] != "all":
                c["fused"] = False
                c["slack"] = rng.choice([0, 1, 64])
        elif op == "clip":
            c = _clip(dtype=rng.choice(["bf16", "f32"]), level=rng.choice([0.5, 3.0, 100.0]), lens=rng.randrange(1000))
            if rng.random() < 0.5:
                c.update(shapes="block", width=_log_int(rng, 256, 4096, 16))
            else:
                c.update(count=rng.randint(1, 60), hi=_log_int(rng, 100, 1 << 20))
        else:
            c = _norm(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), rows=_log_int(rng, 1, 65536), width=_log_int(rng, 64, 14336, rng.choice([1, 16])),
                      y=rng.random() < 0.8, kind=rng.choice(["rms", "rms", "layer"]))
            c["w_dtype"] = "f32" if c["dtype"] == "f32" else rng.choice(["bf16", "f32"])
            if c["y"]:
                c.update(post=rng.random() < 0.5, gate=rng.choice(["no", "channel", "token"]), scale=rng.choice([1.0, 1.0, 0.7]))
        if _cost(c) <= top and _plain_bytes(c) <= 40e9:
            return c


# ---- sizes that follow from the case ------------------------------------------------------------------------------------
def _lengths(case):
    """(queries, keys) of each sequence."""
    rng = random.Random(case["lens"])
    k = [case["hi"]] + [_log_int(rng, case["lo"], case["hi"]) for _ in range(case["seqs"] - 1)]
    q = k if case["queries"] == "all" else [1] * len(k) if case["queries"] == "one" else [_log_int(rng, 1, n) for n in k]
    return q, k


def _starts(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def _shapes(case):
    d = case["width"]
    if case["shapes"] == "block":
        kv, ff = max(16, d // 4), d * 7 // 2
        return [(d, d), (kv, d), (kv, d), (d, d), (ff, d), (ff, d), (d, ff), (d,), (d,)]
    rng = random.Random(case["lens"])
    return [(_log_int(rng, case["lo"], case["hi"]),) for _ in range(case["count"])]


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _normal(gen, *shape, dtype=torch.float32, std=1.0):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype).mul_(std)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _prepare_attention(case, gen, s):
    t, h, g, d = DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"]
    nq, nk = _lengths(case)
    tq, tk = sum(nq), sum(nk) + case["slack"] * len(nk)
    if case["fused"]:
        qkv = _normal(gen, tq, h + 2 * g, d, dtype=t)
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + g], qkv[:, h + g:]
    else:
        s["q"], s["k"], s["v"] = _normal(gen, tq, h, d, dtype=t), _normal(gen, tk, g, d, dtype=t), _normal(gen, tk, g, d, dtype=t)
    s.update(cu_q=_int32(_starts(nq)), cu_k=_int32(_starts([n + case["slack"] for n in nk])), len_k=_int32(nk) if case["slack"] else None,
             max_q=max(nq), max_k=max(nk))
    if case["op"] == "attention_train":
        s["d_out"] = _normal(gen, tq, h, d, dtype=t, std=0.05)


def _prepare_norm(case, gen, s):
    t, w, rows, d = DTYPES[case["dtype"]], DTYPES[case["w_dtype"]], case["rows"], case["width"]
    level = torch.exp(_normal(gen, rows, 1, std=0.5)).to(t)     # tokens differ in size
    big = 1.0 + 19.0 * (torch.rand(d, generator=gen, device=DEV) < 0.005).to(t)   # and some channels stand out
    s["h"] = _normal(gen, rows, d, dtype=t).mul_(level).mul_(big)
    s["y"] = _normal(gen, rows, d, dtype=t, std=0.5).mul_(level) if case["y"] else None
    layer = case["kind"] == "layer"
    par = {"weight": 1.0, "bias": 0.0 if layer else None, "post_weight": 0.3 if case["post"] else None,
           "post_bias": 0.0 if case["post"] and layer else None}
    s["par"] = {n: None if at is None else (_normal(gen, d, std=0.1) + at).to(w) for n, at in par.items()}
    s["gate"] = {"no": lambda: None, "channel": lambda: (_normal(gen, d, std=0.2) + 0.5).to(w), "token": lambda: _normal(gen, rows, d, dtype=t)}[case["gate"]]()
    if case["op"] == "norm_grad":
        s["d_h"], s["d_n"] = _normal(gen, rows, d, dtype=t, std=0.02), _normal(gen, rows, d, dtype=t, std=0.02)


def _prepare_clip(case, gen, s):
    t = DTYPES[case["dtype"]]
    s["grads"] = [_normal(gen, *shape, dtype=t, std=0.01) for shape in _shapes(case)]
    s["out"] = [torch.empty_like(g) for g in s["grads"]]
    s["max_norm"] = 0.01 * math.sqrt(sum(g.numel() for g in s["grads"])) / case["level"]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": case}
    {"attention": _prepare_attention, "attention_train": _prepare_attention, "norm": _prepare_norm, "norm_grad": _prepare_norm,
     "clip": _prepare_clip}[case["op"]](case, gen, s)
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------------
def _padded(x, starts, lengths, longest, groups):
    """Rows of packed sequences as [sequence, longest, groups, heads of a group, dim] in 32 bits, zeros behind the last."""
    at = torch.arange(longest, device=DEV)
    rows = (starts[:-1, None] + at).clamp_(max=x.shape[0] - 1)
    return (x[rows].float() * (at < lengths[:, None])[:, :, None, None]).unflatten(2, (groups, -1))


def _packed(x, starts, total):
    """[sequence, longest, heads, dim] back to the packed rows."""
    token = torch.arange(total, device=DEV)
    seq = torch.searchsorted(starts[1:].contiguous(), token, right=True)
    return x[seq, token - starts[seq]]


def _plain_attention(s):
    case = s["case"]
    g, h, d = case["kv_heads"], case["heads"], case["dim"]
    cu_q, cu_k, lq, lk = s["cu_q"].long(), s["cu_k"].long(), s["max_q"], s["max_k"]
    nq = cu_q.diff()
    nk = cu_k.diff() if s["len_k"] is None else s["len_k"].long()
    n = nq.shape[0]
    # queries of a group of heads lie one below the other: [sequence and group, head and query, dim]
    q = _padded(s["q"], cu_q, nq, lq, g).permute(0, 2, 3, 1, 4).reshape(n * g, -1, d)
    k = _padded(s["k"], cu_k, nk, lk, g).permute(0, 2, 3, 1, 4).reshape(n * g, lk, d)
    v = _padded(s["v"], cu_k, nk, lk, g).permute(0, 2, 3, 1, 4).reshape(n * g, lk, d)
    i, j = torch.arange(lq, device=DEV), torch.arange(lk, device=DEV)
    seen = (j < nk[:, None, None]).expand(n, lq, lk)
    if case["causal"]:
        seen = seen & (j <= i[:, None] + (nk - nq)[:, None, None])
    scale = 1.0 / math.sqrt(d)
    p = torch.bmm(q, k.transpose(1, 2)).mul_(scale)
    heads = p.view(n, h, lq, lk)
    heads.masked_fill_(~seen[:, None], -math.inf)
    top = heads.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    heads.sub_(top).exp_()
    total = heads.sum(3, keepdim=True)
    heads.div_(torch.where(total == 0, 1.0, total))
    out = torch.bmm(p, v)

    def rows(x):     # [sequence and group, head and query, dim] to the packed rows
        return _packed(x.view(n, h, lq, d).transpose(1, 2), cu_q, s["q"].shape[0]).to(s["q"].dtype)

    res = {"out": rows(out)}
    if case["op"] == "attention":
        return res
    lse = (top + total.log())[..., 0].transpose(1, 2)
    res["lse"] = _packed(lse, cu_q, s["q"].shape[0]).t().contiguous()
    do = _padded(s["d_out"], cu_q, nq, lq, g).permute(0, 2, 3, 1, 4).reshape(n * g, -1, d)
    ds = torch.bmm(do, v.transpose(1, 2)).sub_((do * out).sum(2, keepdim=True)).mul_(p)

    def keys(x):
        return _packed(x.view(n, g, lk, d).transpose(1, 2), cu_k, s["k"].shape[0]).to(s["k"].dtype)

    res["dv"] = keys(torch.bmm(p.transpose(1, 2), do))
    res["dq"] = rows(torch.bmm(ds, k) * scale)
    res["dk"] = keys(torch.bmm(ds.transpose(1, 2), q) * scale)
    return res


def _hat(x, kind):
    """(normalised rows, 1 / size)"""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    inv = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * inv, inv


def _scaled(x, weight, bias):
    x = x if weight is None else x * weight
    return x if bias is None else x + bias


def _plain_norm(s):
    case, t = s["case"], DTYPES[s["case"]["dtype"]]
    par = {n: None if p is None else p.float() for n, p in s["par"].items()}
    h = s["h"].float()
    res = {}
    if case["y"]:
        u = s["y"].float()
        if case["post"]:
            u = _scaled(_hat(u, case["kind"])[0], par["post_weight"], par["post_bias"])
        h = case["scale"] * h + (u if s["gate"] is None else s["gate"].float() * u)
        res["h"] = h.to(t)
    res["n"] = _scaled(_hat(h, case["kind"])[0], par["weight"], par["bias"]).to(t)
    return res


def _hat_grad(d, x, inv, kind):
    """Gradient of the rows behind _hat() from that of the normalised rows."""
    g = d - x * (d * x).mean(1, keepdim=True)
    if kind == "layer":
        g = g - d.mean(1, keepdim=True)
    return g * inv


def _plain_norm_grad(s):
    case, t, w = s["case"], DTYPES[s["case"]["dtype"]], DTYPES[s["case"]["w_dtype"]]
    par = {n: None if p is None else p.float() for n, p in s["par"].items()}
    kind, layer = case["kind"], case["kind"] == "layer"
    dn = s["d_n"].float()
    x, inv = _hat(s["h"].float(), kind)
    res = {"weight": (dn * x).sum(0).to(w)}
    if layer:
        res["bias"] = dn.sum(0).to(w)
    g = s["d_h"].float() + _hat_grad(dn * par["weight"], x, inv, kind)
    res["h"] = (case["scale"] * g).to(t)
    if not case["y"]:
        return res
    u = s["y"].float()
    if case["post"]:
        x, inv = _hat(u, kind)
        u = _scaled(x, par["post_weight"], par["post_bias"])
    if case["gate"] != "no":
        res["gate"] = (g * u).sum(0).to(w) if case["gate"] == "channel" else (g * u).to(t)
        g = g * s["gate"].float()
    if case["post"]:
        res["post_weight"] = (g * x).sum(0).to(w)
        if layer:
            res["post_bias"] = g.sum(0).to(w)
        g = _hat_grad(g * par["post_weight"], x, inv, kind)
    res["y"] = g.to(t)
    return res


def _plain_clip(s):
    norm = torch.sqrt(torch.stack([g.float().square().sum() for g in s["grads"]]).sum())
    factor = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
    return {"norm": norm, "grads": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


# ---- the framework's calls ----------------------------------------------------------------------------------------------
def _own_attention(s):
    case, og = s["case"], _api()
    train = case["op"] == "attention_train"
    at = dict(max_q=s["max_q"], max_k=s["max_k"], causal=case["causal"], len_k=s["len_k"])
    out, lse = og.onecomp_attention_forward(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], want_lse=train, **at)
    if not train:
        return {"out": out}
    dq, dk, dv = og.onecomp_attention_backward(s["d_out"], s["q"], s["k"], s["v"], out, lse, s["cu_q"], s["cu_k"], **at)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_norm(s):
    case, og = s["case"], _api()
    h, n = og.onecomp_block_norm_forward(s["h"], s["y"], gate=s["gate"], residual_scale=case["scale"], eps=EPS, kind=case["kind"], **s["par"])
    return {"h": h, "n": n} if case["y"] else {"n": n}


def _own_norm_grad(s):
    case, og = s["case"], _api()
    return og.onecomp_block_norm_backward(s["d_n"], s["d_h"], s["h"], s["y"], gate=s["gate"], residual_scale=case["scale"], eps=EPS, kind=case["kind"],
                                          **s["par"])


def _own_clip(s):
    grads, norm = _api().onecomp_clip_gradients(s["grads"], s["max_norm"], out=s["out"])
    return {"norm": norm, "grads": grads}


def run(s):
    op = s["case"]["op"]
    if own:
        return {"attention": _own_attention, "attention_train": _own_attention, "norm": _own_norm, "norm_grad": _own_norm_grad, "clip": _own_clip}[op](s)
    return {"attention": _plain_attention, "attention_train": _plain_attention, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "clip": _plain_clip}[op](s)


def work(case):
    """Inputs read once, outputs written once, and the operations of the definition: two products over the pairs of a
    query and a key that it sees, and five more for the gradients (the scores and the probabilities' gradients anew)."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("attention"):
        q, k = _lengths(case)
        h, g, d = case["heads"], case["kv_heads"], case["dim"]
        # query i of a sequence with a queries and b keys sees keys 0 .. i + b - a; here a <= b
        pairs = sum(a * (b - a) + a * (a + 1) // 2 if case["causal"] else a * b for a, b in zip(q, k))
        rows = 2 * sum(q) * h * d * e + 2 * sum(k) * g * d * e
        if case["op"] == "attention":
            return {"bytes": rows, "flops": 4 * pairs * h * d}
        return {"bytes": 2 * rows + sum(q) * h * 4, "flops": 14 * pairs * h * d}
    if case["op"] == "clip":
        n = sum(math.prod(shape) for shape in _shapes(case))
        return {"bytes": 2 * n * e + 4, "flops": 3 * n}
    n, d, w = case["rows"] * case["width"], case["width"], 4 if case["w_dtype"] == "f32" else 2
    layer = 2 if case["kind"] == "layer" else 1
    params = layer * (2 if case["post"] else 1) + (case["gate"] == "channel")
    if case["op"] == "norm":
        tensors = 2 + 2 * case["y"] + (case["gate"] == "token")
        return {"bytes": tensors * n * e + params * d * w, "flops": 5 * n + case["y"] * 3 * n + case["post"] * 5 * n}
    tensors = 4 + 2 * case["y"] + 2 * (case["gate"] == "token")
    return {"bytes": tensors * n * e + 2 * params * d * w, "flops": 12 * n + case["y"] * 4 * n + case["post"] * 12 * n}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------
def _attention64(case, s):
    """Sequence by sequence and head by head."""
    nq, nk = _lengths(case)
    sq, sk = _starts(nq), _starts([n + case["slack"] for n in nk])
    h, g, d = case["heads"], case["kv_heads"], case["dim"]
    train = case["op"] == "attention_train"
    res = {"out": torch.zeros(sum(nq), h, d, dtype=torch.float64, device=DEV)}
    if train:
        res["lse"] = torch.zeros(h, sum(nq), dtype=torch.float64, device=DEV)
        res.update({n: torch.zeros(s[n[1]].shape, dtype=torch.float64, device=DEV) for n in ("dq", "dk", "dv")})
    for i, (a, b) in enumerate(zip(nq, nk)):
        # one key and value head's group of query heads at a time, or all of them where the scores are small
        step = g if g * (h // g) * a * b <= 1 << 26 else 1
        for x in range(0, g, step):
            heads, groups = slice(x * (h // g), (x + step) * (h // g)), slice(x, x + step)
            rows, keys = slice(sq[i], sq[i] + a), slice(sk[i], sk[i] + b)
            Q = s["q"][rows, heads].double().transpose(0, 1).contiguous()
            K = s["k"][keys, groups].double().transpose(0, 1).repeat_interleave(h // g, 0)
            V = s["v"][keys, groups].double().transpose(0, 1).repeat_interleave(h // g, 0)
            S = torch.matmul(Q, K.transpose(1, 2)) / math.sqrt(d)
            if case["causal"]:
                S = S.masked_fill(torch.ones(a, b, dtype=torch.bool, device=DEV).triu(b - a + 1), -math.inf)
            P = torch.softmax(S, 2)
            O = torch.matmul(P, V)
            res["out"][rows, heads] = O.transpose(0, 1)
            if not train:
                continue
            res["lse"][heads, rows] = torch.logsumexp(S, 2)
            dO = s["d_out"][rows, heads].double().transpose(0, 1).contiguous()
            dS = P * (torch.matmul(dO, V.transpose(1, 2)) - (dO * O).sum(2, keepdim=True)) / math.sqrt(d)
            res["dq"][rows, heads] = torch.matmul(dS, K).transpose(0, 1)
            res["dk"][keys, groups] = torch.matmul(dS.transpose(1, 2), Q).unflatten(0, (step, -1)).sum(1).transpose(0, 1)
            res["dv"][keys, groups] = torch.matmul(P.transpose(1, 2), dO).unflatten(0, (step, -1)).sum(1).transpose(0, 1)
    return res


def _norm64(case, s):
    """From torch's own differentiation of the definition, where gradients are wanted; rows in chunks."""
    layer, grad = case["kind"] == "layer", case["op"] == "norm_grad"
    leaf = {n: p.double().requires_grad_(grad) for n, p in s["par"].items() if p is not None}
    if case["gate"] == "channel":
        leaf["gate"] = s["gate"].double().requires_grad_(grad)
    res = {}

    def norm(x, weight, bias):
        if layer:
            x = x - x.mean(1, keepdim=True)
        x = x / torch.sqrt(x.square().mean(1, keepdim=True) + EPS) * weight
        return x + bias if layer else x

    chunks = []
    for at in range(0, case["rows"], 4096):
        rows = slice(at, at + 4096)
        h = s["h"][rows].double().requires_grad_(grad)
        got = {}
        if not case["y"]:
            n = norm(h, leaf["weight"], leaf.get("bias"))
            if grad:
                back, = torch.autograd.grad(n, h, s["d_n"][rows].double(), retain_graph=True)
                got["h"] = case["scale"] * (back + s["d_h"][rows].double())
                n.backward(s["d_n"][rows].double(), inputs=list(leaf.values()))
        else:
            y = s["y"][rows].double().requires_grad_(grad)
            gate = None if case["gate"] == "no" else leaf["gate"] if case["gate"] == "channel" else s["gate"][rows].double().requires_grad_(grad)
            u = norm(y, leaf["post_weight"], leaf.get("post_bias")) if case["post"] else y
            u = u if gate is None else gate * u
            if grad:   # here h is the sum itself
                n = norm(h, leaf["weight"], leaf.get("bias"))
                back, = torch.autograd.grad(n, h, s["d_n"][rows].double(), retain_graph=True)
                total = back + s["d_h"][rows].double()
                got["h"] = case["scale"] * total
                n.backward(s["d_n"][rows].double(), inputs=[leaf[p] for p in ("weight", "bias") if p in leaf])
                ends = [y] + ([gate] if case["gate"] == "token" else []) + [leaf[p] for p in ("post_weight", "post_bias", "gate") if p in leaf]
                u.backward(total, inputs=ends)
                got["y"] = y.grad
                if case["gate"] == "token":
                    got["gate"] = gate.grad
            else:
                h = got["h"] = case["scale"] * h + u
                n = norm(h, leaf["weight"], leaf.get("bias"))
        if not grad:
            got["n"] = n
        chunks.append(got)
    for name in chunks[0]:
        res[name] = torch.cat([c[name] for c in chunks])
    if grad:
        res.update({n: p.grad for n, p in leaf.items()})
    return res


def _clip64(s):
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / (norm + 1e-6))
    return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": [g.double() * factor for g in s["grads"]]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        return _clip64(s)
    return _attention64(case, s) if case["op"].startswith("attention") else _norm64(case, s)

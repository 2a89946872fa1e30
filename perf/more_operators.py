"""Cases of the operators that take a quantized model from its tokens to its loss: embeddings, linear layers that run on the 8-bit
codes of a quantized layer, and the loss over the vocabulary, with the gradients that training takes back the same way.

A case is a dict of plain values.  `op` says which calls one pass makes:
    linear        tokens' activations to 8-bit codes with a scale each, and their product with a layer's codes
    lookup        rows of the embedding table
    lookup_grad   the gradient of the table
    loss          each token's loss and log-sum-exp over the vocabulary
    loss_train    the same, then the gradients of the last layer's input and of its weight
All inputs are made on the GPU from the seed.
"""
import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _api():
    import paper_2603_28845_amd
    return paper_2603_28845_amd


# ---- cases --------------------------------------------------------------------------------------------------------------
def _linear(name=None, **kw):
    """tokens x width to tokens x outputs; zero: "middle" (a symmetric grid, zero-point 127) or "range" (a min-max grid)."""
    c = {"op": "linear", "dtype": "bf16", "tokens": 1, "width": 4096, "outputs": 4096, "zero": "middle", "bias": False}
    c.update(kw)
    return dict(c, name=name) if name else c


def _lookup(name=None, op="lookup", **kw):
    """tokens: log-uniform ids (few that are frequent, many that are rare), `padding` of them outside the vocabulary; add: the
    gradient comes on top of another one, as where the table is the last layer's weight too."""
    c = {"op": op, "dtype": "bf16", "tokens": 1, "width": 4096, "vocab": 128000, "scale": 1.0, "padding": 0.0, "add": False}
    c.update(kw)
    return dict(c, name=name) if name else c


def _loss(name=None, op="loss", **kw):
    """left_out: the part of the tokens whose target is outside the vocabulary (prompts); z: the log-sum-exps have a gradient
    too (a penalty on them); freeze: the weight's gradient is not wanted."""
    c = {"op": op, "dtype": "bf16", "tokens": 1, "width": 4096, "vocab": 128000, "scale": 1.0, "left_out": 0.0, "z": False, "freeze": False}
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one step of generation for one request through a quantized projection: latency
        _linear("linear_1x4096x4096"),
        # one step for 16 requests through the wide projection of the 8B-class layers: the codes are read once
        _linear("linear_16x4096x14336", tokens=16, outputs=14336),
        # a batch of prompts through the same layer
        _linear("linear_8192x4096x14336", tokens=8192, outputs=14336),
        # fp32 activations, a min-max grid with bias, odd numbers of tokens and of outputs
        _linear("linear_1999x2000x777_f32", dtype="f32", tokens=1999, width=2000, outputs=777, zero="range", bias=True),
        # one step of generation: eight tokens' rows
        _lookup("lookup_8x4096", tokens=8),
        # a calibration batch of 32 sequences of 2048 tokens, scaled
        _lookup("lookup_65536x4096", tokens=65536, scale=8.0),
        # the table's gradient of a training batch, some padding in it
        _lookup("lookup_grad_16384x4096", op="lookup_grad", tokens=16384, padding=0.05),
        # fp32, odd sizes, added to the gradient that the last layer left (tied weights)
        _lookup("lookup_grad_3001x1359_f32", op="lookup_grad", dtype="f32", tokens=3001, width=1359, vocab=50021, scale=0.5, add=True),
        # scoring 16 next tokens: the weight is read once
        _loss("loss_16x4096x128000", tokens=16),
        # perplexity of a quantized model: eight sequences of 2048 tokens
        _loss("loss_16384x4096x128000", tokens=16384),
        # training on answers: more than a third of the tokens are prompts and left out
        _loss("loss_train_8192x4096x128000", op="loss_train", tokens=8192, left_out=0.4),
        # the smallest model in fp32, odd sizes, a penalty on the log-sum-exps
        _loss("loss_train_1001x500x32003_f32", op="loss_train", dtype="f32", tokens=1001, width=500, vocab=32003, scale=0.7, left_out=0.1, z=True),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / (1e14 if c["dtype"] == "f32" and c["op"] != "linear" else 1e15)


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["linear", "linear", "linear", "lookup", "lookup_grad", "lookup_grad", "loss", "loss", "loss_train", "loss_train"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op == "linear":
            c = _linear(dtype=dtype, tokens=_log_int(rng, 1, 16384), width=_log_int(rng, 64, 14336, 16), outputs=_log_int(rng, 16, 14336, rng.choice([1, 16])),
                        zero=rng.choice(["middle", "range"]), bias=rng.random() < 0.4)
        elif op.startswith("lookup"):
            c = _lookup(op=op, dtype=dtype, tokens=_log_int(rng, 1, 65536), width=_log_int(rng, 64, 8192, rng.choice([1, 16])), vocab=_log_int(rng, 250, 200000),
                        scale=rng.choice([1.0, 0.5, 8.0]), padding=rng.choice([0.0, 0.05, 0.5]))
            c["add"] = op == "lookup_grad" and rng.random() < 0.5
        else:
            c = _loss(op=op, dtype=dtype, tokens=_log_int(rng, 1, 16384), width=_log_int(rng, 64, 8192, rng.choice([8, 64])), vocab=_log_int(rng, 250, 200000),
                      scale=rng.choice([1.0, 1.0, 0.7]), left_out=rng.choice([0.0, 0.1, 0.6]))
            if op == "loss_train":
                c.update(z=rng.random() < 0.3, freeze=rng.random() < 0.3)
        if _cost(c) <= top and c["tokens"] * c.get("vocab", 0) <= 2.2e9:
            return c


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _normal(gen, *shape, dtype=torch.float32, std=1.0):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype).mul_(std)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV)


def _ids(gen, n, vocab, outside, mark):
    """int32 ids whose frequency falls with one over their rank, in no order; `outside` of them are `mark`."""
    rank = torch.exp(_uniform(gen, n) * math.log(vocab)).long().sub_(1).clamp_(0, vocab - 1)
    ids = torch.randperm(vocab, generator=gen, device=DEV)[rank].to(torch.int32)
    return ids.masked_fill_(_uniform(gen, n) < outside, mark)


def _prepare_linear(case, gen, s):
    t, n, d, m = DTYPES[case["dtype"]], case["tokens"], case["width"], case["outputs"]
    level = torch.exp(_normal(gen, n, 1, std=0.5))                                # tokens differ in size
    big = 1.0 + 19.0 * (_uniform(gen, d) < 0.005).float()                         # and some channels stand out
    s["x"] = (_normal(gen, n, d) * level * big).to(t)
    w = _normal(gen, m, d, std=0.02)
    if case["zero"] == "middle":
        s["scales"] = w.abs().amax(1, keepdim=True) / 127
        s["zeros"] = torch.full((m, 1), 127.0, device=DEV)
        top = 254
    else:
        lo, hi = w.amin(1, keepdim=True).clamp_(max=0.0), w.amax(1, keepdim=True).clamp_(min=0.0)
        s["scales"] = (hi - lo) / 255
        s["zeros"] = torch.round(-lo / s["scales"]).clamp_(0, 255)
        top = 255
    s["q"] = torch.round(w / s["scales"]).add_(s["zeros"]).clamp_(0, top).to(torch.uint8)
    s["bias"] = _normal(gen, m, dtype=t) if case["bias"] else None


def _prepare_lookup(case, gen, s):
    t, n, d, v = DTYPES[case["dtype"]], case["tokens"], case["width"], case["vocab"]
    s["tokens"] = _ids(gen, n, v, case["padding"], -1)
    if case["op"] == "lookup":
        s["table"] = _normal(gen, v, d, dtype=t, std=0.02)
        return
    s["d_out"] = _normal(gen, n, d, dtype=t, std=0.02)
    s["base"] = _normal(gen, v, d, dtype=t, std=0.02) if case["add"] else None


def _prepare_loss(case, gen, s):
    t, n, d, v = DTYPES[case["dtype"]], case["tokens"], case["width"], case["vocab"]
    s["h"] = _normal(gen, n, d, dtype=t)
    s["weight"] = _normal(gen, v, d, dtype=t, std=2.0 / math.sqrt(d))
    s["targets"] = _ids(gen, n, v, case["left_out"], -100)
    if case["op"] == "loss_train":
        kept = (s["targets"] >= 0).float()
        s["d_loss"] = kept / kept.sum().clamp_(min=1.0)
        s["d_lse"] = _uniform(gen, n) * 0.1 * s["d_loss"] if case["z"] else None


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": case}
    {"linear": _prepare_linear, "lookup": _prepare_lookup, "lookup_grad": _prepare_lookup, "loss": _prepare_loss, "loss_train": _prepare_loss}[case["op"]](case, gen, s)
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------------
def _plain_linear(s):
    x = s["x"].float()
    top = x.abs().amax(1, keepdim=True)
    scale = top / torch.full_like(top, 127.0)         # divided: by a number, it would be multiplied with the rounded 1 / 127
    codes = torch.where(scale > 0, torch.round(x / scale), 0.0).clamp_(-127, 127)
    y = (codes @ (s["q"].float() - s["zeros"]).t()) * scale * s["scales"].t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return {"codes": codes.to(torch.int8), "token_scales": scale[:, 0], "sums": codes.sum(1, dtype=torch.float64).to(torch.int32), "y": y.to(s["x"].dtype)}


def _inside(ids, vocab):
    return (ids >= 0) & (ids < vocab)


def _plain_lookup(s):
    case = s["case"]
    ok = _inside(s["tokens"], case["vocab"])
    rows = s["table"][torch.where(ok, s["tokens"], 0).long()].float()
    return {"out": (rows * case["scale"] * ok[:, None]).to(s["table"].dtype)}


def _plain_lookup_grad(s):
    case = s["case"]
    ok = _inside(s["tokens"], case["vocab"])
    sums = torch.zeros(case["vocab"], case["width"], device=DEV)
    sums.index_add_(0, s["tokens"][ok].long(), s["d_out"][ok].float() * case["scale"])
    if case["add"]:
        sums += s["base"].float()
    return {"grad": sums.to(s["d_out"].dtype)}


def _plain_loss(s):
    case, t = s["case"], DTYPES[s["case"]["dtype"]]
    h, w = s["h"].float(), s["weight"].float()
    ok = _inside(s["targets"], case["vocab"])
    at = torch.where(ok, s["targets"], 0).long()[:, None]
    z = h @ w.t()
    z *= case["scale"]
    top = z.amax(1, keepdim=True)
    hit = z.gather(1, at)
    z.sub_(top).exp_()
    lse = top + z.sum(1, keepdim=True).log_()
    res = {"loss": torch.where(ok, (lse - hit)[:, 0], 0.0), "lse": torch.where(ok, lse[:, 0], 0.0)}
    if case["op"] == "loss":
        return res
    d = torch.where(ok, s["d_loss"], 0.0)
    both = d if s["d_lse"] is None else d + torch.where(ok, s["d_lse"], 0.0)
    z *= (both * torch.exp(top - lse)[:, 0])[:, None]
    z.scatter_add_(1, at, -d[:, None])
    res["dh"] = (z @ w * case["scale"]).to(t)
    if not case["freeze"]:
        res["dweight"] = (z.t() @ h * case["scale"]).to(t)
    return res


# ---- the framework's calls ----------------------------------------------------------------------------------------------
def _own_linear(s):
    og = _api()
    codes, token_scales, sums = og.onecomp_quantize_tokens(s["x"])
    y = og.onecomp_linear_int8(codes, token_scales, sums, s["q"], s["scales"], s["zeros"], bias=s["bias"], dtype=s["x"].dtype)
    return {"codes": codes, "token_scales": token_scales, "sums": sums, "y": y}


def _own_lookup(s):
    return {"out": _api().onecomp_embedding_forward(s["tokens"], s["table"], scale=s["case"]["scale"])}


def _own_lookup_grad(s):
    case = s["case"]
    return {"grad": _api().onecomp_embedding_backward(s["tokens"], s["d_out"], case["vocab"], scale=case["scale"], base=s["base"])}


def _own_loss(s):
    case, og = s["case"], _api()
    loss, lse = og.onecomp_token_loss_forward(s["h"], s["weight"], s["targets"], scale=case["scale"])
    res = {"loss": loss, "lse": lse}
    if case["op"] == "loss_train":
        dh, dweight = og.onecomp_token_loss_backward(s["d_loss"], s["h"], s["weight"], s["targets"], lse, scale=case["scale"], d_lse=s["d_lse"],
                                                     want_dweight=not case["freeze"])
        res["dh"] = dh
        if not case["freeze"]:
            res["dweight"] = dweight
    return res


def run(s):
    op = s["case"]["op"]
    if own:
        return {"linear": _own_linear, "lookup": _own_lookup, "lookup_grad": _own_lookup_grad, "loss": _own_loss, "loss_train": _own_loss}[op](s)
    return {"linear": _plain_linear, "lookup": _plain_lookup, "lookup_grad": _plain_lookup_grad, "loss": _plain_loss, "loss_train": _plain_loss}[op](s)


def work(case):
    """Inputs read once, outputs written once, and the operations of the definition: one product for the logits and one for each
    of their gradients.  Left-out tokens and padding take no part (in the proportion that the case names)."""
    e, n, d = 4 if case["dtype"] == "f32" else 2, case["tokens"], case["width"]
    if case["op"] == "linear":
        m = case["outputs"]
        return {"bytes": n * d * e + m * d + n * m * e + n * d + 8 * n + 8 * m, "flops": 2 * n * m * d}
    v = case["vocab"]
    if case["op"] == "lookup":
        return {"bytes": 2 * n * d * e + 4 * n, "flops": n * d}
    if case["op"] == "lookup_grad":
        kept = round(n * (1 - case["padding"]))
        return {"bytes": (kept + (2 * v if case["add"] else v)) * d * e + 4 * n, "flops": 2 * kept * d}
    kept = max(1, round(n * (1 - case["left_out"])))
    products = 1 if case["op"] == "loss" else 2 if case["freeze"] else 3
    out = 0 if case["op"] == "loss" else n * d * e + (0 if case["freeze"] else v * d * e)
    return {"bytes": int(kept * d * e + v * d * e + out + 12 * n), "flops": 2 * products * kept * v * d}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------
def _linear64(case, s):
    """The codes are the rounded quotients of 32-bit numbers; everything behind them in 64 bits."""
    x = s["x"].double()
    scale = (x.abs().amax(dim=1) / 127.0).float()
    codes = torch.zeros_like(x)
    for i in range(0, case["tokens"], 4096):
        part = (x[i:i + 4096] / scale[i:i + 4096, None].double()).float()          # rounded to 32 bits once, as a division is
        codes[i:i + 4096] = torch.nan_to_num(part, nan=0.0).round().clamp(-127, 127).double()
    w = (s["q"].double() - s["zeros"].double()) * s["scales"].double()
    y = torch.matmul(codes, w.t().contiguous()) * scale.double()[:, None]
    if case["bias"]:
        y = y + s["bias"].double()
    return {"codes": codes.to(torch.int8), "token_scales": x.abs().amax(dim=1) / 127, "sums": codes.sum(dim=1).to(torch.int32), "y": y}


def _lookup64(case, s):
    tokens = s["tokens"].long()
    known = torch.logical_and(tokens >= 0, tokens < case["vocab"])
    if case["op"] == "lookup":
        out = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device=DEV)
        out[known] = torch.index_select(s["table"], 0, tokens[known]).double() * case["scale"]
        return {"out": out}
    order = torch.argsort(tokens[known], stable=True)
    ids, counts = torch.unique_consecutive(tokens[known][order], return_counts=True)
    res = s["base"].double() if case["add"] else torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device=DEV)
    rows = s["d_out"][known][order]
    ends = counts.cumsum(0)
    for i in range(0, case["width"], 512):                                          # differences of running sums, some columns at a time
        run_sums = torch.cat([torch.zeros(1, min(512, case["width"] - i), dtype=torch.float64, device=DEV), rows[:, i:i + 512].double().cumsum(0)])
        res[ids, i:i + 512] += (run_sums[ends] - run_sums[ends - counts]) * case["scale"]
    return {"grad": res}


def _loss64(case, s):
    """Some tokens at a time; those that are left out are never computed."""
    train = case["op"] == "loss_train"
    W = s["weight"].double()
    Wt = W.t().contiguous()
    kept = torch.nonzero((s["targets"] >= 0) & (s["targets"] < case["vocab"]))[:, 0]
    zero = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device=DEV)      # noqa: E731
    res = {"loss": zero(case["tokens"]), "lse": zero(case["tokens"])}
    if train:
        res["dh"] = zero(case["tokens"], case["width"])
        if not case["freeze"]:
            res["dweight"] = zero(case["vocab"], case["width"])
    for rows in kept.split(1024):
        H = s["h"][rows].double()
        Z = torch.mm(H, Wt) * case["scale"]
        target = s["targets"][rows].long()
        lse = torch.logsumexp(Z, 1)
        res["lse"][rows] = lse
        res["loss"][rows] = lse - Z[torch.arange(len(rows), device=DEV), target]
        if not train:
            continue
        P = torch.exp(Z - lse[:, None])
        dl = s["d_loss"][rows].double()
        G = P * (dl if s["d_lse"] is None else dl + s["d_lse"][rows].double())[:, None]
        G[torch.arange(len(rows), device=DEV), target] -= dl
        res["dh"][rows] = torch.mm(G, W) * case["scale"]
        if not case["freeze"]:
            res["dweight"] += torch.mm(G.t(), H) * case["scale"]
    return res


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _linear64, "lookup": _lookup64, "lookup_grad": _lookup64, "loss": _loss64, "loss_train": _loss64}[case["op"]](case, s)

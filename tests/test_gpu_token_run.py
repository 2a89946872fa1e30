"""The operators from tokens to the loss together: a small model and the table's gradient against 64 bits, and all of them in a HIP
graph and on two streams."""
import os
import sys

import pytest
import torch

import paper_2603_28845_amd as og

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _norm(x, w):
    return x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6) * w


def _reference(model, ids, targets, t, d_loss):
    """Loss and the table's gradient in 64 bits; quantized layers take the codes that the model's own activations were rounded to."""
    table = model.table.double().requires_grad_(True)
    h, y = table[ids.long()] * model.scale, None

    def apply(name, x):
        if name in model.codes:
            codes, scales, _ = t[name]
            x = x + (codes.double() * scales.double()[:, None] - x).detach()        # straight through the rounding
        return x @ model.weight(name).double().t()

    for i in range(model.depth):
        h = h if y is None else h + y
        gate, up = apply(f"{i}.up", _norm(h, model.norms[i].double())).chunk(2, 1)
        y = apply(f"{i}.down", torch.nn.functional.silu(gate) * up)
    z = _norm(h + y, model.norms[-1].double()) @ table.t()
    ok = targets >= 0
    loss = torch.where(ok, torch.logsumexp(z, 1) - z[torch.arange(len(ids), device=DEV), torch.where(ok, targets, 0).long()], 0.0)
    (loss * d_loss.double()).sum().backward()
    return loss.detach(), table.grad


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("n", [48, 700])
def test_model_and_its_table_gradient(n, quantized):
    import score_model as ex
    model = ex.Model(333, 128, 2, seed=n, dtype=F32)
    ids, targets = ex.text(333, n, 5)
    gram = {k: torch.zeros(w.shape[1], w.shape[1], device=DEV) for k, w in model.linear.items()}
    model.forward(ids, targets, lambda name, rows: og.onecomp_hessian_accumulate(rows, gram[name]))
    if quantized:
        model.quantize(gram, 8)
    d_loss = torch.rand(n, generator=torch.Generator(device=DEV).manual_seed(6), device=DEV) / n
    loss, t = model.forward(ids, targets)
    got = model.table_gradient(ids, targets, t, d_loss)
    want, grad = _reference(model, ids, targets, t, d_loss)
    # 32 bits throughout: six products of up to 333 terms in a row, forward and backward, three norms between them; each sum
    # is off by its number of terms times 2^-24 at most, in the norm over all entries by a tenth of that
    off = 12 * 333 * 2.0 ** -24 / 10
    assert float((loss.double() - want).norm() / want.norm()) < off
    assert float((got.double() - grad).norm() / grad.norm()) < off


def test_example_runs():
    import score_model as ex
    before, after, losses = ex.run(vocab=500, width=128, depth=2, tokens=900, steps=3, say=lambda *a: None)
    assert before > 1 and after > 1 and len(losses) == 3 and all(x == x for x in losses)


def _inputs(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, dtype=BF16):
        return torch.randn(*shape, generator=gen, device=DEV).to(dtype)

    n, width, vocab = 300, 144, 1000
    tokens = torch.randint(-20, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    return {"tokens": tokens, "targets": tokens.roll(seed), "table": normal(vocab, width), "q": torch.randint(0, 256, (200, width), generator=gen, device=DEV, dtype=torch.uint8),
            "s": torch.rand(200, generator=gen, device=DEV), "z": torch.randint(0, 256, (200,), generator=gen, device=DEV).float(), "d": torch.rand(n, generator=gen, device=DEV)}


def _buffers(n=300, width=144, vocab=1000):
    def new(*shape, dtype=BF16):
        return torch.zeros(*shape, dtype=dtype, device=DEV)

    return {"h": new(n, width), "codes": new(n, width, dtype=torch.int8), "ts": new(n, dtype=F32), "sums": new(n, dtype=torch.int32), "y": new(n, 200), "few": new(9, 200),
            "loss": new(n, dtype=F32), "lse": new(n, dtype=F32), "loss_few": new(9, dtype=F32), "lse_few": new(9, dtype=F32), "dh": new(n, width),
            "dw": new(vocab, width), "dt": new(vocab, width), "ws": torch.zeros(1 << 26, dtype=torch.uint8, device=DEV)}


def _step(x, b):
    og.onecomp_embedding_forward(x["tokens"], x["table"], scale=3.0, out=b["h"])
    og.onecomp_quantize_tokens(b["h"], b["codes"], b["ts"], b["sums"])
    og.onecomp_linear_int8(b["codes"], b["ts"], b["sums"], x["q"], x["s"], x["z"], out=b["y"])
    og.onecomp_linear_int8(b["codes"][:9], b["ts"][:9], b["sums"][:9], x["q"], x["s"], x["z"], out=b["few"])
    og.onecomp_token_loss_forward(b["h"], x["table"], x["targets"], loss=b["loss"], lse=b["lse"], workspace=b["ws"])
    og.onecomp_token_loss_forward(b["h"][:9], x["table"], x["targets"][:9], loss=b["loss_few"], lse=b["lse_few"], workspace=b["ws"])
    og.onecomp_token_loss_backward(x["d"], b["h"], x["table"], x["targets"], b["lse"], dh=b["dh"], dweight=b["dw"], workspace=b["ws"])
    og.onecomp_embedding_backward(x["tokens"], b["dh"], 1000, scale=3.0, base=b["dw"], d_table=b["dt"], workspace=b["ws"])


def test_replays_equal_eager_calls():
    x, buf = _inputs(0), _buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(x, buf)                    # first calls set the kernels' attributes
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(x, buf)
    for seed in (1, 2, 3, 4):
        fresh = _inputs(seed)
        for name, t in x.items():
            t.copy_(fresh[name])
        for name, t in buf.items():
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        want = _buffers()
        _step(fresh, want)               # the program's own eager work between replays
        torch.cuda.synchronize()
        for name in buf:
            if name != "ws":
                assert torch.equal(buf[name], want[name]), (seed, name)


def test_two_streams_at_once():
    inputs, alone, beside = [_inputs(s) for s in (7, 8)], [_buffers(), _buffers()], [_buffers(), _buffers()]
    for x, b in zip(inputs, alone):
        _step(x, b)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for x, b, s in zip(inputs, beside, streams):
            with torch.cuda.stream(s):
                _step(x, b)
    torch.cuda.synchronize()
    for a, b in zip(alone, beside):
        for name in a:
            if name != "ws":
                assert torch.equal(a[name], b[name]), name

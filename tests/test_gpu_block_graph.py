"""The block operators in a HIP graph: captured once, replayed on new inputs with eager work in between, every replay equal to
the eager calls bit for bit."""
import pytest
import torch

import paper_2603_28845_amd as og

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _step(x, buf):
    """Norm, attention, norm, their gradients, clipping: into the buffers alone."""
    cu, cu_k, len_k = x["cu"], x["cu_k"], x["len_k"]
    og.onecomp_block_norm_forward(x["h"], x["y"], weight=x["w"], gate=x["g"], h_out=buf["h"], n=buf["n"])
    og.onecomp_attention_forward(x["q"], x["k"], x["v"], cu, cu, 300, 300, out=buf["out"], lse=buf["lse"], workspace=buf["ws"])
    og.onecomp_attention_forward(x["q"][:3], x["ck"], x["cv"], x["one"], cu_k, 1, 4000, len_k=len_k, out=buf["few"], lse=buf["few_lse"], workspace=buf["ws"])
    og.onecomp_attention_backward(x["d"], x["q"], x["k"], x["v"], buf["out"], buf["lse"], cu, cu, 300, 300, dq=buf["dq"], dk=buf["dk"], dv=buf["dv"],
                                  workspace=buf["ws"])
    grads = {"h": buf["dh"], "y": buf["dy"], "weight": buf["dw"], "gate": buf["dg"]}
    og.onecomp_block_norm_backward(x["y"], x["h"], buf["h"], x["y"], weight=x["w"], gate=x["g"], out=grads, workspace=buf["ws"])
    og.onecomp_clip_gradients([buf["dw"], buf["dg"]], 0.5, out=[buf["cw"], buf["cg"]], norm=buf["norm"], workspace=buf["ws"])


def _inputs(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device=DEV).to(dtype)

    x = {"h": normal(200, 1000), "y": normal(200, 1000), "w": normal(1000, dtype=torch.float32), "g": normal(1000, dtype=torch.float32),
         "q": normal(500, 8, 64), "k": normal(500, 2, 64), "v": normal(500, 2, 64), "d": normal(500, 8, 64), "ck": normal(9000, 2, 64), "cv": normal(9000, 2, 64)}
    ints = {"cu": [0, 300 - seed, 500], "one": [0, 1, 2, 3], "cu_k": [0, 4000, 4100, 9000], "len_k": [4000 - seed, 100, 2000 + seed]}
    x.update({n: torch.tensor(v, dtype=torch.int32, device=DEV) for n, v in ints.items()})
    return x


def _buffers():
    def new(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype, device=DEV)

    f = torch.float32
    return {"h": new(200, 1000), "n": new(200, 1000), "out": new(500, 8, 64), "lse": new(8, 500, dtype=f), "few": new(3, 8, 64), "few_lse": new(8, 3, dtype=f),
            "dq": new(500, 8, 64), "dk": new(500, 2, 64), "dv": new(500, 2, 64), "dh": new(200, 1000), "dy": new(200, 1000), "dw": new(1000, dtype=f),
            "dg": new(1000, dtype=f), "cw": new(1000, dtype=f), "cg": new(1000, dtype=f), "norm": new(1, dtype=f)[0], "ws": new(1 << 27, dtype=torch.uint8)}


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

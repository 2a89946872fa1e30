"""The example that calibrates, quantizes and tunes a block: its gradients against torch's own differentiation of the same
block in 64 bits, and tuning that brings the output nearer."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _norm(x, w):
    return x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6) * w


def _reference(block, h, cu):
    """The block in 64 bits, with its free parameters as leaves."""
    L = {n: w.double() for n, w in block.linear.items()}
    F = {n: p.double().requires_grad_(True) for n, p in block.free.items()}
    h = h.double()
    q, k, v = (_norm(h, F["norm_attention"]) @ L["qkv"].t()).view(h.shape[0], -1, block.dim).split([block.heads, block.kv_heads, block.kv_heads], 1)
    out = []
    for a, b in zip(cu.tolist(), cu.tolist()[1:]):
        qs, ks, vs = (x[a:b].transpose(0, 1) for x in (q, k, v))
        ks, vs = (x.repeat_interleave(block.heads // block.kv_heads, 0) for x in (ks, vs))
        s = (qs @ ks.transpose(1, 2)) * block.dim ** -0.5
        s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device=h.device).triu(1), -float("inf"))
        out.append((torch.softmax(s, 2) @ vs).transpose(0, 1).reshape(b - a, -1))
    h1 = h + F["scale_attention"] * (torch.cat(out) @ L["o"].t())
    g, u = (_norm(h1, F["norm_mlp"]) @ L["up"].t()).chunk(2, 1)
    return h1 + F["scale_mlp"] * ((torch.nn.functional.silu(g) * u) @ L["down"].t()), F


def test_gradients_of_the_block():
    import tune_block as ex
    block = ex.Block(256, 4, 2, seed=3)
    h, cu = ex.tokens(5, 130, 256, 4)
    got, t = block.forward(h, cu, 130)
    want, leaves = _reference(block, h, cu)
    # a dozen bf16 roundings on the way, each 2^-9 at the middle, of rows whose parts add up: a few of them at most in the norm
    assert float((got.double() - want).detach().norm() / want.detach().norm()) < 6 * 2.0 ** -9
    d = torch.randn(got.shape, generator=torch.Generator(device="cuda:0").manual_seed(5), device="cuda:0").to(torch.bfloat16)
    grads = block.gradients(d, t, cu, 130)
    want.backward(d.double())
    for name, leaf in leaves.items():
        g, w = grads[name].double(), leaf.grad
        # the same dozen roundings of the forward values and as many of the gradients, which sum over hundreds of tokens
        assert float((g - w).norm() / w.norm()) < 16 * 2.0 ** -9, name


def test_tuning_brings_the_output_nearer():
    import tune_block as ex
    errors = ex.run(width=512, heads=4, kv_heads=2, seqs=6, length=300, bits=2, steps=12, say=lambda *a: None)
    assert all(e == e for e in errors) and errors[-1] < 0.97 * errors[0]

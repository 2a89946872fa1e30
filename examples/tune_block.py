"""One decoder block from calibration to tuning, on synthetic weights and tokens.

  1. Calibration: packed sequences go through the block; the rows that enter each linear layer (what its norm, the attention or
     the activation left) are added to that layer's Gram matrix as they come.
  2. Quantization: every linear layer by the column sweep on its own Gram matrix.
  3. Block-wise compensation: the norms' weights and the branches' scales, which stay in floating point, are tuned so that the
     quantized block's output comes back to the original's: gradients through the same kernels, clipped to a global norm, Adam.

    python examples/tune_block.py [--width 1024 --heads 8 --kv-heads 2 --seqs 16 --length 512 --bits 3 --steps 20]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_28845_amd as og  # noqa: E402

DEV = "cuda:0"


class Block:
    """Weights of the linear layers, [outputs, inputs] bf16, and what stays in floating point."""

    def __init__(self, width: int, heads: int, kv_heads: int, seed: int = 0):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.heads, self.kv_heads, self.dim = heads, kv_heads, width // heads
        ff = 3 * width

        def weight(rows, cols):
            return torch.randn(rows, cols, generator=gen, device=DEV).mul_(cols ** -0.5).to(torch.bfloat16)

        self.linear = {"qkv": weight((heads + 2 * kv_heads) * self.dim, width), "o": weight(width, heads * self.dim),
                       "up": weight(2 * ff, width), "down": weight(width, ff)}
        self.free = {n: torch.ones(width, device=DEV) + 0.1 * torch.randn(width, generator=gen, device=DEV)
                     for n in ("norm_attention", "norm_mlp", "scale_attention", "scale_mlp")}

    def forward(self, h, cu, longest, seen=None):
        """The block's output and what the gradients need; seen(name, rows): the inputs of each linear layer."""
        seen = seen or (lambda name, rows: None)
        L, F, t = self.linear, self.free, {"h": h}
        _, t["n1"] = og.onecomp_block_norm_forward(h, weight=F["norm_attention"])
        seen("qkv", t["n1"])
        qkv = (t["n1"] @ L["qkv"].t()).view(h.shape[0], -1, self.dim)
        t["q"], t["k"], t["v"] = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        t["out"], t["lse"] = og.onecomp_attention_forward(t["q"], t["k"], t["v"], cu, cu, longest, longest)
        rows = t["out"].view(h.shape[0], -1)
        seen("o", rows)
        t["y1"] = rows @ L["o"].t()
        t["h1"], t["n2"] = og.onecomp_block_norm_forward(h, t["y1"], weight=F["norm_mlp"], gate=F["scale_attention"])
        seen("up", t["n2"])
        t["gate"], t["up"] = (t["n2"] @ L["up"].t()).chunk(2, 1)
        t["act"] = torch.nn.functional.silu(t["gate"]) * t["up"]
        seen("down", t["act"])
        t["y2"] = t["act"] @ L["down"].t()
        t["h2"], _ = og.onecomp_block_norm_forward(t["h1"], t["y2"], gate=F["scale_mlp"], want_n=False)
        return t["h2"], t

    def gradients(self, dh2, t, cu, longest):
        """Gradients of the free parameters from that of the output."""
        L, F = self.linear, self.free
        g2 = og.onecomp_block_norm_backward(None, dh2, t["h2"], t["y2"], gate=F["scale_mlp"])
        d_act = g2["y"] @ L["down"]
        s = torch.sigmoid(t["gate"])
        d_up = torch.cat([d_act * t["up"] * s * (1 + t["gate"] * (1 - s)), d_act * t["gate"] * s], 1)
        g1 = og.onecomp_block_norm_backward(d_up @ L["up"], g2["h"], t["h1"], t["y1"], weight=F["norm_mlp"], gate=F["scale_attention"])
        d_out = (g1["y"] @ L["o"]).view(t["out"].shape)
        d_qkv = torch.empty(d_out.shape[0], self.heads + 2 * self.kv_heads, self.dim, dtype=d_out.dtype, device=DEV)
        dq, dk, dv = d_qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        og.onecomp_attention_backward(d_out, t["q"], t["k"], t["v"], t["out"], t["lse"], cu, cu, longest, longest, dq=dq, dk=dk, dv=dv)
        g0 = og.onecomp_block_norm_backward(d_qkv.view(d_out.shape[0], -1) @ L["qkv"], g1["h"], t["h"], weight=F["norm_attention"])
        return {"norm_attention": g0["weight"], "norm_mlp": g1["weight"], "scale_attention": g1["gate"], "scale_mlp": g2["gate"]}


def tokens(seqs: int, length: int, width: int, seed: int):
    """Packed sequences of different lengths: rows and starts."""
    gen = torch.Generator()
    gen.manual_seed(seed)
    lengths = torch.randint(length // 4, length + 1, (seqs,), generator=gen)
    lengths[0] = length
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).to(torch.int32).to(DEV)
    dev = torch.Generator(device=DEV)
    dev.manual_seed(seed)
    h = torch.randn(int(lengths.sum()), width, generator=dev, device=DEV)
    return h.mul_(1 + 9 * (torch.rand(width, generator=dev, device=DEV) < 0.01)).to(torch.bfloat16), cu


def run(width=1024, heads=8, kv_heads=2, seqs=16, length=512, bits=3, group=128, steps=20, lr=5e-3, max_norm=1.0, say=print):
    """Returns the mean squared error of the block's output before tuning and after each step, relative to its square."""
    block = Block(width, heads, kv_heads)
    h, cu = tokens(seqs, length, width, 1)
    gram = {n: torch.zeros(w.shape[1], w.shape[1], device=DEV) for n, w in block.linear.items()}
    target, _ = block.forward(h, cu, length, lambda name, rows: og.onecomp_hessian_accumulate(rows, gram[name]))
    target = target.float()
    size = target.square().mean()
    for name, w in block.linear.items():
        U, _, info = og.onecomp_hessian_factor(gram[name], 0.01)
        out = og.onecomp_quantize_layer(w, U, bits, group)
        if int(info) != 0:
            raise RuntimeError(f"the Gram matrix of {name} is not positive definite")
        block.linear[name] = out["W_hat"].to(torch.bfloat16)
    names = list(block.free)
    adam = torch.optim.Adam([block.free[n].requires_grad_(False) for n in names], lr=lr)
    errors, norms = [], []
    for step in range(steps + 1):
        got, t = block.forward(h, cu, length)
        off = got.float() - target
        errors.append(float(off.square().mean() / size))
        say(f"step {step:3d}  relative error {errors[-1]:.5f}" + (f"  gradient norm {norms[-1]:.4f}" if norms else ""))
        if step == steps:
            return errors
        # the loss is the relative error; its gradient in the output's type
        grads = block.gradients((off * (2 / (off.numel() * size))).to(torch.bfloat16), t, cu, length)
        clipped, norm = og.onecomp_clip_gradients([grads[n] for n in names], max_norm)
        norms.append(float(norm))
        for n, g in zip(names, clipped):
            block.free[n].grad = g
        adam.step()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("width", 1024), ("heads", 8), ("kv-heads", 2), ("seqs", 16), ("length", 512), ("bits", 3), ("group", 128), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=default)
    a = vars(ap.parse_args())
    run(**{k.replace("-", "_"): v for k, v in a.items()})

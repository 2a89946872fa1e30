"""A small language model from its tokens to its loss, before and after its layers are quantized, on synthetic weights and tokens.

  1. Calibration: token rows come out of the embedding table and go through the blocks; what enters each linear layer is added to
     that layer's Gram matrix.
  2. Quantization: every linear layer by the column sweep on its own Gram matrix, one group per output channel.
  3. Scoring: the perplexity of the model with its layers as they were and with the layers run on their 8-bit codes.
  4. Tuning: the embedding table, which is the last layer's weight too, follows the loss through the quantized layers (their
     gradients are those of the dequantized weights, straight through the rounding of the activations).

    python examples/score_model.py [--vocab 2000 --width 256 --depth 2 --tokens 4096 --bits 8 --steps 10]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_28845_amd as og  # noqa: E402

DEV = "cuda:0"


class Model:
    """A table that is the last layer's weight too, `depth` blocks of norm, two linear layers with a gate between them and a
    residual, and a last norm."""

    def __init__(self, vocab: int, width: int, depth: int, seed: int = 0, dtype: torch.dtype = torch.bfloat16):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)

        def weight(rows, cols, size):
            return torch.randn(rows, cols, generator=gen, device=DEV).mul_(size).to(dtype)

        self.table, self.scale = weight(vocab, width, width ** -0.5), width ** 0.5
        self.linear = {f"{i}.{n}": weight(rows, cols, cols ** -0.5) for i in range(depth) for n, rows, cols in (("up", 4 * width, width), ("down", width, 2 * width))}
        self.norms = [torch.ones(width, device=DEV, dtype=dtype) for _ in range(depth + 1)]
        self.depth, self.codes = depth, {}

    def quantize(self, gram: dict, bits: int) -> None:
        for name, w in self.linear.items():
            U, _, info = og.onecomp_hessian_factor(gram[name], 0.01)
            out = og.onecomp_quantize_layer(w, U, bits, w.shape[1], grid="symmetric")
            if int(info) != 0:
                raise RuntimeError(f"the Gram matrix of {name} is not positive definite")
            self.codes[name] = out

    def _apply(self, name: str, x: torch.Tensor, t: dict) -> torch.Tensor:
        if name not in self.codes:
            return x @ self.linear[name].t()
        c = self.codes[name]
        t[name] = og.onecomp_quantize_tokens(x)
        return og.onecomp_linear_int8(*t[name], c["Q_codes"], c["scales"], c["zeros"], dtype=x.dtype)

    def forward(self, tokens: torch.Tensor, targets: torch.Tensor, seen=None):
        """Each token's loss and what the gradients need; seen(name, rows): the inputs of each linear layer."""
        seen = seen or (lambda name, rows: None)
        t = {"h": [og.onecomp_embedding_forward(tokens, self.table, scale=self.scale)], "y": [None], "gate": [], "up": []}
        for i in range(self.depth):
            h, n = og.onecomp_block_norm_forward(t["h"][-1], t["y"][-1], weight=self.norms[i])
            t["h"][-1] = h
            seen(f"{i}.up", n)
            gate, up = self._apply(f"{i}.up", n, t).chunk(2, 1)
            act = torch.nn.functional.silu(gate) * up
            seen(f"{i}.down", act)
            t["gate"].append(gate)
            t["up"].append(up)
            t["y"].append(self._apply(f"{i}.down", act, t))
            t["h"].append(h)
        t["h"][-1], t["n"] = og.onecomp_block_norm_forward(t["h"][-1], t["y"][-1], weight=self.norms[-1])
        loss, t["lse"] = og.onecomp_token_loss_forward(t["n"], self.table, targets)
        return loss, t

    def table_gradient(self, tokens, targets, t, d_loss):
        """The table's gradient from those of the losses: as the last layer's weight, then on top of it as the embedding."""
        dn, d_table = og.onecomp_token_loss_backward(d_loss, t["n"], self.table, targets, t["lse"])
        dh = None
        for i in reversed(range(self.depth + 1)):
            g = og.onecomp_block_norm_backward(dn, dh, t["h"][i], t["y"][i], weight=self.norms[i])
            dh = g["h"]
            if i == 0:
                break
            gate, up, s = t["gate"][i - 1], t["up"][i - 1], torch.sigmoid(t["gate"][i - 1])
            d_act = g["y"] @ self.weight(f"{i - 1}.down")
            d_up = torch.cat([d_act * up * s * (1 + gate * (1 - s)), d_act * gate * s], 1)
            dn = d_up @ self.weight(f"{i - 1}.up")
        return og.onecomp_embedding_backward(tokens, dh, self.table.shape[0], scale=self.scale, base=d_table, d_table=d_table)

    def weight(self, name: str) -> torch.Tensor:
        """What a layer multiplies with: its dequantized weight once it is quantized."""
        return self.codes[name]["W_hat"].to(self.table.dtype) if name in self.codes else self.linear[name]


def text(vocab: int, n: int, seed: int):
    """Tokens of log-uniform frequency and what follows them; one in ten targets is left out."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    ids = (vocab ** torch.rand(n + 1, generator=gen, device=DEV)).long().sub_(1).clamp_(0, vocab - 1).to(torch.int32)
    targets = ids[1:].clone()
    targets[torch.rand(n, generator=gen, device=DEV) < 0.1] = -1
    return ids[:-1].contiguous(), targets


def run(vocab=2000, width=256, depth=2, tokens=4096, bits=8, steps=10, lr=1e-3, max_norm=1.0, say=print):
    """Returns (perplexity before quantization, after it, mean losses while the table is tuned)."""
    model = Model(vocab, width, depth)
    ids, targets = text(vocab, tokens, 1)
    kept = (targets >= 0).float()
    d_loss = kept / kept.sum()
    gram = {n: torch.zeros(w.shape[1], w.shape[1], device=DEV) for n, w in model.linear.items()}
    loss, _ = model.forward(ids, targets, lambda name, rows: og.onecomp_hessian_accumulate(rows, gram[name]))
    before = float(torch.exp((loss * d_loss).sum()))
    model.quantize(gram, bits)
    loss, t = model.forward(ids, targets)
    after = float(torch.exp((loss * d_loss).sum()))
    say(f"perplexity {before:.3f}, with layers of {bits} bits {after:.3f}")
    master = model.table.float()
    adam, losses = torch.optim.Adam([master.requires_grad_(False)], lr=lr), []
    for step in range(steps):
        loss, t = model.forward(ids, targets)
        losses.append(float((loss * d_loss).sum()))
        grad = model.table_gradient(ids, targets, t, d_loss)
        (clipped,), norm = og.onecomp_clip_gradients([grad], max_norm)
        master.grad = clipped.float()
        adam.step()
        model.table = master.to(model.table.dtype)
        say(f"step {step:3d}  loss {losses[-1]:.5f}  gradient norm {float(norm):.4f}")
    return before, after, losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("vocab", 2000), ("width", 256), ("depth", 2), ("tokens", 4096), ("bits", 8), ("steps", 10)):
        ap.add_argument("--" + name, type=int, default=default)
    run(**vars(ap.parse_args()))

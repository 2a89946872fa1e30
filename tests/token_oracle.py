"""Plain 64-bit forms of the operators from tokens to the loss, with bounds entry by entry on what a right kernel may be off."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}    # half a step, relative
E = 2.0 ** -24                                                   # of a 32-bit operation


def inside(ids, vocab):
    return (ids >= 0) & (ids < vocab)


def embedding_grad(tokens, d_out, vocab, scale, base=None):
    """(gradient, bound): the additions of a row's tokens in 32 bits, the product with the scale, the addition to base, the
    rounding of the result."""
    ok = inside(tokens, vocab)
    ids, d = tokens[ok].long(), d_out[ok].double()
    zero = torch.zeros(vocab, d_out.shape[1], dtype=torch.float64, device=d_out.device)
    total, size = zero.index_add(0, ids, d) * scale, zero.index_add(0, ids, d.abs()) * abs(scale)
    many = torch.zeros(vocab, dtype=torch.float64, device=d_out.device).index_add(0, ids, torch.ones_like(ids, dtype=torch.float64))
    if base is not None:
        total = total + base.double()
    # a sum of c terms in any fixed order: at most c - 1 additions on a term's way, one more for the product and base each
    bound = (many[:, None] + 2) * E * size * 1.01 + E * total.abs() + HALF[d_out.dtype] * total.abs() * 1.01
    return total, bound + 1e-40


def quantize(x):
    """Codes, scales and sums as the definition has them: scales and quotients are numbers of 32 bits."""
    top = x.float().abs().amax(1)
    scale = top / torch.full_like(top, 127.0)        # divided: by a number, it would be multiplied with the rounded 1 / 127
    codes = torch.where(scale[:, None] > 0, (x.float() / scale[:, None]).round().clamp(-127, 127), torch.zeros((), device=x.device))
    return codes.to(torch.int8), scale, codes.double().sum(1).to(torch.int32)


def linear(codes, token_scales, q, scales, zeros, bias, dtype):
    """(y, bound): the sum is exact; its conversion, two products and the addition of the bias round, then the result."""
    s = torch.mm(codes.double(), (q.double() - zeros.double().reshape(-1, 1)).t().contiguous())
    y = s * token_scales.double()[:, None] * scales.double().reshape(1, -1)
    size = y.abs()
    if bias is not None:
        y = y + bias.double()
    return y, 4 * E * size + (E + HALF[dtype]) * y.abs() * 1.01 + 1e-40


class Loss:
    """The loss over a vocabulary in 64 bits; left-out tokens never enter."""

    def __init__(self, h, weight, targets, scale=1.0):
        self.dtype, self.scale, self.device = h.dtype, scale, h.device
        self.n, (self.vocab, self.width) = h.shape[0], weight.shape
        self.kept = torch.nonzero(inside(targets, self.vocab))[:, 0]
        self.H, self.W = h[self.kept].double(), weight.double()
        self.t = targets[self.kept].long()
        self.rows = torch.arange(len(self.kept), device=self.device)
        Wt = self.W.t().contiguous()
        self.z = torch.mm(self.H, Wt) * scale
        # products of bf16 are exact in 32 bits, those of fp32 round; width additions; the product with the scale
        size = torch.mm(self.H.abs(), Wt.abs()) * scale
        self.z_off = (self.width + 3) * E * size
        self.lse = torch.logsumexp(self.z, 1) if len(self.kept) else torch.zeros(0, dtype=torch.float64, device=self.device)
        top = self.z.abs().amax(1) if len(self.kept) else self.lse
        worst = self.z_off.amax(1) if len(self.kept) else self.lse
        # arguments of the powers of two: the maximum and the product round (2 E |z|), exponentials and logarithms of the hardware
        # (2 steps each), sums of 64 logits, two halves, two waves, and tiles one by one
        tiles = -(-self.vocab // 128)
        self.lse_off = worst + 8 * E * top + (64 + 16 + tiles) * E + 8 * E * self.lse.abs() + 4 * E

    def spread(self, x, value=0.0):
        out = torch.full((self.n, *x.shape[1:]), value, dtype=torch.float64, device=self.device)
        out[self.kept] = x
        return out

    def forward(self):
        """((loss, lse), bounds)"""
        hit = self.z[self.rows, self.t]
        off = self.lse_off + self.z_off[self.rows, self.t] + 8 * E * hit.abs()
        return (self.spread(self.lse - hit), self.spread(self.lse)), (self.spread(off), self.spread(self.lse_off))

    def backward(self, d_loss, d_lse=None):
        """((dh, dweight), bounds), from log-sum-exps that are as far off as the forward call's may be"""
        dl = d_loss[self.kept].double()
        both = dl if d_lse is None else dl + d_lse[self.kept].double()
        p = torch.exp(self.z - self.lse[:, None]) * both[:, None]
        g = p.clone()
        g[self.rows, self.t] -= dl
        half, n = HALF[self.dtype], len(self.kept)
        # of a probability: what the exponent is off by (rounded log-sum-exp and argument among it), the exponential, the product
        # with the gradient, which is itself a rounded sum; then the difference, and g's own rounding
        p_off = p.abs() * (self.z_off + self.lse_off[:, None] + 4 * E * (self.z.abs() + self.lse.abs()[:, None]) + 6 * E) * 1.05
        # (d_loss + d_lse rounds relative to itself)
        g_off = p_off + E * g.abs() + half * (g.abs() + p_off)
        s = self.scale
        dh, dw = torch.mm(g, self.W) * s, torch.mm(g.t().contiguous(), self.H) * s
        dh_off = (torch.mm(g_off, self.W.abs()) + (self.vocab + 24) * E * torch.mm(g.abs() + g_off, self.W.abs())) * s
        dw_off = (torch.mm(g_off.t().contiguous(), self.H.abs()) + (n + 24) * E * torch.mm((g.abs() + g_off).t().contiguous(), self.H.abs())) * s
        dh_off = dh_off + (half + 2 * E) * (dh.abs() + dh_off) + 1e-38
        dw_off = dw_off + (half + 2 * E) * (dw.abs() + dw_off) + 1e-38
        return (self.spread(dh), dw), (self.spread(dh_off), dw_off)


def log_uniform_ids(gen, n, vocab, outside, mark, device):
    rank = torch.exp(torch.rand(n, generator=gen, device=device) * math.log(max(vocab, 2))).long().sub_(1).clamp_(0, vocab - 1)
    ids = torch.randperm(vocab, generator=gen, device=device)[rank].to(torch.int32)
    return ids.masked_fill_(torch.rand(n, generator=gen, device=device) < outside, mark)

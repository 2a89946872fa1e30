"""Attention of packed sequences in 64 bits, one sequence and head at a time, with the bounds that the kernels' roundings
give: each sum is returned together with the sum of its terms' magnitudes, and a rounding of a factor to `u` relative moves
the sum by at most u times that."""
import math

import torch

TINY = 2.0 ** -126     # probabilities below the smallest normal number may be taken as 0
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def attention(q, k, v, cu_q, cu_k, causal, scale, len_k=None, d_out=None):
    """dict of (value, bound) for out, lse and, with d_out, dq, dk, dv: all float64."""
    dev, dtype = q.device, q.dtype
    u, u32 = U[dtype], 2.0 ** -24
    cu_q, cu_k = cu_q.tolist(), cu_k.tolist()
    lens = len_k.tolist() if len_k is not None else None
    H, G, D = q.shape[1], k.shape[1], q.shape[2]

    def zeros(*shape):
        return [torch.zeros(*shape, dtype=torch.float64, device=dev) for _ in range(2)]

    res = {"out": zeros(q.shape), "lse": zeros(H, q.shape[0])}
    res["lse"][0].fill_(-math.inf)
    if d_out is not None:
        res.update(dq=zeros(q.shape), dk=zeros(k.shape), dv=zeros(k.shape))
    for i in range(len(cu_q) - 1):
        a = cu_q[i + 1] - cu_q[i]
        b = cu_k[i + 1] - cu_k[i] if lens is None else lens[i]
        rows, keys = slice(cu_q[i], cu_q[i] + a), slice(cu_k[i], cu_k[i] + b)
        if a == 0 or b == 0:
            continue
        seen = torch.ones(a, b, dtype=torch.bool, device=dev)
        if causal:
            seen = seen.tril(b - a)
        for h in range(H):
            g = h // (H // G)
            Q, K, V = q[rows, h].double(), k[keys, g].double(), v[keys, g].double()
            S = torch.where(seen, scale * (Q @ K.t()), -math.inf)
            lse = torch.logsumexp(S, 1)
            P = torch.where(seen, torch.exp(S - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
            # scores are fp32 sums of D products: their error is that of the exponent, with the maximum and the logarithm
            size = torch.where(seen, scale * (Q.abs() @ K.abs().t()), 0.0).amax(1, keepdim=True)
            eps = (D + 16) * u32 * size + 64 * u32             # relative, of every probability of the row
            sums = b * u32                                     # of fp32 sums over keys
            A = P @ V.abs()
            O = P @ V
            res["out"][0][rows, h] = O
            res["out"][1][rows, h] = (u + 2 * eps + 2 * sums) * A + u * O.abs() + TINY * V.abs().sum(0)
            res["lse"][0][h, rows] = lse
            res["lse"][1][h, rows] = eps[:, 0] + sums + 4 * u32 * torch.where(lse == -math.inf, 0.0, lse.abs())
            if d_out is None:
                continue
            dO = d_out[rows, h].double()
            dP = dO @ V.t()
            delta = (dO * O).sum(1, keepdim=True)
            dS = P * (dP - delta)
            # delta comes from the rounded output; dP is an fp32 sum of D products
            off = (dO.abs() * ((2 * u + 2 * eps + 2 * sums) * A)).sum(1, keepdim=True) + D * u32 * (dO.abs() @ V.abs().t() + (dO.abs() * A).sum(1, keepdim=True))
            eps2 = 2 * eps + sums                              # P anew from the stored lse
            err = (u + eps2) * dS.abs() + P * off * (1 + u) + TINY * (dP.abs() + delta.abs()) * seen
            n = (a * (H // G) + D) * u32
            dQ = scale * (dS @ K)
            res["dq"][0][rows, h] = dQ
            res["dq"][1][rows, h] = scale * (err @ K.abs() + (sums + n) * (dS.abs() @ K.abs())) + u * dQ.abs()
            res["dk"][0][keys, g] += scale * (dS.t() @ Q)
            res["dk"][1][keys, g] += scale * (err.t() @ Q.abs() + n * (dS.abs().t() @ Q.abs()))
            res["dv"][0][keys, g] += P.t() @ dO
            res["dv"][1][keys, g] += ((u + eps2) * P + TINY * seen).t() @ dO.abs() + n * (P.t() @ dO.abs())
    if d_out is not None:
        for name in ("dk", "dv"):
            res[name][1] += u * res[name][0].abs()
    return res


def check(got, want, name):
    """Every entry within its bound (and the smallest numbers of the type); infinities and zeros where they belong."""
    value, bound = want
    got = got.double()
    fine = torch.isfinite(value)
    assert torch.equal(got[~fine], value[~fine]), f"{name}: entries that are not finite"
    off = (got[fine] - value[fine]).abs()
    room = 1.02 * bound[fine] + 1e-37
    bad = ~(off <= room)
    if bool(bad.any()):
        at = int((off / room).nan_to_num(math.inf).argmax())
        raise AssertionError(f"{name}: {int(bad.sum())} of {off.numel()} entries outside their bound, worst {float(off.flatten()[at]):.3g} "
                             f"of {float(room.flatten()[at]):.3g} (value {float(value[fine].flatten()[at]):.3g})")

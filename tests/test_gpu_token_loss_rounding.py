"""What the rounding of the logits' gradients to bf16 leaves in the loss's gradients, where all kept tokens have one weight."""
import pytest
import torch

import paper_2603_28845_amd as og
from token_oracle import Loss

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF, E = 2.0 ** -8, 2.0 ** -24


def _along(got, want):
    """How much longer `got` is than `want`, along `want`, relative."""
    return float(((got.double() - want) * want).sum() / want.square().sum())


def _rounded(want):
    """Ten standard deviations of what independent roundings of the results, each by HALF of its size at most, add to that."""
    return 10 * HALF / 3 ** 0.5 * float(want.pow(4).sum().sqrt() / want.square().sum())


@pytest.mark.parametrize("weight", [1.0, 1.0039, 1.25, 5 / 3, 1.996, 1 / 4915, 1.0039e-20])
@pytest.mark.parametrize("outside", [0.0, 0.4])
def test_one_weight_for_all_tokens(weight, outside):
    """Probabilities of some 1/4096: the targets' -d (1 - p) are the gradients but for a few hundredths, and a common error of
    theirs would be one of all results."""
    gen = torch.Generator(device=DEV).manual_seed(7)
    n, width, vocab = 300, 512, 4096
    h = torch.randn(n, width, generator=gen, device=DEV).bfloat16()
    w = (torch.randn(vocab, width, generator=gen, device=DEV) * 0.25 * width ** -0.5).bfloat16()
    targets = torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    targets[torch.rand(n, generator=gen, device=DEV) < outside] = -1
    d_loss = torch.full((n,), weight, device=DEV)
    d_loss[targets < 0] = float("inf")                             # of left-out tokens: not looked at
    ref = Loss(h, w, targets)
    _, lse = og.onecomp_token_loss_forward(h, w, targets)
    dh, dw = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse)
    (want_dh, want_dw), _ = ref.backward(d_loss)
    # d (1 - p), in units of d's digits, is off by p, or by 2^-9 at most where p is more than that; the other entries by HALF of
    # themselves, which counts by how far their rows lie along the results.  What 32 bits round is below 2^-12 of either.
    p = torch.exp(ref.z - ref.lse[:, None])
    mine = p[ref.rows, ref.t].clamp_max(2.0 ** -9)
    d = float(d_loss[ref.kept[0]].double())
    W, H, dh_kept = ref.W, ref.H, want_dh[ref.kept]
    at_target = (mine * (W[ref.t] * dh_kept).sum(1).abs()).sum() * d
    others = HALF * (p * torch.mm(dh_kept, W.t().contiguous()).abs()).sum() * d
    off = float((at_target + others) / dh_kept.square().sum()) + _rounded(dh_kept) + 2.0 ** -12
    assert off < 1e-3 and abs(_along(dh, want_dh)) <= off, (off, _along(dh, want_dh))
    at_target = (mine * (H * want_dw[ref.t]).sum(1).abs()).sum() * d
    others = HALF * (p * torch.mm(H, want_dw.t().contiguous()).abs()).sum() * d
    off = float((at_target + others) / want_dw.square().sum()) + _rounded(want_dw) + 2.0 ** -12
    assert off < 1e-3 and abs(_along(dw, want_dw)) <= off, (off, _along(dw, want_dw))


def test_largest_weight_among_unequal_ones_and_none():
    """The digits of the largest weight are the unit; weights of zero, and none at all, leave 1."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    n, width, vocab = 130, 64, 700
    h = torch.randn(n, width, generator=gen, device=DEV).bfloat16()
    w = (torch.randn(vocab, width, generator=gen, device=DEV) * width ** -0.5).bfloat16()
    targets = torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    _, lse = og.onecomp_token_loss_forward(h, w, targets)
    for d_loss in (torch.zeros(n, device=DEV), -torch.rand(n, generator=gen, device=DEV), torch.rand(n, generator=gen, device=DEV) * torch.arange(n, device=DEV).eq(n - 1)):
        dh, dw = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse)
        (want_dh, want_dw), (dh_off, dw_off) = Loss(h, w, targets).backward(d_loss)
        assert bool(((dh.double() - want_dh).abs() <= dh_off).all()) and bool(((dw.double() - want_dw).abs() <= dw_off).all())
    # a weight that is not finite reaches its own token's results, and those of the weight
    d_loss = torch.rand(n, generator=gen, device=DEV)
    clean, _ = og.onecomp_token_loss_backward(d_loss * torch.arange(n, device=DEV).ne(3), h, w, targets, lse)
    d_loss[3] = float("inf")
    dh, _ = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse)
    assert not bool(dh[3].isfinite().any()) and torch.equal(dh[4:], clean[4:]) and torch.equal(dh[:3], clean[:3])

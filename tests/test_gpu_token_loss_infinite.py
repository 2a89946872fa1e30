"""Logits of +inf and -inf: log-sum-exps and losses as the definition has them."""
import pytest
import torch

import paper_2603_28845_amd as og

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,vocab", [(1, 9), (4, 1000), (30, 5000), (70, 40), (300, 513), (1100, 700), (4, 70001), (2100, 8000)])
def test_infinite_logits(dtype, n, vocab):
    """Column 1 of the weight holds +inf for entry `up`, -inf for `down`; of h it holds 1, -1 in turn, and NaN for one token."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    h = torch.randn(n, 64, generator=gen, device=DEV).to(dtype)
    w = (torch.randn(vocab, 64, generator=gen, device=DEV) * 0.2).to(dtype)
    up, down = vocab // 2, vocab - 1
    h[:, 1] = 1 - 2 * (torch.arange(n, device=DEV) % 2).to(dtype)
    w[:, 1] = 0
    w[up, 1], w[down, 1] = INF, -INF
    if n > 3:
        h[3, 2] = float("nan")
    targets = torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    targets[:2] = up
    loss, lse = (t.cpu().double() for t in og.onecomp_token_loss_forward(h, w, targets))
    z = h.cpu().double() @ w.cpu().double().t()
    want, hit = torch.logsumexp(z, 1), z[torch.arange(n), targets.cpu().long()]
    assert torch.equal(lse.isnan(), want.isnan()) and torch.equal(lse == INF, want == INF) and bool((lse == INF).any())
    assert torch.equal(loss.isnan(), (want - hit).isnan()) and torch.equal(loss == INF, want - hit == INF)
    # 64 products and additions, the joining of up to 70001 terms, all of logits below 32
    ok = want.isfinite()
    assert bool(((lse - want).abs()[ok] <= (64 + 64 + vocab / 32) * 2.0 ** -24 * 32).all())


@pytest.mark.parametrize("scale", [2.0 ** 60, 1.0])
def test_logits_past_the_largest_number(scale):
    """Logits that 32 bits hold only as infinities."""
    h, w = torch.zeros(70, 8, device=DEV), torch.zeros(200, 8, device=DEV)
    h[:, 0] = 2.0 ** 40
    w[:, 0] = torch.linspace(-1, 1, 200, device=DEV) * (2.0 ** 60 if scale > 1 else 2.0 ** 100)
    targets = torch.arange(70, device=DEV, dtype=torch.int32)
    for many in (70, 5):
        loss, lse = og.onecomp_token_loss_forward(h[:many], w, targets[:many], scale=scale)
        assert bool((lse == INF).all()) and bool((loss == INF).all())


@pytest.mark.parametrize("n", [6, 200])
def test_gradients_stay_with_what_is_infinite(n):
    """A logit of -inf takes no part; one of +inf leaves its token's dh and its entry's row of dweight without a value, no others."""
    h = torch.randn(n, 64, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    w = torch.randn(500, 64, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16()
    h[:, 1], w[:, 1] = -1, 0
    h[2, 1] = 1
    w[7, 1] = INF
    targets = torch.full((n,), 3, dtype=torch.int32, device=DEV)
    loss, lse = og.onecomp_token_loss_forward(h, w, targets)
    keep = torch.arange(n, device=DEV) != 2
    assert float(loss[2]) == INF and bool(loss[keep].isfinite().all())
    dh, dw = og.onecomp_token_loss_backward(torch.ones(n, device=DEV), h, w, targets, lse)
    others = torch.arange(64, device=DEV) != 1                    # 0 * inf has no value: column 1 of dh is left open
    assert bool(dh[keep][:, others].isfinite().all()) and bool(dh[2].isnan().all())
    assert bool(dw[7].isnan().all()) and bool(dw[torch.arange(500, device=DEV) != 7].isfinite().all())

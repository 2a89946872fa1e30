"""The loss over a vocabulary and its gradients against plain forms in 64 bits, with bounds from the roundings."""
import pytest
import torch

import paper_2603_28845_amd as og
from token_oracle import Loss, log_uniform_ids

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _inputs(gen, n, width, vocab, dtype, outside=0.0, level=2.0):
    h = torch.randn(n, width, generator=gen, device=DEV).to(dtype)
    w = (torch.randn(vocab, width, generator=gen, device=DEV) * level * width ** -0.5).to(dtype)
    return h, w, log_uniform_ids(gen, n, vocab, outside, -100, DEV)


def _check(name, got, want, off):
    bad = ~((got.double() - want).abs() <= off)
    assert not bool(bad.any()), (name, int(bad.sum()), float(((got.double() - want).abs() / off.clamp_min(1e-300)).max()))


SIZES = [(1, 8, 1, 0.0), (1, 64, 777, 0.0), (2, 16, 128, 0.0), (16, 4096, 1000, 0.0), (17, 200, 257, 0.1), (31, 72, 5000, 0.0), (33, 1000, 129, 0.3),
         (64, 136, 2049, 0.0), (65, 8, 300, 0.5), (128, 96, 383, 0.0), (129, 520, 1024, 0.2), (200, 40, 30001, 0.6), (300, 264, 513, 0.0), (1000, 128, 5003, 0.4),
         (257, 64, 50000, 0.1), (16500, 16, 17001, 0.05)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,width,vocab,outside", SIZES)
def test_loss_and_gradients(dtype, n, width, vocab, outside):
    gen = _gen(n + width + vocab)
    h, w, targets = _inputs(gen, n, width, vocab, dtype, outside)
    scale = 0.7 if vocab % 2 else 1.0
    ref = Loss(h, w, targets, scale)
    loss, lse = og.onecomp_token_loss_forward(h, w, targets, scale=scale)
    want, off = ref.forward()
    _check("loss", loss, want[0], off[0])
    _check("lse", lse, want[1], off[1])
    d_loss = torch.rand(n, generator=gen, device=DEV) / n
    d_lse = torch.randn(n, generator=gen, device=DEV) * 0.1 / n if n % 2 else None
    dh, dw = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse, scale=scale, d_lse=d_lse)
    want, off = ref.backward(d_loss, d_lse)
    _check("dh", dh, want[0], off[0])
    _check("dweight", dw, want[1], off[1])
    # each alone, and again: the same bits
    again, none = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse, scale=scale, d_lse=d_lse, want_dweight=False)
    assert none is None and torch.equal(again, dh)
    none, again = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse, scale=scale, d_lse=d_lse, want_dh=False)
    assert none is None and torch.equal(again, dw)
    again, none = og.onecomp_token_loss_forward(h, w, targets, scale=scale, want_lse=False)
    assert none is None and torch.equal(again, loss)


@pytest.mark.parametrize("n", [5, 200, 400])
def test_gradients_by_differences(n):
    """Along a direction, the loss changes as the gradients say: central differences in 64 bits of the definition itself."""
    gen = _gen(n)
    h, w, targets = _inputs(gen, n, 48, 90, F32, 0.2)
    d_loss = torch.rand(n, generator=gen, device=DEV)
    _, lse = og.onecomp_token_loss_forward(h, w, targets)
    dh, dw = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse)
    eh, ew = torch.randn_like(h), torch.randn_like(w)
    step = 2.0 ** -12                                              # differences are off by step^2 of the third derivatives, a few 1e-7 of the size

    def value(sign):
        z = torch.mm(h.double() + sign * step * eh.double(), (w.double() + sign * step * ew.double()).t().contiguous())
        ok = targets >= 0
        t = torch.where(ok, targets, 0).long()
        return float((d_loss.double() * ok * (torch.logsumexp(z, 1) - z[torch.arange(n, device=DEV), t])).sum())

    along = (value(1) - value(-1)) / (2 * step)
    parts = (dh.double() * eh.double()).sum() + (dw.double() * ew.double()).sum()
    size = float((dh.double() * eh.double()).abs().sum() + (dw.double() * ew.double()).abs().sum())
    assert abs(along - float(parts)) <= 1e-5 * size


def test_targets_outside_leave_their_tokens_out():
    gen = _gen(3)
    h, w, targets = _inputs(gen, 150, 64, 500, BF16)
    targets[::3] = torch.tensor([-1, -100, 500, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV).repeat(10)
    out = torch.arange(150, device=DEV) % 3 == 0
    h[out] = float("nan")                                          # never read into anything
    d_loss = torch.rand(150, generator=gen, device=DEV)
    d_loss[out] = float("nan")
    loss, lse = og.onecomp_token_loss_forward(h, w, targets)
    lse_there = lse.clone()
    lse_there[out] = float("nan")
    dh, dw = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse_there)
    ref = Loss(h, w, targets)
    want, off = ref.forward()
    _check("loss", loss, want[0], off[0])
    want, off = ref.backward(d_loss)
    _check("dh", dh, want[0], off[0])
    _check("dweight", dw, want[1], off[1])
    assert not bool(loss[out].any()) and not bool(lse[out].any()) and not bool(dh[out].any())


@pytest.mark.parametrize("n", [1, 20, 300])
def test_all_tokens_left_out_or_none_there(n):
    h, w = torch.ones(n, 32, device=DEV, dtype=BF16), torch.ones(70, 32, device=DEV, dtype=BF16)
    targets = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    loss, lse = og.onecomp_token_loss_forward(h, w, targets)
    dh, dw = og.onecomp_token_loss_backward(torch.ones(n, device=DEV), h, w, targets, lse)
    assert not any(bool(t.any()) for t in (loss, lse, dh, dw))
    dw = torch.full_like(w, 3.0)
    loss, lse = og.onecomp_token_loss_forward(h[:0], w, targets[:0])
    dh, _ = og.onecomp_token_loss_backward(torch.ones(0, device=DEV), h[:0], w, targets[:0], lse, dweight=dw)
    assert loss.shape == (0,) and dh.shape == (0, 32) and not bool(dw.any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [3, 40, 300])
def test_not_finite_rows_stay_by_themselves(dtype, n):
    gen = _gen(n)
    h, w, targets = _inputs(gen, n, 64, 333, dtype)
    clean = og.onecomp_token_loss_forward(h, w, targets)
    h[1, 5], h[2, 7] = float("nan"), float("inf")
    loss, lse = og.onecomp_token_loss_forward(h, w, targets)
    keep = torch.arange(n, device=DEV) % n != 1
    keep[2] = False
    assert bool(loss[1].isnan()) and not bool(loss[2].isfinite())
    assert torch.equal(loss[keep], clean[0][keep]) and torch.equal(lse[keep], clean[1][keep])
    dh, _ = og.onecomp_token_loss_backward(torch.ones(n, device=DEV), h, w, targets, lse)
    assert bool(dh[1].isnan().all()) and bool(dh[keep].isfinite().all())


@pytest.mark.parametrize("n", [2, 150])
def test_logits_far_apart(n):
    """Logits of +-1e4 and columns of -inf: the largest decides, nothing overflows."""
    w = torch.zeros(300, 16, device=DEV)
    w[:, 0] = torch.linspace(-1.0, 1.0, 300, device=DEV)
    w[7, 1] = -float("inf")
    h = torch.zeros(n, 16, device=DEV)
    h[:, 0], h[:, 1] = 1e4, 1.0
    h[1, 0] = -1e4
    targets = torch.full((n,), 299, dtype=torch.int32, device=DEV)
    loss, lse = og.onecomp_token_loss_forward(h, w, targets)
    z = torch.mm(h.double(), w.double().nan_to_num(neginf=0.0).t().contiguous())
    z[:, 7] = -float("inf")
    want = torch.logsumexp(z, 1)
    # 16 products, the scale, the joining: each rounding is 2^-24 of 1e4
    assert bool(((lse.double() - want).abs() <= 32 * 2.0 ** -24 * 1e4).all())
    assert bool(((loss.double() - (want - z[:, 299])).abs() <= 64 * 2.0 ** -24 * 1e4).all())


def test_strided_rows_side_stream_and_used_workspace():
    gen = _gen(9)
    n, width, vocab = 190, 72, 700
    rows = torch.randn(n, 104, generator=gen, device=DEV).to(BF16)
    table = torch.randn(vocab, 88, generator=gen, device=DEV).to(BF16)
    h, w = rows[:, 16:88], table[:, 8:80]
    targets = log_uniform_ids(gen, n, vocab, 0.2, -1, DEV)
    d_loss = torch.rand(n, generator=gen, device=DEV)
    dh_room, dw_room = torch.full((n, 96), 5.0, dtype=BF16, device=DEV), torch.full((vocab, 80), 5.0, dtype=BF16, device=DEV)
    ws = torch.full((1 << 25,), 255, dtype=torch.uint8, device=DEV)
    loss, lse = torch.full((n,), 9.0, device=DEV), torch.full((n,), 9.0, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        og.onecomp_token_loss_forward(h, w, targets, loss=loss, lse=lse, workspace=ws)
        og.onecomp_token_loss_backward(d_loss, h, w, targets, lse, dh=dh_room[:, 8:80], dweight=dw_room[:, 0:72], workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    ref = Loss(h, w, targets)
    want, off = ref.forward()
    _check("loss", loss, want[0], off[0])
    want, off = ref.backward(d_loss)
    _check("dh", dh_room[:, 8:80], want[0], off[0])
    _check("dweight", dw_room[:, :72], want[1], off[1])
    assert bool((dh_room[:, :8] == 5).all()) and bool((dh_room[:, 80:] == 5).all()) and bool((dw_room[:, 72:] == 5).all())


@pytest.mark.parametrize("n,width,vocab", [(20000, 16, 30000), (3, 4104, 530000), (70, 4104, 530000)])
def test_pieces_and_weights_past_32_bits(n, width, vocab):
    """Two pieces of logit gradients; weights of 2.2e9 entries, with a target in the last row."""
    gen = _gen(vocab)
    h, w, targets = _inputs(gen, n, width, vocab, BF16, 0.1 if n > 100 else 0.0)
    targets[-1] = vocab - 1
    ref = Loss(h, w, targets)
    loss, lse = og.onecomp_token_loss_forward(h, w, targets)
    want, off = ref.forward()
    _check("loss", loss, want[0], off[0])
    _check("lse", lse, want[1], off[1])
    d_loss = torch.rand(n, generator=gen, device=DEV) / n
    dh, dw = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse)
    want, off = ref.backward(d_loss)
    _check("dh", dh, want[0], off[0])
    _check("dweight", dw, want[1], off[1])

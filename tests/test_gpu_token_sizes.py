"""Every form of the products from tokens to the loss (tests/token_sizes.py) on inputs whose results are exact, so that each row, column
and inner index shows, and on whole-number logits, whose log-sum-exps hold each entry of the vocabulary."""
import pytest
import torch

import paper_2603_28845_amd as og
from token_oracle import E, Loss, inside, log_uniform_ids
from token_sizes import LAYER, LOSS, TABLE

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LOSSES = [(name, *size) for name, sizes in LOSS.items() for size in sizes]


def _whole(gen, rows, cols, most, dtype):
    return torch.randint(-most, most + 1, (rows, cols), generator=gen, device=DEV, dtype=torch.int8).to(dtype)


class Certain:
    """Each token has one entry of the vocabulary with logit 0; all others have -1000, so that its probability is 1 and theirs 0 in
    32 bits.  Columns by threes: in the first kind a token of h selects its entry, in the second h alone holds numbers, in the third
    weight alone.  Gradients of logits are then 0, d and -d, and sums of whole numbers."""

    def __init__(self, gen, n, width, vocab, dtype, live=None):
        a = max(1, width // 3)
        b = (width - a) // 2
        if live is None:
            live = torch.randperm(vocab, generator=gen, device=DEV)[:a]
        a = len(live)
        self.h, self.w = torch.zeros(n, width, dtype=dtype, device=DEV), torch.zeros(vocab, width, dtype=dtype, device=DEV)
        mine = torch.randint(0, a, (n,), generator=gen, device=DEV)
        mine[:a] = torch.arange(min(n, a), device=DEV)
        self.entry = live[mine]
        self.h[torch.arange(n, device=DEV), mine] = 1
        self.h[:, a:a + b] = _whole(gen, n, b, 8, dtype)
        self.w[:, :a] = -1000
        self.w[live, torch.arange(a, device=DEV)] = 0
        self.w[:, a + b:] = _whole(gen, vocab, width - a - b, 8, dtype)
        self.targets = log_uniform_ids(gen, n, vocab, 0.2 if n > 4 else 0.0, -1, DEV)
        self.targets[n // 2] = vocab - 1
        self.d = 2.0 ** torch.randint(0, 3, (n,), generator=gen, device=DEV).float()

    def check(self, scale):
        h, w, t = self.h, self.w, self.targets
        loss, lse = og.onecomp_token_loss_forward(h, w, t, scale=scale)
        ok = inside(t, w.shape[0])
        kept = torch.nonzero(ok)[:, 0]
        tk, ek, dk = t[kept].long(), self.entry[kept], self.d[kept].double()
        assert not bool(lse.any()) and not bool(loss[~ok].any())
        hit = tk == ek
        # -1000 times the scale, times log2(e) and its reverse: five roundings and the constants' own
        assert bool(((loss[kept].double() - torch.where(hit, 0.0, 1000.0 * scale)).abs() <= 8 * E * 1000 * scale).all())
        dh, dw = og.onecomp_token_loss_backward(self.d, h, w, t, lse, scale=scale)
        want = torch.zeros(h.shape, dtype=torch.float64, device=DEV)
        want[kept] = (w[ek].double() - w[tk].double()) * dk[:, None] * scale
        assert torch.equal(dh, want.float().to(h.dtype))
        rows, back = torch.unique(torch.cat([ek, tk]), return_inverse=True)
        parts = h[kept].double() * dk[:, None] * scale
        want = torch.zeros(len(rows), h.shape[1], dtype=torch.float64, device=DEV).index_add(0, back, torch.cat([parts, -parts]))
        assert torch.equal(dw[rows], want.float().to(h.dtype))
        dw[rows] = 0
        assert not bool(dw.any())


@pytest.mark.parametrize("name,n,width,vocab", LOSSES)
def test_loss_of_certain_tokens(name, n, width, vocab):
    gen = torch.Generator(device=DEV).manual_seed(n + width + vocab)
    Certain(gen, n, width, vocab, DTYPES[name]).check(0.5 if vocab % 2 else 1.0)


class Exact(Loss):
    """Logits of whole numbers: exact until they are scaled."""

    def __init__(self, h, weight, targets, scale):
        super().__init__(h, weight, targets, scale)
        self.z_off.zero_()
        self.lse_off = 8 * E * self.z.abs().amax(1) + (64 + 16 + self.vocab // 128 + 1) * E + 8 * E * self.lse.abs() + 4 * E


@pytest.mark.parametrize("name,n,width,vocab", LOSSES)
def test_loss_of_whole_logits(name, n, width, vocab):
    gen = torch.Generator(device=DEV).manual_seed(n + width + vocab)
    h, w = _whole(gen, n, width, 2, DTYPES[name]), _whole(gen, vocab, width, 2, DTYPES[name])
    targets = log_uniform_ids(gen, n, vocab, 0.1 if n > 4 else 0.0, -1, DEV)
    scale = 1.0
    while scale * 2 * width ** 0.5 > 2:                            # logits of a size of 1 to 2
        scale /= 2
    ref = Exact(h, w, targets, scale)
    (want_loss, want_lse), (off_loss, off_lse) = ref.forward()
    loss, lse = og.onecomp_token_loss_forward(h, w, targets, scale=scale)
    assert bool(((lse.double() - want_lse).abs() <= off_lse).all()) and bool(((loss.double() - want_loss).abs() <= off_loss).all())
    # what the inputs are worth: nine in ten entries have a larger share of some token than the bound, and would be missed (where the
    # bound's additions do not outgrow an entry's share, one in `vocab`: vocab^2 / 128 steps of 2^-24)
    if vocab <= 30000:
        assert float((torch.exp(ref.z - ref.lse[:, None]).amax(0) > off_lse[ref.kept].max()).double().mean()) > 0.9
    d_loss = torch.rand(n, generator=gen, device=DEV) / n
    dh, dw = og.onecomp_token_loss_backward(d_loss, h, w, targets, lse, scale=scale)
    (want_dh, want_dw), (off_dh, off_dw) = ref.backward(d_loss)
    assert bool(((dh.double() - want_dh).abs() <= off_dh).all()) and bool(((dw.double() - want_dw).abs() <= off_dw).all())


@pytest.mark.parametrize("name,n,width,vocab", [("bf16", 3, 4104, 530000), ("bf16", 70, 4104, 530000), ("f32", 3, 2056, 530000), ("f32", 40, 2056, 530000), ("bf16", 3, 32776, 65536)])
def test_certain_entries_past_32_bits(name, n, width, vocab):
    """Weights of more than 2^32 bytes: half of the tokens' entries lie behind them, the last one among these, and so does a target."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    border = -(-(1 << 32) // (width * (2 if name == "bf16" else 4)))
    assert border < vocab - 2
    far = torch.randint(border, vocab, (1,), generator=gen, device=DEV)
    live = torch.cat([torch.tensor([vocab - 1, 0, border], device=DEV), far[far != border], torch.randperm(border - 1, generator=gen, device=DEV)[:2] + 1])
    Certain(gen, n, width, vocab, DTYPES[name], torch.unique(live, sorted=False)).check(1.0)


@pytest.mark.parametrize("n,width,outputs", LAYER)
def test_layer(n, width, outputs):
    """Scales of one: the sums themselves, which 32 bits round once."""
    gen = torch.Generator(device=DEV).manual_seed(n + outputs)
    codes = torch.randint(-127, 128, (n, width), generator=gen, device=DEV, dtype=torch.int8)
    q = torch.randint(0, 256, (outputs, width), generator=gen, device=DEV, dtype=torch.uint8)
    z = torch.randint(0, 256, (outputs,), generator=gen, device=DEV).float()
    want = torch.mm(codes.double(), (q.double() - z.double()[:, None]).t().contiguous()).float()
    one = torch.ones(max(n, outputs), device=DEV)
    sums = codes.sum(1, dtype=torch.int32)
    for dtype in DTYPES.values():
        got = og.onecomp_linear_int8(codes, one[:n], sums, q, one[:outputs], z, dtype=dtype)
        assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("dtype", list(DTYPES.values()))
@pytest.mark.parametrize("n,width,vocab", TABLE)
def test_table(dtype, n, width, vocab):
    """Sums of whole numbers."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    tokens, d_out = log_uniform_ids(gen, n, vocab, 0.05, -1, DEV), _whole(gen, n, width, 100, dtype)
    ok = inside(tokens, vocab)
    want = torch.zeros(vocab, width, dtype=torch.float64, device=DEV).index_add(0, tokens[ok].long(), d_out[ok].double())
    assert torch.equal(og.onecomp_embedding_backward(tokens, d_out, vocab), want.float().to(dtype))

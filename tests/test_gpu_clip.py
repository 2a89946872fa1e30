"""Clipping of gradients to a global norm on the GPU, against 64 bits."""
import math

import pytest
import torch

import paper_2603_28845_amd as og

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
U = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def _grads(sizes, dtypes, seed, std=1.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return [torch.randn(n, generator=gen, device=DEV).mul_(std).to(dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def _check(grads, max_norm, out, norm):
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    f = min(1.0, max_norm / (want + 1e-6))
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for g, o in zip(grads, out):
        assert o.dtype == g.dtype
        # the factor is rounded to 32 bits, and so is the product before it gets the type's own bits
        room = (U[g.dtype] * 1.01 + 4 * 2.0 ** -24) * (g.double() * f).abs() + 1e-38
        assert bool(((o.double() - g.double() * f).abs() <= room).all())


@pytest.mark.parametrize("level", [0.5, 2.0, 1e6])
@pytest.mark.parametrize("dtypes", [[F32], [BF16], [F32, BF16]])
@pytest.mark.parametrize("sizes", [[1], [7, 0, 1, 3], [16384, 16385, 5], [3000000, 17], [i * 37 % 501 for i in range(250)]])
def test_sizes(sizes, dtypes, level):
    print(f"[case] {len(sizes)} tensors {dtypes} {level}", flush=True)
    grads = _grads(sizes, dtypes, 1)
    max_norm = math.sqrt(sum(sizes)) / level
    before = [g.clone() for g in grads]
    out, norm = og.onecomp_clip_gradients(grads, max_norm, out=[torch.full_like(g, 9.0) for g in grads])
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    _check(grads, max_norm, out, norm)
    inplace, norm2 = og.onecomp_clip_gradients(grads, max_norm)
    assert inplace is grads and float(norm2) == float(norm) and all(torch.equal(a, b) for a, b in zip(grads, out))


def test_slices_at_odd_addresses():
    wide = _grads([10000], [BF16], 2)[0]
    grads = [wide[1:3002], wide[3003:3004], wide[3005:9998]]
    outside = wide.clone()
    kept = [g.clone() for g in grads]
    out, norm = og.onecomp_clip_gradients(grads, 1.0)
    _check(kept, 1.0, out, norm)
    for at in (0, 3002, 3004, 9998, 9999):
        assert float(wide[at]) == float(outside[at])


def test_squares_that_fp32_cannot_hold():
    for std in (1e30, 1e-30):
        grads = _grads([5000, 33], [F32], 3, std)
        out, norm = og.onecomp_clip_gradients(grads, 1.0, out=[torch.empty_like(g) for g in grads])
        _check(grads, 1.0, out, norm)


def test_limits():
    grads = _grads([100], [F32], 4)
    out, norm = og.onecomp_clip_gradients(grads, math.inf, out=[torch.empty_like(grads[0])])
    assert torch.equal(out[0], grads[0])
    out, _ = og.onecomp_clip_gradients(grads, 0.0, out=[torch.empty_like(grads[0])])
    assert bool((out[0] == 0).all())
    zeros, norm = og.onecomp_clip_gradients([torch.zeros(5, device=DEV)], 1.0)
    assert float(norm) == 0 and bool((zeros[0] == 0).all())
    _, norm = og.onecomp_clip_gradients([], 1.0, norm=torch.full((), 7.0, device=DEV))
    assert float(norm) == 0


def test_not_finite():
    grads = _grads([100, 50], [F32, BF16], 5)
    grads[1][3] = math.inf
    out, norm = og.onecomp_clip_gradients(grads, 1.0, out=[torch.empty_like(g) for g in grads])
    assert float(norm) == math.inf and bool((out[0] == 0).all()) and math.isnan(float(out[1][3]))
    grads[1][3] = math.nan
    out, norm = og.onecomp_clip_gradients(grads, 1.0, out=[torch.empty_like(g) for g in grads])
    assert math.isnan(float(norm)) and bool(torch.isnan(out[0]).all())


def test_the_same_bits_every_time():
    grads = _grads([1 << 20, 12345, 1 << 18], [F32, BF16], 6)
    first = og.onecomp_clip_gradients(grads, 1.0, out=[torch.empty_like(g) for g in grads])
    for _ in range(3):
        again = og.onecomp_clip_gradients(grads, 1.0, out=[torch.empty_like(g) for g in grads])
        assert float(again[1]) == float(first[1]) and all(torch.equal(a, b) for a, b in zip(first[0], again[0]))

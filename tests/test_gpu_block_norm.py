"""The fused norms of a block and their gradients on the GPU against 64 bits, each entry within what fp32 arithmetic and the one
rounding of the result allow."""
import math

import pytest
import torch

import paper_2603_28845_amd as og

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
U = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
# fp32 roundings along one entry: a thread's sum of up to 32 squares, 6 and 16 more where lanes and waves meet, and the few
# operations on the way, taken twice (a norm's sum and its use)
C = 128 * 2.0 ** -24


def _inputs(rows, width, dtype, w_dtype, seed, y=True, post=False, gate="no", kind="rms", pad=0, offset=0.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, dtype=dtype, std=1.0):
        if pad and len(shape) == 2:      # rows of a wider buffer, from an odd element on
            wide = torch.full((shape[0], shape[1] + pad), math.nan, dtype=dtype, device=DEV)
            wide[:, 1:1 + shape[1]] = torch.randn(*shape, generator=gen, device=DEV).mul_(std)
            return wide[:, 1:1 + shape[1]]
        return torch.randn(*shape, generator=gen, device=DEV).mul_(std).to(dtype)

    layer = kind == "layer"
    x = {"h": normal(rows, width), "y": normal(rows, width) if y else None,
         "weight": 1 + normal(width, dtype=w_dtype, std=0.3), "bias": normal(width, dtype=w_dtype) if layer else None,
         "post_weight": 1 + normal(width, dtype=w_dtype, std=0.3) if post else None,
         "post_bias": normal(width, dtype=w_dtype) if post and layer else None,
         "gate": None if gate == "no" else normal(width, dtype=w_dtype) if gate == "channel" else normal(rows, width)}
    if offset:
        x["h"] += offset
    grads = {"dn": normal(rows, width), "dh_out": normal(rows, width)}
    return x, grads


class Exact:
    """A value in 64 bits with the bound of its error: sums and products of such."""

    def __init__(self, v, e=None):
        self.v = v.double()
        self.e = torch.zeros_like(self.v) if e is None else e

    def __add__(self, o):
        v = self.v + o.v
        return Exact(v, self.e + o.e + C / 64 * v.abs())

    def __mul__(self, o):
        v = self.v * o.v
        return Exact(v, self.e * o.v.abs() + o.e * self.v.abs() + self.e * o.e + C / 64 * v.abs())

    def mean(self):
        return Exact(self.v.mean(1, keepdim=True), (self.e + C * self.v.abs()).mean(1, keepdim=True))

    def sum(self):
        depth = self.v.shape[0] * 2.0 ** -24
        return Exact(self.v.sum(0), (self.e + (C + depth) * self.v.abs()).sum(0))

    def scaled(self, f):
        return Exact(f * self.v, abs(f) * self.e + C / 64 * (f * self.v).abs())


def _hat(x, kind, eps):
    """Normalised rows and 1 / size."""
    if kind == "layer":
        m = x.mean()
        x = x + m.scaled(-1.0)
    square = (x * x).mean()
    size = torch.sqrt(square.v + eps)
    # a relative error of the mean square is halved by the root
    inv = Exact(1 / size, (square.e / (2 * (square.v + eps)) + C) / size)
    return x * inv, inv


def _affine(x, w, b):
    x = x if w is None else x * Exact(w)
    return x if b is None else x + Exact(b)


def _forward(x, scale, eps, kind):
    h = Exact(x["h"])
    if x["y"] is not None:
        u = Exact(x["y"])
        if x["post_weight"] is not None:
            u = _affine(_hat(u, kind, eps)[0], x["post_weight"], x["post_bias"])
        if x["gate"] is not None:
            u = u * Exact(x["gate"])
        h = h.scaled(scale) + u
    return h, _affine(_hat(h, kind, eps)[0], x["weight"], x["bias"])


def _hat_grad(d, x, inv, kind):
    g = d + (x * (d * x).mean()).scaled(-1.0)
    if kind == "layer":
        g = g + d.mean().scaled(-1.0)
    return g * inv


def _backward(x, grads, scale, eps, kind):
    res = {}
    G = None if grads["dh_out"] is None else Exact(grads["dh_out"])
    if grads["dn"] is not None:
        dn = Exact(grads["dn"])
        hat, inv = _hat(Exact(x["h"]), kind, eps)
        res["weight"] = (dn * hat).sum()
        if kind == "layer":
            res["bias"] = dn.sum()
        back = _hat_grad(_affine(dn, x["weight"], None), hat, inv, kind)
        G = back if G is None else G + back
    res["h"] = G.scaled(scale) if x["y"] is not None else G
    if x["y"] is None:
        return res
    u = Exact(x["y"])
    if x["post_weight"] is not None:
        hat, inv = _hat(u, kind, eps)
        u = _affine(hat, x["post_weight"], x["post_bias"])
    if x["gate"] is not None:
        g = G * u
        res["gate"] = g.sum() if x["gate"].dim() == 1 else g
        G = G * Exact(x["gate"])
    if x["post_weight"] is not None:
        res["post_weight"] = (G * hat).sum()
        if kind == "layer":
            res["post_bias"] = G.sum()
        G = _hat_grad(_affine(G, x["post_weight"], None), hat, inv, kind)
    res["y"] = G
    return res


def _check(got, want, name):
    assert got.shape == want.v.shape, name
    off = (got.double() - want.v).abs()
    room = 1.01 * (want.e + U[got.dtype] * (want.v.abs() + want.e)) + 1e-37
    assert bool((off <= room).all()), f"{name}: {float((off / room).max()):.3g} of its bound, {int((off > room).sum())} of {off.numel()} entries"


def _run(x, grads, scale=1.0, eps=1e-6, kind="rms"):
    h, n = og.onecomp_block_norm_forward(**x, residual_scale=scale, eps=eps, kind=kind)
    want_h, want_n = _forward(x, scale, eps, kind)
    if x["y"] is not None:
        _check(h, want_h, "h'")
    _check(n, want_n, "n")
    back = dict(x, h=h)
    got = og.onecomp_block_norm_backward(grads["dn"], grads["dh_out"], **back, residual_scale=scale, eps=eps, kind=kind)
    want = _backward(back, grads, scale, eps, kind)
    assert {k for k, v in got.items() if v is not None} == set(want)
    for name in want:
        _check(got[name], want[name], "gradient of " + name)
    again = og.onecomp_block_norm_backward(grads["dn"], grads["dh_out"], **back, residual_scale=scale, eps=eps, kind=kind)
    for name in want:
        assert torch.equal(got[name], again[name]), name


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [1, 7, 64, 511, 512, 515, 1359, 2048, 4096, 4099, 8192, 8200, 14336, 16385, 28672, 32768])
def test_widths(width, dtype, kind):
    print(f"[case] width {width} {dtype} {kind}", flush=True)
    x, grads = _inputs(37, width, dtype, F32, 1, post=True, gate="channel", kind=kind)
    _run(x, grads, 0.5, kind=kind)


@pytest.mark.parametrize("rows", [1, 2, 255, 1024, 5000])
@pytest.mark.parametrize("width", [48, 1000, 4096])
def test_rows(rows, width):
    x, grads = _inputs(rows, width, BF16, BF16, 2, post=True, gate="rows")
    _run(x, grads)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype,w_dtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("y,post,gate", [(False, False, "no"), (True, False, "no"), (True, True, "no"), (True, False, "channel"), (True, False, "rows"),
                                         (True, True, "channel"), (True, True, "rows")])
def test_forms(y, post, gate, dtype, w_dtype, kind):
    x, grads = _inputs(70, 640, dtype, w_dtype, 3, y=y, post=post, gate=gate, kind=kind)
    _run(x, grads, 0.7, kind=kind)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_odd_strides_and_offsets(dtype):
    x, grads = _inputs(19, 1001, dtype, dtype, 4, post=True, gate="rows", kind="layer", pad=4)
    _run(x, grads, kind="layer")


@pytest.mark.parametrize("missing", ["dn", "dh_out"])
def test_one_gradient_alone(missing):
    x, grads = _inputs(33, 256, F32, F32, 5, post=True, gate="channel")
    grads[missing] = None
    if missing == "dn":
        h, _ = og.onecomp_block_norm_forward(**x)
        got = og.onecomp_block_norm_backward(None, grads["dh_out"], **dict(x, h=h))
        want = _backward(dict(x, h=h), grads, 1.0, 1e-6, "rms")
        assert got["weight"] is None
        for name in want:
            _check(got[name], want[name], name)
    else:
        _run(x, grads)


def test_means_far_from_zero():
    """Layer norms of rows whose mean is a hundred times their spread: the mean goes before squares are formed."""
    x, grads = _inputs(12, 4096, F32, F32, 6, y=False, kind="layer", offset=100.0)
    _run(x, grads, kind="layer")


def test_large_and_small_rows():
    x, grads = _inputs(8, 2048, F32, F32, 7, post=True)
    x["h"][1] *= 1e15
    x["y"][2] *= 1e-12
    x["h"][3] = 0
    x["y"][3] = 0
    _run(x, grads)


def test_gradients_against_differences():
    x, grads = _inputs(6, 40, F32, F32, 8, post=True, gate="rows", kind="layer")
    kw = dict(residual_scale=0.6, kind="layer", eps=1e-5)

    def value(x):
        h, n = og.onecomp_block_norm_forward(**x, **kw)
        return float((h.double() * grads["dh_out"].double()).sum() + (n.double() * grads["dn"].double()).sum())

    h, _ = og.onecomp_block_norm_forward(**x, **kw)
    got = og.onecomp_block_norm_backward(grads["dn"], grads["dh_out"], **dict(x, h=h), **kw)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    for name, g in got.items():
        step = torch.randn(g.shape, generator=gen, device=DEV)
        step /= step.norm()
        eps = 1e-2
        slope = (value(dict(x, **{name: x[name] + eps * step})) - value(dict(x, **{name: x[name] - eps * step}))) / (2 * eps)
        want = float((g.double() * step.double()).sum())
        # fp32 noise of values around 100 over 2e-2, and eps^2 times a third derivative
        assert abs(slope - want) <= 5e-3 + 5e-3 * float(g.double().norm()), name


@pytest.mark.parametrize("width", [1024, 9000])
def test_in_place_and_given_buffers(width):
    x, grads = _inputs(50, width, BF16, BF16, 10, post=True, gate="channel")
    h, n = og.onecomp_block_norm_forward(**x)
    mine = x["h"].clone()
    h2, n2 = og.onecomp_block_norm_forward(**dict(x, h=mine), h_out=mine)
    assert h2 is mine and torch.equal(h, h2) and torch.equal(n, n2)
    want = og.onecomp_block_norm_backward(grads["dn"], grads["dh_out"], **dict(x, h=h))
    dn, dh = grads["dn"].clone(), grads["dh_out"].clone()
    out = {"h": dh, "y": dn, "weight": torch.empty_like(x["weight"])}
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device=DEV)
    got = og.onecomp_block_norm_backward(dn, dh, **dict(x, h=h), out=out, workspace=ws)
    assert torch.equal(dh, want["h"]) and torch.equal(dn, want["y"]) and torch.equal(got["weight"], want["weight"])
    assert got["gate"] is None and got["post_weight"] is None


def test_no_rows():
    x, grads = _inputs(0, 64, F32, F32, 11, post=True, gate="channel")
    h, n = og.onecomp_block_norm_forward(**x)
    assert h.shape == n.shape == (0, 64)
    got = og.onecomp_block_norm_backward(grads["dn"], grads["dh_out"], **dict(x, h=h))
    assert all(bool((got[name] == 0).all()) for name in ("weight", "post_weight", "gate"))


def test_a_row_that_is_not_finite_stays_alone():
    x, _ = _inputs(9, 512, BF16, BF16, 12, post=True)
    clean = og.onecomp_block_norm_forward(**x)
    x["y"][4, 100] = math.nan
    got = og.onecomp_block_norm_forward(**x)
    for c, g in zip(clean, got):
        assert torch.equal(c[:4], g[:4]) and torch.equal(c[5:], g[5:]) and bool(torch.isnan(g[4].float()).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [1, 3, 7, 9, 1001, 1359, 4099, 9001])
def test_odd_rows_in_place_and_their_neighbours(width, dtype):
    """Rows that end inside a vector: results over the inputs are those beside them, and the entries between rows keep theirs."""
    print(f"[case] width {width} {dtype}", flush=True)
    x, grads = _inputs(21, width, dtype, dtype, 13, post=True, gate="rows")

    def over(values):
        whole = torch.full((values.shape[0], width + 3), 77.0, dtype=dtype, device=DEV)
        whole[:, :width] = values
        return whole, whole[:, :width]

    h, n = og.onecomp_block_norm_forward(**x)
    want = og.onecomp_block_norm_backward(grads["dn"], grads["dh_out"], **dict(x, h=h))
    (all_h, mine), (all_dn, dn), (all_dh, dh) = over(x["h"]), over(grads["dn"]), over(grads["dh_out"])
    h2, n2 = og.onecomp_block_norm_forward(**dict(x, h=mine), h_out=mine)
    assert torch.equal(h, h2) and torch.equal(n, n2)
    og.onecomp_block_norm_backward(dn, dh, **dict(x, h=mine), out={"h": dh, "y": dn})
    assert torch.equal(dh, want["h"]) and torch.equal(dn, want["y"])
    for whole in (all_h, all_dn, all_dh):
        assert bool((whole[:, width:] == 77.0).all())

"""Norms without an eps: parameters' gradients where the rows do not fill a workgroup's groups of rows."""
import pytest
import torch

import paper_2603_28845_amd as og
from test_gpu_block_norm import BF16, F32, _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 3, 37])
@pytest.mark.parametrize("width", [64, 500, 2048, 4096, 9000])
def test_no_eps(width, rows, dtype, kind):
    print(f"[case] {rows} x {width} {dtype} {kind}", flush=True)
    for gate in ("channel", "rows"):
        x, grads = _inputs(rows, width, dtype, F32, 20, post=True, gate=gate, kind=kind)
        _run(x, grads, 0.5, eps=0.0, kind=kind)


def test_no_eps_and_no_norm_in_front():
    """Only the norm behind the block: the one in front has no gradient."""
    x, grads = _inputs(3, 64, F32, F32, 21, post=True)
    h, _ = og.onecomp_block_norm_forward(**x, eps=0.0)
    got = og.onecomp_block_norm_backward(None, grads["dh_out"], **dict(x, h=h), eps=0.0)
    assert all(bool(torch.isfinite(t).all()) for t in got.values() if t is not None)

"""What the norms' gradients write besides their results, and what they may be written over."""
import pytest
import torch

import paper_2603_28845_amd as og

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _inputs(rows, width, dtype, kind, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV).to(dtype)

    layer = kind == "layer"
    x = dict(h=normal(rows, width), y=normal(rows, width), weight=normal(width), bias=normal(width) if layer else None, post_weight=normal(width),
             post_bias=normal(width) if layer else None, gate=normal(rows, width), kind=kind)
    return x, normal(rows, width), normal(rows, width)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [640, 4099, 8200, 9000, 20000])
def test_rows_gradients_alone_leave_the_workspace(width, dtype, kind):
    """dh, dy and a gate's gradient without any parameter's: the same as beside them, and nothing else is written."""
    print(f"[case] {width} {dtype} {kind}", flush=True)
    x, dn, dh_out = _inputs(21, width, dtype, kind, 1)
    want = og.onecomp_block_norm_backward(dn, dh_out, **x)
    room = torch.full((1 << 20,), 77, dtype=torch.uint8, device=DEV)
    out = {name: torch.empty_like(x[name]) for name in ("h", "y", "gate")}
    for ws in (room[1 << 19:(1 << 19) + 256], room[1 << 19:1 << 19]):
        og.onecomp_block_norm_backward(dn, dh_out, **x, out=out, workspace=ws)
        for name in out:
            assert torch.equal(out[name], want[name]), name
        assert bool((room == 77).all())


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("width", [640, 9000])
@pytest.mark.parametrize("over", [{"h": "h"}, {"h": "y"}, {"y": "y", "h": "dh_out"}, {"y": "h"}, {"gate": "gate"}, {"gate": "dn", "y": "gate"}])
def test_results_over_any_input(over, width, kind):
    """dh, dy and a gate's gradient written over what the call reads: the rows in place, and the parameters' sums over all of them."""
    print(f"[case] {over} {width} {kind}", flush=True)
    x, dn, dh_out = _inputs(40, width, BF16, kind, 2)
    want = og.onecomp_block_norm_backward(dn, dh_out, **x)
    x, given = dict(x), {"dn": dn.clone(), "dh_out": dh_out.clone()}
    for name in ("h", "y", "gate"):
        given[name] = x[name] = x[name].clone()
    out = {name: torch.empty_like(t) for name, t in x.items() if torch.is_tensor(t)}
    out.update({result: given[name] for result, name in over.items()})
    og.onecomp_block_norm_backward(given["dn"], given["dh_out"], **x, out=out)
    for name in out:
        assert torch.equal(out[name], want[name]), name

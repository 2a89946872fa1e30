"""Host-side checks of attention's arguments (no GPU): what a call makes of them before anything is launched."""
import ctypes

import pytest

from test_block_host import INVALID, P, UNSUPPORTED, WORKSPACE, _backward, _forward, _heads, _shape, lib  # noqa: F401


@pytest.mark.parametrize("total_q,total_k", [(3000, 100000), (40, 5000), (4, 200000)])
@pytest.mark.parametrize("name", ["onecomp_attention_workspace_bytes", "onecomp_attention_backward_workspace_bytes"])
def test_longest_lengths_beyond_the_tensors(lib, name, total_q, total_k):  # noqa: F811
    """A caller that does not know the longest sequence may say any number: no workspace grows with it beyond that of all tokens in one."""
    def need(max_q, max_k):
        return getattr(lib, name)(ctypes.byref(_shape(total_q=total_q, total_k=total_k, max_q=max_q, max_k=max_k)))

    want = need(total_q, total_k)
    for most in (1 << 40, 1 << 60, (1 << 60) + 1, 1 << 62, (1 << 63) - 1):
        assert need(total_q, most) == want
        # launch shapes of many queries need no more than those of few
        assert need(most, total_k) <= want and need(most, most) <= want


def test_results_over_what_is_still_read(lib):  # noqa: F811
    """Gradients of queries over q or d_out, which those of keys are formed from next, and the like: refused before anything runs."""
    def apart():
        return [_heads(data=P * (i + 1)) for i in range(8)]           # q, k, v, out, d_out, dq, dk, dv

    for result, over in ((5, 0), (5, 1), (5, 2), (5, 4), (6, 0), (6, 4), (7, 0), (7, 4), (6, 5), (7, 5), (7, 6)):
        views = apart()
        views[result] = views[over]
        assert _backward(lib, views=views) == INVALID, (result, over)
    q, k, v, out = apart()[:4]
    assert _forward(lib, q=q, k=k, v=v, out=k) == INVALID
    assert _forward(lib, q=q, k=k, v=v, out=v) == INVALID


def test_scales_beyond_what_the_arithmetic_holds(lib):  # noqa: F811
    """With 1e-38 the gradients' log-sum-exps over the scale were infinite, and dv 0; with 3e38 scale log2(e) was."""
    for call in (_forward, _backward):
        for scale in (1e-38, 1e-45, 2.0 ** -101, 2.0 ** 101, 3e38):
            assert call(lib, scale=scale, ws=None) == UNSUPPORTED, scale
    for scale in (2.0 ** -100, 1e-3, 1.0, 2.0 ** 100):
        assert _backward(lib, scale=scale, ws=None) == WORKSPACE, scale

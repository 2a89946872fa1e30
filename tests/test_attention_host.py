"""Host-side checks of attention's arguments (no GPU): what a call makes of them before anything is launched."""
import ctypes

import pytest

from test_block_host import _shape, lib  # noqa: F401


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

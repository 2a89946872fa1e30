"""Host-side checks of the operators around a block's linear layers (no GPU): what the entry points refuse, and that a refused
call says so before anything is launched."""
import ctypes

import pytest
import torch

import paper_2603_28845_amd as og
from paper_2603_28845_amd import binding

OK, INVALID, UNSUPPORTED, NOT_POSDEF, WORKSPACE, HIP = range(6)
P, NULL = 0x10000, None     # a non-null, aligned address that is never dereferenced on these paths


@pytest.fixture(scope="module")
def lib():
    return og.load_library()


def _shape(**kw):
    s = dict(dtype=1, n_heads=8, n_kv_heads=2, head_dim=64, n_seqs=2, causal=1, scale=0.125, total_q=100, total_k=100, max_q=60, max_k=60,
             cu_q=P, cu_k=P, len_k=None)
    s.update(kw)
    return binding.AttentionShape(**s)


def _heads(data=P, token=512, head=64):
    return ctypes.byref(binding.Heads(data, token, head))


BIG = ctypes.c_size_t(1 << 40)


def _forward(lib, shape=None, q=None, k=None, v=None, out=None, lse=P, ws=P, ws_bytes=BIG, **kw):
    s = _shape(**kw) if shape is None else shape
    return lib.onecomp_attention_forward(ctypes.byref(s), q or _heads(), k or _heads(), v or _heads(), out or _heads(), lse, ws, ws_bytes, NULL)


def _backward(lib, ws=P, ws_bytes=BIG, lse=P, views=None, **kw):
    h = views or [_heads() for _ in range(8)]
    return lib.onecomp_attention_backward(ctypes.byref(_shape(**kw)), *h[:4], lse, *h[4:], ws, ws_bytes, NULL)


@pytest.mark.parametrize("call", [_forward, _backward])
def test_attention_refusals(lib, call):
    assert call(lib, dtype=2) == UNSUPPORTED
    assert call(lib, head_dim=136) == UNSUPPORTED
    assert call(lib, head_dim=60) == UNSUPPORTED                   # 8 bf16 are 16 bytes
    assert call(lib, dtype=0, head_dim=62) == UNSUPPORTED
    assert call(lib, head_dim=0) == INVALID
    assert call(lib, n_heads=7) == INVALID                         # not a multiple of the key heads
    assert call(lib, n_kv_heads=0) == INVALID
    assert call(lib, n_heads=0) == INVALID
    assert call(lib, n_seqs=-1) == INVALID
    assert call(lib, total_q=-1) == INVALID
    assert call(lib, total_k=1 << 31) == INVALID
    assert call(lib, max_q=-1) == INVALID
    assert call(lib, cu_q=None) == INVALID
    assert call(lib, cu_k=None) == INVALID
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(lib, scale=scale) == INVALID


def test_attention_views(lib):
    for bad in (_heads(data=None), _heads(data=P + 8), _heads(token=60), _heads(token=516), _heads(head=68), _heads(token=1 << 23), _heads(head=-64)):
        for name in ("q", "k", "v", "out"):
            assert _forward(lib, **{name: bad}) == INVALID, name
        for i in range(8):
            views = [_heads() for _ in range(8)]
            views[i] = bad
            assert _backward(lib, views=views) == INVALID, i
    assert _backward(lib, lse=None) == INVALID
    assert lib.onecomp_attention_forward(None, _heads(), _heads(), _heads(), _heads(), P, P, BIG, NULL) == INVALID


def test_attention_workspaces(lib):
    few = dict(max_q=1, max_k=100000, total_q=2, total_k=200000)
    need = lib.onecomp_attention_workspace_bytes(ctypes.byref(_shape(**few)))
    assert need > 0
    assert _forward(lib, ws=None, **few) == WORKSPACE
    assert _forward(lib, ws_bytes=ctypes.c_size_t(need - 1), **few) == WORKSPACE
    assert _forward(lib, ws=P + 16, **few) == WORKSPACE
    assert lib.onecomp_attention_workspace_bytes(ctypes.byref(_shape(dtype=9))) == 0
    assert lib.onecomp_attention_backward_workspace_bytes(ctypes.byref(_shape())) >= 100 * 8 * 8
    assert _backward(lib, ws=None) == WORKSPACE
    assert _backward(lib, ws_bytes=ctypes.c_size_t(100)) == WORKSPACE
    assert _forward(lib, total_q=0, ws=None) == OK                 # nothing to do, nothing launched


def test_attention_binding_checks():
    q, k = torch.zeros(4, 2, 8), torch.zeros(4, 1, 8)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        og.onecomp_attention_forward(q, k, k, cu, cu, 4, 4)        # not on the GPU

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


def _norm_shape(**kw):
    s = dict(dtype=1, w_dtype=1, kind=0, gate_kind=0, post_norm=0, rows=10, width=64, residual_scale=1.0, eps=1e-6)
    s.update(kw)
    return binding.NormShape(**s)


def _rows(data=P, stride=64):
    return ctypes.byref(binding.Rows(data, stride))


Q = P + 0x10000     # another buffer


def _norm(lib, h=0, y=None, weight=P, bias=None, pw=None, pb=None, gate=None, h_out=None, n=0, **kw):
    """h, n: given unless None"""
    return lib.onecomp_block_norm_forward(ctypes.byref(_norm_shape(**kw)), _rows() if h == 0 else h, y, weight, bias, pw, pb, gate, h_out,
                                          _rows(Q) if n == 0 else n, NULL)


def test_norm_refusals(lib):
    assert _norm(lib, dtype=3) == UNSUPPORTED
    assert _norm(lib, w_dtype=3) == UNSUPPORTED
    assert _norm(lib, kind=2) == UNSUPPORTED
    assert _norm(lib, gate_kind=3) == UNSUPPORTED
    assert _norm(lib, width=32769) == UNSUPPORTED
    assert _norm(lib, width=0) == INVALID
    assert _norm(lib, rows=-1) == INVALID
    for eps in (-1.0, float("nan"), float("inf")):
        assert _norm(lib, eps=eps) == INVALID
    assert _norm(lib, residual_scale=float("nan")) == INVALID
    assert _norm(lib, h=None) == INVALID
    assert _norm(lib, h=_rows(None)) == INVALID
    assert _norm(lib, h=_rows(stride=63)) == INVALID                # rows overlap
    assert _norm(lib, h=_rows(P + 1)) == INVALID                    # not even an element's address
    assert _norm(lib, weight=P + 1) == INVALID
    assert _norm(lib, n=None) == INVALID                            # nothing to do
    assert _norm(lib, n=_rows(P)) == INVALID                        # n over h
    assert _norm(lib, h_out=_rows()) == INVALID                     # without y, h' is h
    assert _norm(lib, bias=P) == INVALID                            # rms norms have none
    assert _norm(lib, post_norm=1) == INVALID                       # without y
    assert _norm(lib, y=_rows(), pw=P) == INVALID                   # without post_norm
    assert _norm(lib, y=_rows(), gate_kind=1) == INVALID            # no gate
    assert _norm(lib, y=_rows(), gate=_rows()) == INVALID           # a gate that no kind announces
    assert _norm(lib, y=_rows(), gate_kind=2, gate=_rows(stride=3)) == INVALID
    assert _norm(lib, y=_rows(), h_out=_rows(Q)) == INVALID         # n over h'
    assert _norm(lib, rows=0) == OK


def _norm_back(lib, dn=0, dh_out=0, h=0, y=None, weight=P, pw=None, gate=None, out=0, ws=P, ws_bytes=BIG, grads=None, **kw):
    g = binding.NormGradients(*(grads or [ctypes.pointer(binding.Rows(P, 64)), None, None, P, None, None, None, None]))
    pick = lambda x: _rows() if x == 0 else x  # noqa: E731
    return lib.onecomp_block_norm_backward(ctypes.byref(_norm_shape(**kw)), pick(dn), pick(dh_out), pick(h), y, weight, pw, None, gate,
                                           ctypes.byref(g) if out == 0 else out, ws, ws_bytes, NULL)


def test_norm_gradient_refusals(lib):
    r = ctypes.pointer(binding.Rows(P, 64))
    assert _norm_back(lib, dtype=3) == UNSUPPORTED
    assert _norm_back(lib, h=None) == INVALID
    assert _norm_back(lib, dn=None, dh_out=None) == INVALID
    assert _norm_back(lib, out=None) == INVALID
    assert _norm_back(lib, dn=None) == INVALID                      # the weight's gradient without that of n
    assert _norm_back(lib, grads=[r, r, None, None, None, None, None, None]) == INVALID      # dy without y
    assert _norm_back(lib, grads=[r, None, r, None, None, None, None, None]) == INVALID      # a gate's without a gate
    assert _norm_back(lib, grads=[r, None, None, None, None, None, None, P]) == INVALID
    assert _norm_back(lib, grads=[r, None, None, None, P, None, None, None]) == INVALID      # a bias of an rms norm
    assert _norm_back(lib, grads=[r, None, None, None, None, P, None, None]) == INVALID      # no norm behind the block
    assert _norm_back(lib, ws=None) == WORKSPACE
    assert _norm_back(lib, ws_bytes=ctypes.c_size_t(64)) == WORKSPACE
    assert lib.onecomp_block_norm_workspace_bytes(ctypes.byref(_norm_shape())) >= 10 * 64 * 4
    assert lib.onecomp_block_norm_workspace_bytes(ctypes.byref(_norm_shape(width=0))) == 0


def test_clip_refusals(lib):
    def call(grad=P, out=P, numel=10, dtype=1, n=1, max_norm=1.0, norm=P, ws=P, ws_bytes=BIG, table=True):
        g = (binding.Gradient * 1)(binding.Gradient(grad, out, numel, dtype))
        return lib.onecomp_clip_gradients(g if table else None, n, max_norm, norm, ws, ws_bytes, NULL)

    assert call(dtype=2) == UNSUPPORTED
    assert call(grad=None) == INVALID
    assert call(out=None) == INVALID
    assert call(grad=P + 1) == INVALID
    assert call(dtype=0, out=P + 2) == INVALID
    assert call(numel=-1) == INVALID
    assert call(n=-1) == INVALID
    assert call(table=False) == INVALID
    assert call(max_norm=-1.0) == INVALID
    assert call(max_norm=float("nan")) == INVALID
    assert call(norm=P + 2) == INVALID
    assert call(ws=None) == WORKSPACE
    assert call(ws_bytes=ctypes.c_size_t(lib.onecomp_clip_workspace_bytes() - 1)) == WORKSPACE


def test_packed_structures():
    """The binding packs the structures by format: the same size and places as the header's."""
    assert binding._SHAPE.size == ctypes.sizeof(binding.AttentionShape) and binding._NORM_SHAPE.size == ctypes.sizeof(binding.NormShape)
    x = binding.AttentionShape.from_buffer_copy(binding._SHAPE.pack(1, 2, 3, 4, 5, 6, 0.5, 7, 8, 9, 10, 11, 12, 13))
    assert [getattr(x, f) for f, _ in x._fields_] == [1, 2, 3, 4, 5, 6, 0.5, 7, 8, 9, 10, 11, 12, 13]
    x = binding.NormShape.from_buffer_copy(binding._NORM_SHAPE.pack(1, 2, 3, 4, 5, 6, 7, 0.5, 0.25))
    assert [getattr(x, f) for f, _ in x._fields_] == [1, 2, 3, 4, 5, 6, 7, 0.5, 0.25]
    assert (ctypes.sizeof(binding.Heads), ctypes.sizeof(binding.Rows), ctypes.sizeof(binding.Gradient)) == (24, 16, 8 * binding._GRAD_FIELDS)


def test_structures_against_the_compiler(tmp_path):
    """Sizes and offsets of the header's structures as a C compiler lays them out."""
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    names = {"onecomp_heads": binding.Heads, "onecomp_attention_shape": binding.AttentionShape, "onecomp_rows": binding.Rows,
             "onecomp_norm_shape": binding.NormShape, "onecomp_norm_gradients": binding.NormGradients, "onecomp_gradient": binding.Gradient}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "onecomp.h"', "int main(void) {"]
    for name, cls in names.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "sizes.c"
    src.write_text("\n".join(lines + ["return 0;", "}"]).replace("\\\\", "\\"))
    import os
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run([gcc, "-I", inc, str(src), "-o", str(tmp_path / "sizes")], check=True)
    said = dict(l.split() for l in subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, cls in names.items():
        assert int(said[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(said[f"{name}.{f}"]) == getattr(cls, f).offset, f


def test_binding_checks():
    x = torch.zeros(4, 8)
    for call in (lambda: og.onecomp_block_norm_forward(x), lambda: og.onecomp_block_norm_backward(x, x, x), lambda: og.onecomp_clip_gradients([x], 1.0)):
        with pytest.raises(ValueError):
            call()                                                  # not on the GPU
    with pytest.raises(ValueError):
        og.onecomp_clip_gradients([x], 1.0, out=[])
    with pytest.raises(ValueError):
        og.onecomp_clip_gradients([], 1.0)

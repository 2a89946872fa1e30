"""The operators from tokens to the loss, on the host: what they refuse before anything is launched, workspace sizes, and the
structures that the Python binding packs."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2603_28845_amd as og
from paper_2603_28845_amd import binding

OK, INVALID, UNSUPPORTED, NOT_POSDEF, WORKSPACE, HIP = range(6)
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    return og.load_library()


def rows(data, stride):
    return ctypes.byref(binding.Rows(data, stride))


# addresses that nothing reads: every call below is refused, or has nothing to do
A, B, C, D = (0x10000 * i for i in range(1, 5))


def test_embedding_forward_refusals(lib):
    def call(tokens=A, n=8, dtype=1, table=(B, 64), vocab=100, width=64, scale=1.0, out=(C, 64)):
        return lib.onecomp_embedding_forward(tokens, n, dtype, rows(*table) if table else None, vocab, width, scale, rows(*out) if out else None, None)

    assert call(dtype=2) == UNSUPPORTED
    for bad in ({"tokens": None}, {"tokens": A + 2}, {"n": -1}, {"n": 1 << 24}, {"table": None}, {"out": None}, {"table": (0, 64)}, {"out": (0, 64)},
                {"vocab": 0}, {"vocab": (1 << 24) + 1}, {"width": 0}, {"table": (B, 63)}, {"out": (C, 63)}, {"table": (B + 1, 64)}, {"out": (C + 1, 64)},
                {"out": (B, 64)}, {"scale": float("nan")}, {"scale": float("inf")}, {"dtype": 0, "table": (B + 2, 64)}):
        assert call(**bad) == INVALID, bad
    assert call(n=0, tokens=None, out=(0, 64)) == OK


def test_embedding_backward_refusals(lib):
    def call(tokens=A, n=8, dtype=1, d_out=(B, 64), vocab=100, width=64, scale=1.0, base=None, d_table=(C, 64), ws=D, size=BIG):
        return lib.onecomp_embedding_backward(tokens, n, dtype, rows(*d_out) if d_out else None, vocab, width, scale, rows(*base) if base else None,
                                              rows(*d_table) if d_table else None, ws, size, None)

    assert call(dtype=-1) == UNSUPPORTED
    for bad in ({"tokens": None}, {"n": -1}, {"d_out": None}, {"d_table": None}, {"vocab": 0}, {"width": 0}, {"d_out": (B, 60)}, {"d_table": (C, 60)},
                {"d_table": (B, 64)}, {"base": (C, 65)}, {"base": (0, 64)}, {"base": (B + 1, 64)}, {"scale": float("nan")}):
        assert call(**bad) == INVALID, bad
    # more workgroups than a launch has: refused before anything is launched
    assert call(n=(1 << 24) - 1, width=1 << 23, d_out=(B, 1 << 23), d_table=(C, 1 << 23)) == UNSUPPORTED
    need = lib.onecomp_embedding_workspace_bytes(8, 100, 64)
    for bad in ({"ws": None}, {"ws": D + 16}, {"size": need - 1}):
        assert call(**bad) == WORKSPACE, bad
    assert lib.onecomp_embedding_workspace_bytes(-1, 100, 64) == 0 and lib.onecomp_embedding_workspace_bytes(8, 0, 64) == 0


def test_quantize_tokens_refusals(lib):
    def call(x=(A, 64), dtype=1, tokens=4, width=64, codes=B, scales=C, sums=D):
        return lib.onecomp_quantize_tokens(rows(*x) if x else None, dtype, tokens, width, codes, scales, sums, None)

    assert call(dtype=3) == UNSUPPORTED and call(width=72, x=(A, 72)) == UNSUPPORTED and call(width=65536, x=(A, 65536)) == UNSUPPORTED
    for bad in ({"x": None}, {"x": (0, 64)}, {"x": (A + 1, 64)}, {"x": (A, 63)}, {"tokens": -1}, {"width": 0}, {"codes": None}, {"codes": B + 8}, {"scales": None},
                {"scales": C + 2}, {"sums": None}, {"codes": A}, {"tokens": 1 << 24}, {"scales": D}):
        assert call(**bad) == INVALID, bad
    assert call(tokens=0, x=(0, 64), codes=None, scales=None, sums=None) == OK


def test_linear_refusals(lib):
    def call(codes=A, ts=B, sums=B, q=C, scales=B, zeros=B, bias=None, dtype=1, tokens=4, d_out=32, d_in=64, y=(D, 32)):
        return lib.onecomp_linear_int8(codes, ts, sums, q, scales, zeros, bias, dtype, tokens, d_out, d_in, rows(*y) if y else None, None)

    assert call(dtype=9) == UNSUPPORTED and call(d_in=72) == UNSUPPORTED and call(d_in=65536) == UNSUPPORTED
    assert call(tokens=1 << 20, d_out=1 << 16, y=(D, 1 << 16)) == UNSUPPORTED
    for bad in ({"codes": None}, {"ts": None}, {"sums": None}, {"q": None}, {"scales": None}, {"zeros": None}, {"codes": A + 8}, {"q": C + 8}, {"bias": B + 1},
                {"tokens": -1}, {"d_out": 0}, {"d_in": 0}, {"y": None}, {"y": (0, 32)}, {"y": (D, 31)}, {"y": (D + 1, 32)}, {"y": (A, 32)}, {"y": (C, 32)}):
        assert call(**bad) == INVALID, bad
    assert call(tokens=0, codes=None, ts=None, sums=None, y=(0, 32)) == OK


def loss_shape(dtype=1, tokens=10, width=64, vocab=1000, scale=1.0):
    return binding.LossShape(dtype, tokens, width, vocab, scale)


SHAPES = [({"dtype": 4}, UNSUPPORTED), ({"tokens": -1}, INVALID), ({"width": 0}, INVALID), ({"vocab": 0}, INVALID), ({"width": 60}, UNSUPPORTED),
          ({"width": 62, "dtype": 0}, UNSUPPORTED), ({"scale": 0.0}, INVALID), ({"scale": -1.0}, INVALID), ({"scale": float("nan")}, INVALID),
          ({"scale": float("inf")}, INVALID), ({"scale": 2.0 ** 101}, UNSUPPORTED), ({"scale": 2.0 ** -101}, UNSUPPORTED), ({"tokens": (1 << 20) + 1}, UNSUPPORTED),
          ({"vocab": (1 << 24) + 1}, UNSUPPORTED), ({"width": 1 << 22}, UNSUPPORTED),
          ({"tokens": 1 << 20, "vocab": 1 << 16}, UNSUPPORTED), ({"vocab": 1 << 20, "width": 1 << 16}, UNSUPPORTED)]


def test_loss_forward_refusals(lib):
    def call(h=(A, 64), w=(B, 64), targets=C, loss=D, lse=D + 64, ws=D, size=BIG, **kw):
        return lib.onecomp_token_loss_forward(ctypes.byref(loss_shape(**kw)), rows(*h) if h else None, rows(*w) if w else None, targets, loss, lse, ws, size, None)

    for kw, want in SHAPES:
        stride = max(64, kw.get("width", 64))
        assert call(h=(A, stride), w=(B, stride), **kw) == want, kw
        assert lib.onecomp_token_loss_workspace_bytes(ctypes.byref(loss_shape(**kw))) == 0
        assert lib.onecomp_token_loss_backward_workspace_bytes(ctypes.byref(loss_shape(**kw))) == 0
    assert lib.onecomp_token_loss_forward(None, None, None, None, None, None, None, 0, None) == INVALID
    for bad in ({"h": None}, {"w": None}, {"h": (0, 64)}, {"h": (A + 8, 64)}, {"h": (A, 68)}, {"h": (A, 56)}, {"w": (B + 2, 64)}, {"w": (B, 1 << 22)}, {"targets": None},
                {"targets": C + 2}, {"loss": D, "lse": D}, {"loss": None, "lse": None}, {"loss": D + 1}):
        assert call(**bad) == INVALID, bad
    need = lib.onecomp_token_loss_workspace_bytes(ctypes.byref(loss_shape()))
    for bad in ({"ws": None}, {"ws": D + 8}, {"size": need - 1}):
        assert call(**bad) == WORKSPACE, bad
    assert call(tokens=0, h=(0, 64), targets=None, loss=None, lse=None) == OK


def test_loss_backward_refusals(lib):
    def call(d_loss=C, d_lse=None, h=(A, 64), w=(B, 64), targets=C, lse=C, dh=(D, 64), dw=(2 * D, 64), ws=D, size=BIG, **kw):
        return lib.onecomp_token_loss_backward(ctypes.byref(loss_shape(**kw)), d_loss, d_lse, rows(*h), rows(*w), targets, lse, rows(*dh) if dh else None,
                                               rows(*dw) if dw else None, ws, size, None)

    for kw, want in SHAPES:
        stride = max(64, kw.get("width", 64))
        assert call(h=(A, stride), w=(B, stride), dh=(D, stride), dw=(2 * D, stride), **kw) == want, kw
    for bad in ({"d_loss": None}, {"lse": None}, {"targets": None}, {"d_lse": C + 1}, {"dh": None, "dw": None}, {"dh": (A, 64)}, {"dh": (B, 64)}, {"dw": (A, 64)},
                {"dw": (B, 64)}, {"dw": (D, 64)}, {"dh": (D + 8, 64)}, {"dw": (2 * D, 60)}, {"dh": (0, 64)}):
        assert call(**bad) == INVALID, bad
    need = lib.onecomp_token_loss_backward_workspace_bytes(ctypes.byref(loss_shape()))
    for bad in ({"ws": None}, {"ws": D + 8}, {"size": need - 1}):
        assert call(**bad) == WORKSPACE, bad


def test_workspaces_do_not_hold_logits(lib):
    one = ctypes.byref(loss_shape(tokens=65536, width=4096, vocab=128000))
    assert lib.onecomp_token_loss_workspace_bytes(one) < 65536 * 4096 * 2 + 65536 * 128000 // 8
    assert lib.onecomp_token_loss_backward_workspace_bytes(one) < 65536 * 4096 * 6 + (1100 << 20)


def test_tensors_on_the_host_and_wrong_shapes_are_refused():
    tokens, x = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 64)
    codes = torch.zeros(4, 64, dtype=torch.int8)
    for call in (lambda: og.onecomp_embedding_forward(tokens, x), lambda: og.onecomp_embedding_backward(tokens, x, 10), lambda: og.onecomp_quantize_tokens(x),
                 lambda: og.onecomp_linear_int8(codes, x, x, x, x, x), lambda: og.onecomp_token_loss_forward(x, x, tokens),
                 lambda: og.onecomp_token_loss_backward(x, x, x, tokens, x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        og.onecomp_linear_int8(codes, x, x, x, x, x, dtype=torch.float16)


def test_packed_structure_is_the_headers(tmp_path):
    assert binding._LOSS_SHAPE.size == ctypes.sizeof(binding.LossShape)
    x = binding.LossShape.from_buffer_copy(binding._LOSS_SHAPE.pack(1, 2, 3, 4, 0.5))
    assert (x.dtype, x.tokens, x.width, x.vocab, x.scale) == (1, 2, 3, 4, 0.5)
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    fields = [f for f, _ in binding.LossShape._fields_]
    source = '#include <stdio.h>\n#include <stddef.h>\n#include "onecomp.h"\nint main(void) {\n printf("%zu", sizeof(onecomp_loss_shape));\n'
    source += "".join(f' printf(" %zu", offsetof(onecomp_loss_shape, {f}));\n' for f in fields) + " return 0;\n}\n"
    (tmp_path / "sizes.c").write_text(source)
    subprocess.run([gcc, "-I", os.path.join(ROOT, "include"), str(tmp_path / "sizes.c"), "-o", str(tmp_path / "sizes")], check=True)
    said = [int(v) for v in subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()]
    assert said == [ctypes.sizeof(binding.LossShape)] + [getattr(binding.LossShape, f).offset for f in fields]


def test_tiles_sharing_and_workspaces(tmp_path):
    """csrc/token_plan.hpp is plain host logic: tests/token_plan_check.cpp runs it over sizes."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    here, exe = os.path.dirname(os.path.abspath(__file__)), tmp_path / "token_plan_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", os.path.join(here, "token_plan_check.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.split()[0] == "ok", r.stdout + r.stderr

"""Host-side checks of the norms' arguments (no GPU): results that cannot be written over what they are given for."""
import ctypes

from test_block_host import BIG, INVALID, NULL, P, Q, WORKSPACE, _norm, _norm_shape, _rows, lib  # noqa: F401
from paper_2603_28845_amd import binding


def _pointer(data, stride=64):
    return ctypes.pointer(binding.Rows(data, stride))


def test_forward_over_rows_of_another_stride(lib):  # noqa: F811
    R = Q + 0x10000
    assert _norm(lib, y=_rows(R), h_out=_rows(P, 128)) == INVALID               # over h
    assert _norm(lib, y=_rows(R), h_out=_rows(R, 128)) == INVALID               # over y
    assert _norm(lib, y=_rows(R), n=_rows(R, 128)) == INVALID
    assert _norm(lib, y=_rows(R), gate_kind=2, gate=_rows(R + 0x10000), h_out=_rows(R + 0x10000, 128)) == INVALID
    assert _norm(lib, rows=0, y=_rows(R), h_out=_rows(P, 128)) == 0


def test_gradients_over_rows_of_another_stride(lib):  # noqa: F811
    def call(dh=None, dy=None, dgate=None, ws=P):
        shape = _norm_shape(gate_kind=2)
        inputs = [_pointer(P * (i + 1)) for i in range(5)]                      # dn, dh_out, h, y, gate
        g = binding.NormGradients(dh, dy, dgate, P * 9, None, None, None, None)
        return lib.onecomp_block_norm_backward(ctypes.byref(shape), *inputs[:4], P, None, None, inputs[4], ctypes.byref(g), ws, BIG, NULL)

    for i in range(5):
        for name in ("dh", "dy", "dgate"):
            assert call(**{name: _pointer(P * (i + 1), 128)}) == INVALID, (name, i)
    for pair in (("dh", "dy"), ("dh", "dgate"), ("dy", "dgate")):
        assert call(**{name: _pointer(P * 7) for name in pair}) == INVALID, pair
    assert call(dh=_pointer(P * 6), dy=_pointer(P * 7), ws=None) == WORKSPACE

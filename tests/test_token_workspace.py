"""Workspaces of the loss and its gradients against what include/onecomp.h says they hold, and the errors it names for sizes."""
import ctypes

import pytest

import paper_2603_28845_amd as og
from paper_2603_28845_amd import binding

GB, INVALID, UNSUPPORTED = 1 << 30, 1, 2
SIZES = [(1, 8, 1), (16, 4096, 128000), (700, 1024, 4000), (4096, 4096, 128000), (8192, 4096, 128000), (16384, 512, 50000), (65536, 1024, 32000), (1 << 20, 256, 2048)]


@pytest.fixture(scope="module")
def lib():
    return og.load_library()


@pytest.mark.parametrize("dtype,esz", [(1, 2), (0, 4)])
@pytest.mark.parametrize("n,width,vocab", SIZES)
def test_sizes(lib, dtype, esz, n, width, vocab):
    shape = ctypes.byref(binding.LossShape(dtype, n, width, vocab, 1.0))
    rows = n * (-(-width * esz // 64) * 64)
    small = 64 * n + 4096                                          # some words a token, and whole 256 bytes
    assert lib.onecomp_token_loss_workspace_bytes(shape) <= rows + 8 * n * (vocab // 32 + 1) + small
    g = min(max(GB, 2048 * n * esz), n * (-(-vocab // 256) * 256) * esz + 256 * n * esz)
    sums = max(min(GB, 16 * n * width * 4), n * width * 4)
    bytes_ = lib.onecomp_token_loss_backward_workspace_bytes(shape)
    assert n * width * (4 + esz) <= bytes_ <= rows + g + sums + small


def test_errors_of_sizes(lib):
    row, far = ctypes.byref(binding.Rows(0x10000, 1 << 25)), ctypes.byref(binding.Rows(0x20000, 1 << 25))
    most = 1 << 24
    for n, vocab, width in ((most, 8, 8), (8, most + 1, 8), (8, 8, most + 1)):
        assert lib.onecomp_embedding_forward(0x30000, n, 1, row, vocab, width, 1.0, far, None) == INVALID
        assert lib.onecomp_embedding_backward(0x30000, n, 1, row, vocab, width, 1.0, None, far, 0x40000, 1 << 60, None) == INVALID
    assert lib.onecomp_quantize_tokens(row, 1, most, 16, 0x30000, 0x40000, 0x50000, None) == INVALID
    for n, d_out in ((most, 8), (8, most + 1)):
        assert lib.onecomp_linear_int8(0x30000, 0x30000, 0x30000, 0x30000, 0x30000, 0x30000, None, 1, n, d_out, 16, far, None) == INVALID
    for n, width, vocab in (((1 << 20) + 1, 8, 8), (8, 1 << 24, 8), (8, 8, most + 1)):
        shape = ctypes.byref(binding.LossShape(1, n, width, vocab, 1.0))
        assert lib.onecomp_token_loss_forward(shape, row, far, 0x30000, 0x40000, 0x50000, 0x60000, 1 << 60, None) == UNSUPPORTED

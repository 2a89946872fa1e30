"""Tokens of any 32 bits in the gradient of the embedding table: which row they belong to, on the host, and the gradient itself."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2603_28845_amd as og
from token_oracle import embedding_grad

HERE = os.path.dirname(os.path.abspath(__file__))


def test_rows_of_tokens(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no C++ compiler")
    exe = tmp_path / "token_rows_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(HERE, "token_rows_check.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.split()[0] == "ok", r.stdout + r.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("n", [40, 700, 17000])
@pytest.mark.parametrize("vocab", [1, 65, 777, 70000])
def test_tokens_outside_have_no_part(n, vocab):
    dev = "cuda:0"
    gen = torch.Generator(device=dev).manual_seed(n)
    marks = torch.tensor([-2 ** 31, -2 ** 31 + 1, -100, -1, vocab, vocab + 63, 2 ** 31 - 1], dtype=torch.int32, device=dev)
    tokens = torch.randint(0, vocab, (n,), generator=gen, device=dev, dtype=torch.int32)
    out = torch.rand(n, generator=gen, device=dev) < 0.5
    tokens[out] = marks[torch.randint(0, len(marks), (int(out.sum()),), generator=gen, device=dev)]
    d_out = torch.randn(n, 24, generator=gen, device=dev)
    d_out[out] = float("nan")
    want, off = embedding_grad(tokens, d_out, vocab, 0.5)
    got = og.onecomp_embedding_backward(tokens, d_out, vocab, scale=0.5)
    assert bool(((got.double() - want).abs() <= off).all())

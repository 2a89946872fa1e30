"""Attention of many sequences: a workgroup's is searched for, not counted."""
import pytest
import torch

import paper_2603_28845_amd as og
from test_gpu_attention import BF16, F32, _check, _inputs, _starts
from test_gpu_attention_not_finite import _time

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [63, 65, 255, 256, 700])
def test_numbers_of_sequences(n, dtype):
    """Around a wave's lanes and beyond; empty ones, one of several tiles and room behind the keys among them."""
    print(f"[case] {n} {dtype}", flush=True)
    nq = [(5 * i) % 19 for i in range(n)]
    nq[n // 3], nq[n - 1] = 300, 0
    nk = [a + (i % 4) * 30 for i, a in enumerate(nq)]
    room = [b + i % 3 for i, b in enumerate(nk)]
    _check(_inputs(nq, nk, 2, 1, 32, dtype, 40), nq, nk, True, True)
    _check(_inputs(nq, nk, 2, 1, 32, dtype, 41, room=room), nq, nk, False, True)
    # single tokens, one of them on a long cache
    ones = [1] * n
    nk[n // 2] = 3000
    _check(_inputs(ones, nk, 6, 2, 32, dtype, 42), ones, nk, True, False)


@pytest.mark.parametrize("n", [1023, 1024, 1100])
def test_many_single_tokens(n):
    nk = [(7 * i) % 200 for i in range(n)]
    nk[n // 2], nk[5] = 4000, 0
    ones = [1] * n
    _check(_inputs(ones, nk, 3, 1, 32, BF16, 45), ones, nk, True, False)


@pytest.mark.parametrize("n", [63, 100, 300, 1200])
def test_padding_rows(n):
    nq = [3] * n
    x = _inputs(nq + [200], nq + [200], 2, 1, 32, BF16, 43)
    x["cu_q"] = x["cu_k"] = _starts(nq)
    out, lse = og.onecomp_attention_forward(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], 3, 3)
    assert bool((out[3 * n:] == 0).all()) and bool((lse[:, 3 * n:] == -float("inf")).all()) and bool(torch.isfinite(lse[:, :3 * n]).all())
    dq, dk, dv = og.onecomp_attention_backward(x["d_out"], x["q"], x["k"], x["v"], out, lse, x["cu_q"], x["cu_k"], 3, 3)
    assert all(bool((t[3 * n:] == 0).all()) and bool((t[:3 * n] != 0).any()) for t in (dq, dk, dv))


def test_time_of_many_sequences():
    """Eight times the sequences of the same lengths are eight times the work: 16 leaves twice that; a workgroup that reads all
    sequences before its own takes 64 times as long in all."""
    times = {}
    for n in (4096, 32768):
        nq = [(3 * i) % 16 for i in range(n)]
        tokens, longest = sum(nq), 15
        x = _inputs(nq, nq, 4, 2, 32, BF16, 44)
        out, lse = og.onecomp_attention_forward(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], longest, longest)
        one, cache = _starts([1] * n), x["cu_k"]
        q = x["q"].new_ones((n, 4, 32))
        times[n] = [_time(call, 2) for call in (
            lambda: og.onecomp_attention_forward(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], longest, longest),
            lambda: og.onecomp_attention_backward(x["d_out"], x["q"], x["k"], x["v"], out, lse, x["cu_q"], x["cu_k"], longest, longest),
            lambda: og.onecomp_attention_forward(q, x["k"], x["v"], one, cache, 1, longest))]
        print(f"[time] {n} sequences, {tokens} tokens: " + " ".join(f"{t:.3f}" for t in times[n]) + " ms", flush=True)
    for few, many in zip(times[4096], times[32768]):
        assert many <= 16 * few

"""Attention of packed sequences on the GPU against 64 bits: lengths from none to long, head layouts, strides, caches with
room behind their keys, queries that see nothing, and what must not be seen."""
import math

import pytest
import torch

import paper_2603_28845_amd as og
from attention_oracle import attention, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _starts(lengths):
    return torch.tensor([0] + torch.tensor(lengths, dtype=torch.int64).cumsum(0).tolist(), dtype=torch.int32, device=DEV)


def _inputs(nq, nk, heads, kv_heads, dim, dtype, seed, room=None, layout="packed", std=1.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(tokens, h):
        if layout == "head_first":       # [heads, tokens, dim] in memory
            return torch.randn(h, tokens, dim, generator=gen, device=DEV).mul_(std).to(dtype).transpose(0, 1)
        if layout == "padded":           # rows of a wider buffer, with NaN in between
            t = torch.full((tokens, h, dim + 8), math.nan, device=DEV, dtype=dtype)
            t[..., :dim] = torch.randn(tokens, h, dim, generator=gen, device=DEV).mul_(std)
            return t[..., :dim]
        return torch.randn(tokens, h, dim, generator=gen, device=DEV).mul_(std).to(dtype)

    tq, tk = sum(nq), sum(room or nk)
    x = {"q": normal(tq, heads), "k": normal(tk, kv_heads), "v": normal(tk, kv_heads), "d_out": normal(tq, heads)}
    if room:
        x["len_k"] = torch.tensor(nk, dtype=torch.int32, device=DEV)
        at = _starts(room).tolist()
        for i, n in enumerate(nk):       # what lies behind a sequence's keys must not matter
            x["k"][at[i] + n:at[i + 1]] = math.nan
            x["v"][at[i] + n:at[i + 1]] = math.inf
    x.update(cu_q=_starts(nq), cu_k=_starts(room or nk))
    return x


def _forward(x, nq, nk, causal, **kw):
    return og.onecomp_attention_forward(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], max(nq), max(nk), causal=causal, len_k=x.get("len_k"), **kw)


def _check(x, nq, nk, causal, grad, scale=None):
    scale = x["q"].shape[2] ** -0.5 if scale is None else scale
    out, lse = _forward(x, nq, nk, causal, scale=scale)
    want = attention(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], causal, scale, x.get("len_k"), x["d_out"] if grad else None)
    check(out, want["out"], "out")
    check(lse, want["lse"], "lse")
    if not grad:
        return
    got = og.onecomp_attention_backward(x["d_out"], x["q"], x["k"], x["v"], out, lse, x["cu_q"], x["cu_k"], max(nq), max(nk), causal=causal,
                                        scale=scale, len_k=x.get("len_k"))
    for name, t in zip(("dq", "dk", "dv"), got):
        check(t, want[name], name)
    again = og.onecomp_attention_backward(x["d_out"], x["q"], x["k"], x["v"], out, lse, x["cu_q"], x["cu_k"], max(nq), max(nk), causal=causal,
                                          scale=scale, len_k=x.get("len_k"))
    assert all(torch.equal(a, b) for a, b in zip(got, again))


# lengths: one token, around the sizes of tiles, none at all, more queries than keys, chunks behind a cache, single tokens
LENGTHS = {
    "one": ([1], [1]),
    "edges": ([31, 32, 33, 63, 64, 65], [31, 32, 33, 63, 64, 65]),
    "none": ([0, 5, 0, 7, 3], [0, 5, 9, 0, 3]),
    "more_queries": ([100, 40, 300], [20, 39, 257]),
    "chunk": ([17, 1, 260], [530, 64, 300]),
    "long": ([513, 1030], [513, 1030]),
    "tokens": ([1, 1, 1, 1], [1, 700, 2049, 64]),
    "few": ([2, 3, 5], [900, 3, 1500]),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", LENGTHS)
def test_lengths(name, dtype, causal):
    nq, nk = LENGTHS[name]
    print(f"[case] {name} {dtype} causal={causal}", flush=True)
    _check(_inputs(nq, nk, 4, 2, 64, dtype, 1), nq, nk, causal, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 8), (3, 1, 32), (5, 5, 40), (8, 2, 80), (6, 3, 96), (16, 2, 128), (32, 8, 128), (9, 1, 120), (70, 2, 64)])
def test_heads_and_dims(heads, kv_heads, dim, dtype):
    print(f"[case] {heads} {kv_heads} {dim} {dtype}", flush=True)
    for nq, nk in (([70, 3, 129], [70, 3, 129]), ([1, 1], [333, 20])):
        _check(_inputs(nq, nk, heads, kv_heads, dim, dtype, 2), nq, nk, True, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", ["head_first", "padded"])
def test_layouts(layout, dtype):
    for nq, nk in (([70, 3, 129], [70, 3, 129]), ([1, 2], [333, 20])):
        _check(_inputs(nq, nk, 6, 2, 64, dtype, 3, layout=layout), nq, nk, True, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq", [[1, 1, 1, 1], [40, 1, 7, 130]])
def test_room_behind_the_keys(nq, dtype):
    nk, room = [100, 1, 65, 300], [164, 3, 65, 1000]
    x = _inputs(nq, nk, 4, 2, 64, dtype, 4, room=room)
    _check(x, nq, nk, True, True)
    _check(x, nq, nk, False, True)


def test_strides_of_outputs_and_padding_rows():
    """Results into slices of wider buffers; rows behind the last sequence are set to nothing."""
    nq = [50, 77]
    x = _inputs([50, 77, 30], [50, 77, 30], 4, 2, 64, BF16, 5)
    x["q"][127:], x["k"][127:], x["v"][127:], x["d_out"][127:] = math.nan, math.nan, math.inf, math.nan
    x["cu_q"] = x["cu_k"] = _starts(nq)
    qkv = torch.full((157, 8, 64), 3.0, dtype=BF16, device=DEV)
    wide = torch.full((157, 4, 72), 3.0, dtype=BF16, device=DEV)
    lse = torch.full((4, 157), 3.0, device=DEV)
    og.onecomp_attention_forward(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], 77, 77, out=wide[..., :64], lse=lse)
    og.onecomp_attention_backward(x["d_out"], x["q"], x["k"], x["v"], wide[..., :64], lse, x["cu_q"], x["cu_k"], 77, 77,
                                  dq=qkv[:, :4], dk=qkv[:, 4:6], dv=qkv[:, 6:])
    want = attention(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], True, 0.125, None, x["d_out"])
    check(wide[..., :64], want["out"], "out")
    check(lse, want["lse"], "lse")
    for name, t in (("dq", qkv[:, :4]), ("dk", qkv[:, 4:6]), ("dv", qkv[:, 6:])):
        check(t, want[name], name)
    assert bool((wide[..., 64:] == 3.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores(dtype):
    """Scores of hundreds: the maximum moves from tile to tile and most probabilities vanish."""
    nq = nk = [300, 65]
    x = _inputs(nq, nk, 2, 1, 64, dtype, 6, std=5.0)
    x["k"][200] *= 8
    _check(x, nq, nk, True, True, scale=0.5)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_unseen_keys_may_hold_anything(dtype):
    """NaN and infinities in keys and values that a query does not see: later tokens of its own prompt, other sequences."""
    nq = nk = [150, 90]
    x = _inputs(nq, nk, 4, 2, 64, dtype, 7)
    want = attention(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], True, 0.125, None, x["d_out"])
    clean, clean_lse = _forward(x, nq, nk, True)
    dirty = {n: x[n].clone() for n in ("k", "v")}
    for name in ("k", "v"):
        dirty[name][100], dirty[name][140] = math.nan, math.inf
    out, lse = _forward(dict(x, **dirty), nq, nk, True)
    for rows in (slice(0, 100), slice(150, 240)):
        check(out[rows], [t[rows] for t in want["out"]], "out")
        check(lse[:, rows], [t[:, rows] for t in want["lse"]], "lse")
    assert bool(torch.isnan(out[100:150].float()).all())
    # values alone: the scores are fine, and infinity stays infinity where it is seen
    dirty = dict(x, v=x["v"].clone())
    dirty["v"][100, :, 3] = math.inf
    out, lse = _forward(dirty, nq, nk, True)
    check(lse, want["lse"], "lse")
    assert bool((out[100:150, :, 3] == math.inf).all())
    out[100:150, :, 3] = clean[100:150, :, 3]
    check(out, want["out"], "out")
    # keys that a query does not see, in its gradient
    args = (x["cu_q"], x["cu_k"], 150, 150)
    dirty = x["k"].clone()
    dirty[100] = math.nan
    dq = og.onecomp_attention_backward(x["d_out"], x["q"], dirty, x["v"], clean, clean_lse, *args)[0]
    for rows in (slice(0, 100), slice(150, 240)):
        check(dq[rows], [t[rows] for t in want["dq"]], "dq")
    assert bool(torch.isnan(dq[100:150].float()).all())
    # a token's d_out that is no number reaches its own dq and the keys that it sees
    d = x["d_out"].clone()
    d[20] = math.nan
    dq, dk, dv = og.onecomp_attention_backward(d, x["q"], x["k"], x["v"], clean, clean_lse, *args)
    for rows in (slice(0, 20), slice(21, 240)):
        check(dq[rows], [t[rows] for t in want["dq"]], "dq")
    for got, name in ((dk, "dk"), (dv, "dv")):
        check(got[21:], [t[21:] for t in want[name]], name)
        assert bool(torch.isnan(got[:21].float()).all())
    assert bool(torch.isnan(dq[20].float()).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_unseen_keys_of_a_few_rows(dtype):
    """The same where the keys are split: tokens of a chunk that come after the query."""
    nq, nk = [4, 3], [1000, 600]
    x = _inputs(nq, nk, 4, 2, 64, dtype, 14)
    want = attention(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], True, 0.125)
    x["k"][998], x["v"][998:1000], x["v"][1599] = math.nan, math.nan, math.inf
    out, lse = _forward(x, nq, nk, True)
    for rows in (slice(0, 2), slice(4, 6)):
        check(out[rows], [t[rows] for t in want["out"]], "out")
        check(lse[:, rows], [t[:, rows] for t in want["lse"]], "lse")
    assert bool(torch.isnan(out[2:4].float()).all()) and not bool(torch.isfinite(out[6].float()).any())


def test_gradients_against_differences():
    """fp32: the gradients of a random functional against central differences of the forward call."""
    nq, nk = [5, 20], [9, 20]
    x = _inputs(nq, nk, 2, 1, 16, F32, 8)
    out, lse = _forward(x, nq, nk, True)
    grads = og.onecomp_attention_backward(x["d_out"], x["q"], x["k"], x["v"], out, lse, x["cu_q"], x["cu_k"], 20, 20)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    for name, g in zip(("q", "k", "v"), grads):
        step = torch.randn(g.shape, generator=gen, device=DEV)
        eps, value = 1e-2, {}
        for sign in (1, -1):
            moved = dict(x, **{name: x[name] + sign * eps * step})
            value[sign] = float((_forward(moved, nq, nk, True)[0].double() * x["d_out"].double()).sum())
        slope, want = (value[1] - value[-1]) / (2 * eps), float((g.double() * step.double()).sum())
        # fp32 values of size up to 100 over 2e-2, and the third derivative's eps^2
        assert abs(slope - want) <= 2e-2 + 2e-3 * float((g.double() * step.double()).norm())


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB between a sequence's first and last key, whole and behind another sequence's."""
    tokens = 600_000
    wide = torch.zeros((tokens, 1, 4096), dtype=BF16, device=DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(10)
    wide[..., :128] = torch.randn(tokens, 1, 128, generator=gen, device=DEV)
    k, v = wide[..., :64], wide[..., 64:128]
    for nk in ([tokens], [tokens - 100, 100]):
        q = torch.randn(3 * len(nk), 4, 64, generator=gen, device=DEV).to(BF16)
        cu_q, cu_k = _starts([3] * len(nk)), _starts(nk)
        for max_q in (3, 300):           # both launch shapes
            out, lse = og.onecomp_attention_forward(q, k, v, cu_q, cu_k, max_q, tokens)
            want = attention(q, k, v, cu_q, cu_k, True, 0.125)
            check(out, want["out"], "out")
            check(lse, want["lse"], "lse")
    d = torch.randn(q.shape, generator=gen, device=DEV).to(BF16)
    got = og.onecomp_attention_backward(d, q, k, v, out, lse, cu_q, cu_k, 3, tokens)
    want = attention(q, k, v, cu_q, cu_k, True, 0.125, None, d)
    for name, t in zip(("dq", "dk", "dv"), got):
        check(t, want[name], name)


def test_another_stream_and_a_workspace_at_hand():
    nq, nk = [1, 1, 40], [3000, 17, 40]
    x = _inputs(nq, nk, 8, 2, 128, BF16, 11)
    want, want_lse = _forward(x, nq, nk, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.full((1 << 26,), 255, dtype=torch.uint8, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = _forward(x, nq, nk, True, workspace=ws)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_empty_calls():
    q, k = torch.zeros((0, 4, 64), dtype=BF16, device=DEV), torch.ones((5, 2, 64), dtype=BF16, device=DEV)
    cu_q, cu_k = _starts([0]), _starts([5])
    out, lse = og.onecomp_attention_forward(q, k, k, cu_q, cu_k, 0, 5)
    assert out.shape == (0, 4, 64)
    dq, dk, dv = og.onecomp_attention_backward(q, q, k, k, out, lse, cu_q, cu_k, 0, 5)
    assert bool((dk == 0).all()) and bool((dv == 0).all())
    q = torch.ones((3, 4, 64), dtype=BF16, device=DEV)
    out, lse = og.onecomp_attention_forward(q, k[:0], k[:0], _starts([3]), _starts([0]), 3, 0)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv = og.onecomp_attention_backward(q, q, k[:0], k[:0], out, lse, _starts([3]), _starts([0]), 3, 0)
    assert bool((dq == 0).all()) and dk.shape == (0, 2, 64)


def test_sequences_by_the_hundred():
    """More sequences than a wave has lanes."""
    nq = [(7 * i) % 23 for i in range(150)]
    nk = [n + (i % 5) * 40 for i, n in enumerate(nq)]
    x = _inputs(nq, nk, 4, 4, 32, BF16, 12)
    _check(x, nq, nk, True, True)
    ones = [1] * 150
    _check(_inputs(ones, nk, 4, 4, 32, BF16, 13), ones, nk, True, False)

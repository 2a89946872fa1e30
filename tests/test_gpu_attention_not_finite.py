"""Attention whose inputs hold infinities and NaN here and there: what they must not reach is as without them, what they reach is
not finite, and a call takes a few times as long at most."""
import math

import pytest
import torch

import paper_2603_28845_amd as og
from attention_oracle import attention, check
from test_gpu_attention import BF16, F32, _forward, _inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# queries and keys of each sequence: prompts, chunks behind a cache, more than one share of keys and of queries, a few rows
LENGTHS = [([150, 90], [150, 90]), ([70, 33, 129], [300, 64, 200]), ([1100], [1100]), ([4, 3], [1000, 600]), ([2, 40], [2, 2500])]
SHAPES = [(4, 2, 64), (3, 1, 32), (2, 2, 80), (4, 1, 128)]


def _where(x, nq, nk):
    """Sequence of each query, the first key that it does not see (both counted over all rows), and the first key it may see."""
    first, end, at_k = [], [], 0
    for a, b in zip(nq, nk):
        first += [at_k] * a
        end += [at_k + max(0, i + b - a + 1) for i in range(a)]
        at_k += b
    return torch.tensor(first, device=DEV), torch.tensor(end, device=DEV)


def _sees(x, nq, nk, key):
    first, end = _where(x, nq, nk)
    return (key >= first) & (key < end)


@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nk", LENGTHS)
def test_values(nq, nk, dtype, heads, kv_heads, dim):
    print(f"[case] {nq} {nk} {dtype} {heads} {kv_heads} {dim}", flush=True)
    x = _inputs(nq, nk, heads, kv_heads, dim, dtype, 30)
    gen = torch.Generator()
    gen.manual_seed(sum(nk) + dim)
    group, total = heads // kv_heads, sum(nk)
    marks = []
    for kind in (math.nan, math.inf, -math.inf) * 3:
        # the last rows of a sequence, where some of its queries do not see them, or any
        at = total - 1 - int(torch.randint(0, min(total, 40), (1,), generator=gen)) if len(marks) % 2 else int(torch.randint(0, total, (1,), generator=gen))
        marks.append((at, int(torch.randint(0, kv_heads, (1,), generator=gen)), int(torch.randint(0, dim, (1,), generator=gen)), kind))
    clean = x["v"].clone()
    for at, g, c, kind in marks:
        x["v"][at, g, c] = kind
        clean[at, g, c] = 0
    out, lse = _forward(x, nq, nk, True)
    value, bound = attention(x["q"], x["k"], clean, x["cu_q"], x["cu_k"], True, dim ** -0.5)["out"]
    for at, g, c, _ in marks:
        kind = float(x["v"][at, g, c])                             # the last of marks that fell on the same entry
        value[_sees(x, nq, nk, at), g * group:(g + 1) * group, c] += kind
    broken = torch.isnan(value)
    assert torch.equal(torch.isnan(out), broken)
    check(torch.where(broken, 0.0, out.double()), [torch.where(broken, 0.0, value), bound], "out")
    check(lse, attention(x["q"], x["k"], clean, x["cu_q"], x["cu_k"], True, dim ** -0.5)["lse"], "lse")


def _gradients(x, nq, nk, out, lse, **dirty):
    y = dict(x, **dirty)
    return og.onecomp_attention_backward(y["d_out"], y["q"], y["k"], y["v"], out, lse, x["cu_q"], x["cu_k"], max(nq), max(nk))


def _same(got, want, rows, name):
    check(got[rows], [t[rows] for t in want[name]], name)


def _none_finite(t):
    return not bool(torch.isfinite(t.float()).any())


@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nk", LENGTHS)
def test_gradients(nq, nk, dtype, heads, kv_heads, dim):
    print(f"[case] {nq} {nk} {dtype} {heads} {kv_heads} {dim}", flush=True)
    x = _inputs(nq, nk, heads, kv_heads, dim, dtype, 31)
    out, lse = _forward(x, nq, nk, True)
    want = attention(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], True, dim ** -0.5, None, x["d_out"])
    first, end = _where(x, nq, nk)
    keys, everything = torch.arange(sum(nk), device=DEV), torch.ones(sum(nk), dtype=torch.bool, device=DEV)
    for query in (0, nq[0] // 2, sum(nq) - 1):
        seen = (keys >= first[query]) & (keys < end[query])
        others = torch.arange(sum(nq), device=DEV) != query
        # one entry of d_out: a column of dv, and dk, of the keys that its query sees
        d = x["d_out"].clone()
        d[query, 0, 5] = math.inf
        dq, dk, dv = _gradients(x, nq, nk, out, lse, d_out=d)
        _same(dq, want, others, "dq")
        _same(dk, want, ~seen, "dk")
        _same(dv, want, ~seen, "dv")
        column = torch.zeros_like(dv, dtype=torch.bool)
        column[seen, 0, 5] = True
        check(torch.where(column, 0.0, dv.double()), [torch.where(column, 0.0, want["dv"][0]), want["dv"][1]], "dv")
        assert _none_finite(dv[column]) and _none_finite(dk[seen][:, 0]) and _none_finite(dq[query, 0])
        # a query
        q = x["q"].clone()
        q[query] = math.nan
        dq, dk, dv = _gradients(x, nq, nk, out, lse, q=q)
        _same(dq, want, others, "dq")
        _same(dk, want, ~seen, "dk")
        _same(dv, want, ~seen, "dv")
        assert _none_finite(dk[seen]) and _none_finite(dv[seen]) and _none_finite(dq[query])
    for key in (0, nk[0] // 2, nk[0] - 1, sum(nk) - 1):
        sees = _sees(x, nq, nk, key)
        # a key, then a value: the dq of the queries that see it
        for name in ("k", "v"):
            dirty = x[name].clone()
            dirty[key, 0, 7] = math.nan
            dq, dk, dv = _gradients(x, nq, nk, out, lse, **{name: dirty})
            _same(dq, want, ~sees, "dq")
            group = slice(0, heads // kv_heads)
            assert _none_finite(dq[sees][:, group])
            _same(dv, want, everything if name == "v" else keys != key, "dv")


def _time(call, passes):
    call()
    torch.cuda.synchronize()
    best = math.inf
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(passes):
            call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) / passes)
    return best


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nk", [([2048, 2048], [2048, 2048]), ([2, 2, 2], [20000, 3000, 9000])])
def test_cost(nq, nk, dtype):
    """One more pass over the tiles, which it brings and works on one after the other between two barriers (three times a tile's time
    in the first pass), finding what is not finite (its reads of LDS are a fraction of the products'): 10 times leaves twice that."""
    x = _inputs(nq, nk, 8, 2, 64, dtype, 32)
    out, lse = _forward(x, nq, nk, True)
    v, d = x["v"].clone(), x["d_out"].clone()
    v[:, :, 3], d[:, :, 3] = math.nan, math.inf
    passes = 5
    clean, dirty = (_time(lambda: _forward(y, nq, nk, True), passes) for y in (x, dict(x, v=v)))
    print(f"[time] forward {clean:.3f} {dirty:.3f} ms", flush=True)
    assert dirty <= 10 * clean
    clean, dirty = (_time(lambda: _gradients(x, nq, nk, out, lse, d_out=y), passes) for y in (x["d_out"], d))
    print(f"[time] gradients {clean:.3f} {dirty:.3f} ms", flush=True)
    assert dirty <= 10 * clean
    everything = torch.full_like(x["v"], math.nan)
    dirty = _time(lambda: _gradients(x, nq, nk, out, lse, v=everything, k=everything), passes)
    print(f"[time] all keys and values {dirty:.3f} ms", flush=True)
    assert dirty <= 10 * clean


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_smallest_scale(dtype):
    """Probabilities are all alike, whatever the log-sum-exps over the scale are."""
    nq = nk = [70, 33]
    x = _inputs(nq, nk, 2, 1, 64, dtype, 33)
    scale = 2.0 ** -100
    out, lse = _forward(x, nq, nk, True, scale=scale)
    want = attention(x["q"], x["k"], x["v"], x["cu_q"], x["cu_k"], True, scale, None, x["d_out"])
    check(out, want["out"], "out")
    check(lse, want["lse"], "lse")
    dq, dk, dv = og.onecomp_attention_backward(x["d_out"], x["q"], x["k"], x["v"], out, lse, x["cu_q"], x["cu_k"], 70, 70, scale=scale)
    check(dv, want["dv"], "dv")
    check(dq, want["dq"], "dq")
    check(dk, want["dk"], "dk")

"""Embedding lookup and the table's gradient against plain forms in 64 bits."""
import pytest
import torch

import paper_2603_28845_amd as og
from token_oracle import embedding_grad, inside, log_uniform_ids

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape, dtype=F32):
    return torch.randn(*shape, generator=gen, device=DEV).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,width,vocab,scale", [(1, 1, 1, 1.0), (1, 4096, 1000, 8.0), (7, 63, 5, 0.5), (300, 1359, 777, 1.0), (1000, 64, 128000, -2.0)])
def test_lookup(dtype, n, width, vocab, scale):
    gen = _gen(n)
    table, tokens = _normal(gen, vocab, width, dtype=dtype), log_uniform_ids(gen, n, vocab, 0.1, -1, DEV)
    if n > 5:
        tokens[3], tokens[4], tokens[5] = vocab, -2 ** 31, 2 ** 31 - 1
    out = og.onecomp_embedding_forward(tokens, table, scale=scale)
    ok = inside(tokens, vocab)
    want = (table[torch.where(ok, tokens, 0).long()].float() * scale).to(dtype) * ok[:, None].to(dtype)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_lookup_of_strided_rows(dtype):
    gen = _gen(1)
    room, out = _normal(gen, 50, 101, dtype=dtype), torch.full((9, 77), 5.0, dtype=dtype, device=DEV)
    tokens = torch.tensor([3, 0, 49, -1, 7, 7, 3, 50, 1], dtype=torch.int32, device=DEV)
    table = room[:, 3:64]
    og.onecomp_embedding_forward(tokens, table, out=out[:, 1:62])
    want = table[tokens.clamp(0, 49).long()] * inside(tokens, 50)[:, None].to(dtype)
    assert torch.equal(out[:, 1:62], want) and bool((out[:, 0] == 5).all()) and bool((out[:, 62:] == 5).all())


def test_rows_of_padding_hold_zeros_whatever_the_table_holds():
    table = torch.full((4, 40), float("nan"), dtype=BF16, device=DEV)
    table[2] = 1.0
    out = og.onecomp_embedding_forward(torch.tensor([-1, 2, 9, 0], dtype=torch.int32, device=DEV), table, scale=float(3))
    assert bool((out[0] == 0).all()) and bool((out[1] == 3).all()) and bool((out[2] == 0).all()) and bool(out[3].isnan().all())


def _check(got, want, off):
    bad = (got.double() - want).abs() > off
    assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - want).abs() / off).max()))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,width,vocab,outside", [
    (1, 1, 1, 0.0), (1, 64, 1000, 0.0), (16, 100, 3, 0.0), (17, 513, 64, 0.2), (65, 8, 70000, 0.0), (500, 1359, 777, 0.05), (1000, 250, 65, 0.9),
    (3000, 72, 5, 0.0), (17000, 40, 2000, 0.1), (20001, 130, 1, 0.0), (33000, 24, 200000, 0.5)])
def test_gradient(dtype, n, width, vocab, outside):
    gen = _gen(n + width)
    tokens, d_out = log_uniform_ids(gen, n, vocab, outside, -1, DEV), _normal(gen, n, width, dtype=dtype)
    base = _normal(gen, vocab, width, dtype=dtype)
    want, off = embedding_grad(tokens, d_out, vocab, 0.5)
    got = og.onecomp_embedding_backward(tokens, d_out, vocab, scale=0.5)
    _check(got, want, off)
    assert torch.equal(got, og.onecomp_embedding_backward(tokens, d_out, vocab, scale=0.5))     # the same bits again
    want, off = embedding_grad(tokens, d_out, vocab, 2.0, base)
    got = og.onecomp_embedding_backward(tokens, d_out, vocab, scale=2.0, base=base)
    _check(got, want, off)
    # in place: the same, rows without a token left as they are
    there = base.clone()
    there[~torch.isin(torch.arange(vocab, device=DEV), tokens.long())] = float("inf")
    og.onecomp_embedding_backward(tokens, d_out, vocab, scale=2.0, base=there, d_table=there)
    used = torch.isin(torch.arange(vocab, device=DEV), tokens.long())
    assert torch.equal(there[used], got[used]) and bool((there[~used] == float("inf")).all())


def test_sorted_equal_and_alternating_tokens():
    """Runs that end with a segment, that fill several, and that alternate."""
    gen = _gen(5)
    for n in (15, 16, 17, 32, 33, 48, 200):
        for ids in (torch.zeros(n), torch.arange(n) // 16, torch.arange(n) // 7, torch.arange(n) % 2, torch.full((n,), 12.0), torch.arange(n).flip(0)):
            tokens, d_out = ids.to(torch.int32).to(DEV), _normal(gen, n, 24)
            want, off = embedding_grad(tokens, d_out, 201, 1.0)
            _check(og.onecomp_embedding_backward(tokens, d_out, 201), want, off)


def test_gradient_of_lookup_by_differences():
    """<d, lookup(table + e) - lookup(table - e)> is the gradient along e: the lookup is linear."""
    gen = _gen(6)
    tokens, table, e, d = log_uniform_ids(gen, 90, 40, 0.2, -1, DEV), _normal(gen, 40, 36), _normal(gen, 40, 36), _normal(gen, 90, 36)
    up, down = (og.onecomp_embedding_forward(tokens, (table + x).contiguous(), scale=1.5).double() for x in (e, -e))
    along = float((d.double() * (up - down)).sum() / 2)
    got = float((og.onecomp_embedding_backward(tokens, d, 40, scale=1.5).double() * e.double()).sum())
    # 90 x 36 differences of numbers of a few units, each off by 3 roundings of 2^-24; the gradient's sums as many
    size = float((d.double().abs() * 8).sum())
    assert abs(along - got) <= 8 * 2.0 ** -24 * size


def test_padding_is_not_read_and_results_only_where_they_belong():
    gen = _gen(7)
    n, vocab, width = 300, 50, 70
    tokens = log_uniform_ids(gen, n, vocab, 0.3, -1, DEV)
    d_out = _normal(gen, n, 90, dtype=BF16)[:, 11:81]
    d_out[tokens < 0] = float("nan")
    room = torch.full((vocab, 100), 7.0, dtype=BF16, device=DEV)
    ws = torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV)
    got = og.onecomp_embedding_backward(tokens, d_out, vocab, d_table=room[:, 5:75], workspace=ws)
    want, off = embedding_grad(tokens, d_out, vocab, 1.0)
    _check(got, want, off)
    assert bool((room[:, :5] == 7).all()) and bool((room[:, 75:] == 7).all())


def test_nothing_to_look_up():
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    assert og.onecomp_embedding_forward(none, torch.ones(3, 8, device=DEV)).shape == (0, 8)
    assert bool((og.onecomp_embedding_backward(none, torch.empty(0, 8, device=DEV), 5) == 0).all())
    base = torch.ones(5, 8, device=DEV)
    assert torch.equal(og.onecomp_embedding_backward(none, torch.empty(0, 8, device=DEV), 5, base=base), base)
    assert torch.equal(og.onecomp_embedding_backward(none, torch.empty(0, 8, device=DEV), 5, base=base, d_table=base), torch.ones(5, 8, device=DEV))
    outside = torch.full((40,), -1, dtype=torch.int32, device=DEV)
    assert bool((og.onecomp_embedding_backward(outside, torch.ones(40, 8, device=DEV), 5) == 0).all())


def test_tables_past_32_bits():
    gen = _gen(8)
    vocab, width = 530000, 4104                                    # 2.2e9 entries
    table = torch.zeros(vocab, width, dtype=BF16, device=DEV)
    rows = torch.tensor([0, 523264, 523265, vocab - 1], device=DEV)
    table[rows] = _normal(gen, 4, width, dtype=BF16)
    tokens = rows.to(torch.int32).repeat(3)
    assert torch.equal(og.onecomp_embedding_forward(tokens, table), table[rows].repeat(3, 1))
    d_out = _normal(gen, 12, width, dtype=BF16)
    want = d_out.double().view(3, 4, width).sum(0)
    got = og.onecomp_embedding_backward(tokens, d_out, vocab, d_table=table)
    off = (5 * 2.0 ** -24) * d_out.double().abs().view(3, 4, width).sum(0) + 2.0 ** -8 * want.abs() * 1.01
    _check(got[rows], want, off + 1e-40)
    got[rows] = 0
    assert not bool(got.any())

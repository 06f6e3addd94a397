"""Calls of more blocks than one launch holds, 2^32 threads: very many sequences, ranges of few rows by very wide weights, and
as many rows as an operator takes."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2609_06086_amd import layers as L  # noqa: E402
from paper_2609_06086_amd import poseidon as P  # noqa: E402

V = 2.0 ** -23          # two roundings in 32 bits


def _gpu(gigabytes):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"less than {gigabytes} GB free")
    return torch.device("cuda:0")


def test_blocks_past_31_bits_are_refused():
    a, heads, no = 1 << 20, [1 << 20, 8192, 8], ctypes.c_void_p(None)
    f, b = L.lib().poseidon_attention_forward, L.lib().poseidon_attention_backward
    for sequences, tokens in ((1 << 21, 16), ((1 << 21) - 1, 128)):
        assert f(*heads * 3, 2, tokens, 1024, 1024, 8, 0.5, a, sequences, *heads, a, no) == P.POSEIDON_E_RANGE
        assert b(*heads * 5, a, 2, tokens, 1024, 1024, 8, 0.5, a, sequences, *heads * 3, a, 1 << 40, no) == P.POSEIDON_E_RANGE


@pytest.mark.gpu
def test_attention_of_a_million_sequences():
    """One token each, so a token's result is its value; some tokens lie before the first sequence and after the last.  34 heads on
    17: 36 million blocks forward and for dq, 18 million for dk and dv."""
    dev = _gpu(40)
    n, heads, kv, dim, out_of = 1 << 20, 34, 17, 8, 100
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    q, k, v, dout = (torch.randn(n, h, dim, generator=g, device=dev).bfloat16() for h in (heads, kv, kv, heads))
    offsets = torch.arange(out_of, n - out_of + 1, dtype=torch.int32, device=dev)
    out, lse = L.poseidon_attention_forward(q, k, v, offsets)
    inside = slice(out_of, n - out_of)
    wide = v.repeat_interleave(2, 1)
    assert torch.equal(out[inside], wide[inside])
    # a sum of 8 products, the scale, and the logarithm of a sum of one: some ten roundings of what the score's parts add up to
    scores, size = ((x(q.double()) * x(k.repeat_interleave(2, 1).double())).sum(2).t() * dim ** -0.5 for x in (lambda t: t, torch.abs))
    assert ((lse.double() - scores).abs() <= 12 * V * (size + 1))[:, inside].all()
    for t in (slice(0, out_of), slice(n - out_of, n)):
        assert not out[t].any() and torch.isneginf(lse[:, t]).all()
    del scores, size
    dq, dk, dv = L.poseidon_attention_backward(dout, q, k, v, out, lse, offsets)
    both = dout.double().view(n, kv, 2, dim)
    off = (dv.double() - both.sum(2)).abs() - 2.0 ** -8 * both.sum(2).abs() - 3 * 2.0 ** -8 * both.abs().sum(2)   # p is 1 to a rounding of bf16
    assert (off[inside] <= 0).all()
    # ds = p (dp - delta), two sums of the same 8 products: what is left are their roundings
    parts = (dout.double() * wide.double()).abs().sum(2, keepdim=True) * 20 * V * dim ** -0.5
    assert (dq[inside].double().abs() <= (parts * k.repeat_interleave(2, 1).double().abs())[inside]).all()
    over = (parts * q.double().abs()).view(n, kv, 2, dim).sum(2)
    assert (dk[inside].double().abs() <= over[inside]).all()
    for x in (dq, dk, dv):
        assert not x[:out_of].any() and not x[n - out_of:].any()


@pytest.mark.gpu
def test_products_of_few_rows_by_very_wide_weights():
    """300 ranges of one row by 2^20 x 8 weights, with rows of no range before and after: 20 million blocks."""
    dev = _gpu(40)
    ranges, wide, deep = 300, 1 << 20, 8
    g = torch.Generator(device=dev)
    g.manual_seed(2)
    w = torch.randn(ranges, wide, deep, generator=g, device=dev, dtype=torch.bfloat16)
    x = torch.randn(ranges + 5, deep, generator=g, device=dev).bfloat16()
    offsets = torch.arange(2, ranges + 3, dtype=torch.int32, device=dev)
    out = torch.full((ranges + 5, wide), 7.0, dtype=torch.bfloat16, device=dev)
    L.poseidon_expert_product(x, w, offsets, out=out)
    assert not out[:2].any() and not out[ranges + 2:].any()
    for r in range(ranges):
        each = w[r].double() * x[r + 2].double()
        want, size = each.sum(1), each.abs().sum(1)
        assert ((out[r + 2].double() - want).abs() <= 2.0 ** -8 * want.abs() + (1 + 2.0 ** -8) * (deep + 2) * V * size).all()


@pytest.mark.gpu
@pytest.mark.parametrize("transposed", [False, True])
def test_products_of_the_most_rows(transposed):
    """2^31 - 1 rows of one value: each result is one product, rounded once."""
    dev = _gpu(40)
    n = L.ROWS_MAX
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    x = torch.randn(n, 1, generator=g, device=dev, dtype=torch.bfloat16)
    w = torch.full((1, 1), 1.7109375, dtype=torch.bfloat16, device=dev)
    out = torch.full((n, 1), 7.0, dtype=torch.bfloat16, device=dev)
    L.poseidon_expert_product(x, w, transposed=transposed, out=out)
    for a in range(0, n, 1 << 28):
        assert torch.equal(out[a:a + (1 << 28)], x[a:a + (1 << 28)] * w)

"""Variants of norm, expert product and attention that only larger calls reach, each with a check that its shapes do reach it: the
larger tiles of products in both directions and types, blocks that go through several heads of several tiles, norms of two slices
a lane over many rows, and norms with streaming accesses.

References are in 64 bits on the GPU.  Bounds as in the tests beside this one: ROUND is a rounding to nearest, relative, V two
roundings in 32 bits.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_06086_amd import layers as L  # noqa: E402
from test_gpu_transformer import KIND, KINDS, ROUND, SHORT, STEP, V, _attention_case, _make, _same, dev, test_norm as _norm  # noqa: E402, F401

pytestmark = pytest.mark.gpu


# ---- products ----

def _tiles(rows, ranges, wide, size, columns):
    return (rows // size + ranges) * -(-wide // columns)


def _check_product(got, x, w, offsets, transposed, out_kind):
    for r, (a, b) in enumerate(zip(offsets, offsets[1:])):
        m = w[r].double()
        m = m if transposed else m.t().contiguous()
        want, size = x[a:b].double() @ m, x[a:b].double().abs() @ m.abs()
        slack = (x.shape[1] + 2) * V * size
        off = (got[a:b].double() - want).abs() - (slack + ROUND[out_kind] * (want.abs() + slack) + STEP[out_kind])
        assert b == a or float(off.max()) <= 0, (r, float(off.max()))
    assert not got[:offsets[0]].any() and not got[offsets[-1]:].any()


def _run_product(rng, dev, kind, rows, offsets, deep, wide, transposed, pad=0, shift=0):  # noqa: F811
    o, i = (deep, wide) if transposed else (wide, deep)
    ranges = len(offsets) - 1
    x = _make(rng, (rows, deep), kind, dev, pad=pad, shift=shift)
    w = _make(rng, (ranges * o, i), kind, dev, spread=0.5).contiguous().view(ranges, o, i)
    at = torch.tensor(offsets, dtype=torch.int32, device=dev)
    for out_kind in (kind, "f32"):
        got = L.poseidon_expert_product(x, w, at, transposed=transposed, dtype=KIND[out_kind])
        _check_product(got, x, w, offsets, transposed, out_kind)


@pytest.mark.parametrize("kind", SHORT)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("deep, wide", [(64, 1000), (72, 1024), (128, 1000), (200, 1000), (264, 1000), (392, 1000), (456, 1000), (584, 1000),
                                        (37, 1001), (64, 1001), (129, 1000), (200, 1001), (257, 1001), (333, 1001), (400, 1003),
                                        (449, 1001), (577, 1001)])
def test_products_over_the_largest_tiles(dev, kind, transposed, deep, wide):  # noqa: F811
    """256 x 256 tiles, of whole pieces and of odd rows, one stage of the sum to ten; ranges end anywhere, one is empty, and
    rows lie before and after them."""
    rows, offsets = 12000, [3, 4100, 4100, 4357, 11900]
    assert _tiles(rows, 4, wide, 256, 256) >= 180
    rng = np.random.default_rng(deep + wide)
    _run_product(rng, dev, kind, rows, offsets, deep, wide, transposed)


@pytest.mark.parametrize("kind", SHORT)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("deep, wide, pad, shift", [(64, 1000, 0, 0), (200, 1000, 0, 0), (264, 1000, 8, 0), (392, 1000, 0, 0), (37, 1001, 0, 0),
                                                    (200, 1001, 0, 0), (264, 1000, 3, 1), (333, 1003, 0, 0), (449, 1001, 0, 0)])
def test_products_over_the_middle_tiles(dev, kind, transposed, deep, wide, pad, shift):  # noqa: F811
    """128 x 128 tiles, of whole pieces and of odd rows or addresses."""
    rows, offsets = 4300, [0, 1000, 1001, 2900, 4290]
    assert _tiles(rows, 4, wide, 256, 256) < 180 and _tiles(rows, 4, wide, 128, 128) >= 256
    rng = np.random.default_rng(deep + wide + pad)
    _run_product(rng, dev, kind, rows, offsets, deep, wide, transposed, pad, shift)


# ---- attention ----

def _split(tokens, sequences, heads, kv_heads, dim):
    """Blocks that share a key's query heads (sequences 0: a call without offsets)."""
    group = heads // kv_heads
    tiles = tokens // 128 + sequences if sequences else -(-tokens // 128)
    n = 1
    while n < group and (tiles * kv_heads * n < (2048 if sequences > 1 else 1024) or group % n):
        n += 1
    while n > 1 and (group % n or n * tokens * kv_heads * dim * 8 > 1 << 30):
        n -= 1
    return n


def _attention64(q, k, v, dout, out, offsets, scale, kind):
    """((out, lse, dq, dk, dv) in 64 bits from the `out` that was given, what each may be off by but for its own rounding), a
    sequence and a head at a time.  A score is off by `a`, an exponential relatively by that and a few roundings; p and ds are
    rounded to `kind` before their products, and are off by up to `step` where they are smaller than what is held."""
    Q, K, X, D, U = (x.double() for x in (q, k, v, dout, out))
    n, heads, dim = Q.shape
    group, r, step = heads // K.shape[1], ROUND[kind], max(STEP[kind], 2.0 ** -126)
    want = [torch.zeros_like(x) for x in (Q, Q[:, :, 0].t(), Q, K, K)]
    slack = [torch.zeros_like(x) for x in want]
    want[1].fill_(-float("inf"))

    def times(a, b):
        return a @ b.contiguous()
    for lo, hi in zip(offsets, offsets[1:]):
        m, of = hi - lo, slice(lo, hi)
        if not m:
            continue
        later = torch.ones(m, m, dtype=torch.bool, device=q.device).triu(1)
        for h in range(heads):
            j = h // group
            x, y, z, d, u = Q[of, h], K[of, j], X[of, j], D[of, h], U[of, h]
            s = times(x, y.t()).mul_(scale)
            a = (dim + 6) * V * abs(scale) * times(x.abs(), y.abs().t())
            top = s.masked_fill(later, -float("inf")).amax(1, keepdim=True)
            a = (a + 4 * V * (s.abs() + top.abs())).masked_fill_(later, 0)
            s.masked_fill_(later, -float("inf"))
            total = torch.exp(s - top).sum(1, keepdim=True)
            p = torch.exp(s - top) / total
            elog = a.amax(1, keepdim=True) + (m + 10) * V + 4 * V * top.abs()
            want[1][h, of], slack[1][h, of] = (top + torch.log(total))[:, 0], elog[:, 0]
            rel = a + elog + 6 * V
            want[0][of, h] = times(p, z)
            slack[0][of, h] = times((r + 2 * rel + (m + 8) * V) * p, z.abs()) + step / total.clamp(min=1) * z.abs().sum(0)
            dp = times(d, z.t()) - (d * u).sum(1, keepdim=True)
            edp = (dim + 4) * V * (times(d.abs(), z.abs().t()) + (d.abs() * u.abs()).sum(1, keepdim=True))
            ds = p * dp
            more = rel + r + (m * group + 8) * V
            eds = (more * (ds.abs() + p * edp) + p * edp + step).masked_fill_(later, 0)
            ep = (more * p + step).masked_fill_(later, 0)
            want[2][of, h], slack[2][of, h] = scale * times(ds, y), abs(scale) * times(eds, y.abs())
            want[3][of, j] += scale * times(ds.t(), x)
            slack[3][of, j] += abs(scale) * times(eds.t(), x.abs())
            want[4][of, j] += times(p.t(), d)
            slack[4][of, j] += times(ep.t(), d.abs())
    return want, slack


@pytest.mark.parametrize("kind", SHORT)
@pytest.mark.parametrize("n, heads, kv, dim, cuts, split", [(2048, 128, 32, 16, None, 2), (200, 1024, 512, 8, None, 1), (4096, 64, 16, 128, None, 2),
                                                             (4096, 128, 32, 64, [5, 1000, 1001, 4000], 2), (3000, 96, 48, 72, None, 1),
                                                             (1500, 12, 2, 128, [0, 700, 1500], 6)])
def test_several_heads_of_several_tiles(dev, kind, n, heads, kv, dim, cuts, split):  # noqa: F811
    """A block of the kernel for dk and dv goes through its query heads at each tile of queries; or through one head, and the
    blocks' parts are added."""
    offsets = [0, n] if cuts is None else cuts
    assert _split(n, 0 if cuts is None else len(cuts) - 1, heads, kv, dim) == split
    rng = np.random.default_rng(n + heads)
    q, k, v, dout = _attention_case(rng, dev, kind, n, heads, kv, dim, spread=1.2)
    at = None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device=dev)
    out, lse = L.poseidon_attention_forward(q, k, v, at)
    got = (out, *L.poseidon_attention_backward(dout, q, k, v, out, lse, at))
    got = (out, lse, *got[1:])
    for i, (x, want, slack) in enumerate(zip(got, *_attention64(q, k, v, dout, out, offsets, dim ** -0.5, kind))):
        own, step = (2 * V, 0.0) if i == 1 else (ROUND[kind], STEP[kind])
        off = (x.double() - want).abs() - (slack + own * (want.abs() + slack) + step)
        off = off.t() if i == 1 else off
        assert float(off[offsets[0]:offsets[-1]].max()) <= 0, (i, float(off.max()))
        x = x.t() if i == 1 else x
        outside = torch.cat([x[:offsets[0]], x[offsets[-1]:]])
        assert torch.isneginf(outside).all() if i == 1 else not outside.any()


def test_offsets_that_descend_stay_in_the_buffers(dev):  # noqa: F811
    """Which rows are written is open, but none outside of the results."""
    rng = np.random.default_rng(18)
    down = torch.tensor([30, 10, 35, 0, 40], dtype=torch.int32, device=dev)

    def guarded(rows, *inner):
        size = int(np.prod(inner))
        whole = torch.full((rows + 200, size + 16), 7.0, dtype=torch.bfloat16, device=dev)
        return whole, whole[100:100 + rows, 8:8 + size].unflatten(1, inner) if len(inner) > 1 else whole[100:100 + rows, 8:8 + size]

    def untouched(whole, rows):
        edges = whole.clone()
        edges[100:100 + rows, 8:-8] = 7
        assert (edges == 7).all()
    for rows, wide in ((40, 300), (400, 304)):
        x, w = _make(rng, (rows, 64), "bf16", dev), _make(rng, (4 * wide, 64), "bf16", dev).contiguous().view(4, wide, 64)
        whole, out = guarded(rows, wide)
        L.poseidon_expert_product(x, w, down, out=out)
        untouched(whole, rows)
        whole, out = guarded(rows, 64)
        L.poseidon_expert_product(_make(rng, (rows, wide), "bf16", dev), w, down, transposed=True, out=out)
        untouched(whole, rows)
    n = 40
    q, k, v, dout = _attention_case(rng, dev, "bf16", n, 4, 2, 64)
    whole, out = guarded(n, 4, 64)
    _, lse = L.poseidon_attention_forward(q, k, v, down, out=out)
    untouched(whole, n)
    (wq, dq), (wk, dk), (wv, dv) = guarded(n, 4, 64), guarded(n, 2, 64), guarded(n, 2, 64)
    L.poseidon_attention_backward(dout, q, k, v, out, lse, down, dq=dq, dk=dk, dv=dv)
    for whole in (wq, wk, wv):
        untouched(whole, n)


# ---- norm ----

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d, pad, shift", [(12200, 0, 0), (16384, 0, 0), (9001, 3, 1)])
def test_norm_of_two_slices_over_many_rows(dev, kind, d, pad, shift):  # noqa: F811
    """At most 256 blocks of one row each at a time: every block takes a second and a third."""
    _norm(dev, kind, (700, d), True, pad, shift)


@pytest.mark.parametrize("kind, d, residual", [("bf16", 64, True), ("bf16", 512, True), ("f16", 1000, False), ("bf16", 4096, True), ("f16", 4096, True),
                                               ("f32", 4096, True), ("bf16", 4095, True), ("bf16", 9216, True), ("f32", 640, False)])
def test_norm_with_streaming_accesses(dev, kind, d, residual):  # noqa: F811
    """A call of more than 256 MB gives a row what a call of a few rows gives it; the weight's gradient adds up over all."""
    n = (290 << 20) // (4 if kind == "f32" else 2) // d // 2 + 1
    g = torch.Generator(device=dev)
    g.manual_seed(d)
    x, dout, *more = (torch.randn(n, d, generator=g, device=dev).to(KIND[kind]) for _ in range(4 if residual else 2))
    r, dsum = more if residual else (None, None)
    weight = 1 + 0.2 * torch.randn(d, generator=g, device=dev)
    size = x.element_size()
    assert n * d * size * 2 > 256 << 20
    y = L.poseidon_norm_forward(x, weight, r, keep_out=True, keep_sum=True)
    h = x if r is None else y.sum
    kept_x, dweight = L.poseidon_norm_backward(dout, y.kept_sum, y.rstd, weight, dsum)
    whole_x, whole_w = L.poseidon_norm_backward(dout, h, y.rstd, weight, dsum)
    step = n // 16 + 1
    assert step * d * (5 * size + 2) < 256 << 20
    each = -(-d // 64)
    for a in range(0, n, step):
        b = min(n, a + step)
        part = slice(a, b)
        few = L.poseidon_norm_forward(x[part], weight, None if r is None else r[part], keep_out=True, keep_sum=True)
        _same(y.out[part], few.out)
        _same(y.rstd[part], few.rstd)
        if residual:
            _same(y.sum[part], few.sum)
        for got, want in ((y.kept_out, few.kept_out), (y.kept_sum, few.kept_sum)):
            assert got.codes.shape[1] == each * 64
            _same(got.codes[part], want.codes)
            _same(got.scales[part], want.scales)
        s = None if dsum is None else dsum[part]
        _same(kept_x[part], L.poseidon_norm_backward(dout[part], few.kept_sum, few.rstd, weight, s)[0])
        _same(whole_x[part], L.poseidon_norm_backward(dout[part], h[part], few.rstd, weight, s)[0])
    for got, at in ((dweight, L.poseidon_restore(y.kept_sum, dtype=torch.float32)), (whole_w, h)):
        want, sizes = torch.zeros(d, dtype=torch.float64, device=dev), torch.zeros(d, dtype=torch.float64, device=dev)
        for a in range(0, n, step):
            one = dout[a:a + step].double() * at[a:a + step].double() * y.rstd[a:a + step].double().unsqueeze(1)
            want += one.sum(0)
            sizes += one.abs().sum(0)
        assert ((got.double() - want).abs() <= (n + 8) * V * sizes).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_norm_of_rows_of_zeros(dev, kind):  # noqa: F811
    """1 / sqrt(eps), infinite without one; the rows beside them are what they are alone."""
    x = torch.randn(3, 200, device=dev).to(KIND[kind])
    x[1] = 0
    weight = torch.ones(200, device=dev)
    for eps in (0.0, 1e-6, 1e30):
        y = L.poseidon_norm_forward(x, weight, eps=eps)
        if eps:
            assert abs(float(y.rstd[1]) - eps ** -0.5) <= 4 * V * eps ** -0.5 and not y.out[1].any()
        else:
            assert torch.isinf(y.rstd[1]) and torch.isnan(y.out[1]).all()
        _same(y.out[::2].contiguous(), L.poseidon_norm_forward(x[::2].contiguous(), weight, eps=eps).out)

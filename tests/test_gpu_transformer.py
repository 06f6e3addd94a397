"""Norm, products by expert and attention on the GPU against the 64-bit oracle.

Bounds, derived before the first run: ROUND is a rounding to nearest relative to the value (half a unit in the last place at
the lower end of a binade), STEP half of the least step below the normal range, V two roundings in 32 bits.  A sum of n
products in 32 bits is off by at most (n + 2) V times the sum of their absolute values, whatever its order.
"""
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layers as O  # noqa: E402
from paper_2609_06086_amd import layers as L  # noqa: E402
from paper_2609_06086_amd import poseidon as P  # noqa: E402

pytestmark = pytest.mark.gpu

KIND = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
STEP = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}
V = 2.0 ** -23
KINDS, SHORT = ["f32", "f16", "bf16"], ["f16", "bf16"]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _make(rng, shape, kind, dev, spread=1.0, pad=0, shift=0):
    """Values over a few binades; pad: extra columns of the rows' pitch, shift: values before the first one."""
    n, d = shape
    v = np.clip(rng.normal(size=shape) * np.exp(rng.normal(size=shape) * spread), -1e3, 1e3)
    flat = torch.full((shift + n * (d + pad) + 8,), float("nan"), dtype=KIND[kind], device=dev)
    x = flat[shift:shift + n * (d + pad)].view(n, d + pad)[:, :d]
    x.copy_(torch.from_numpy(v).to(dev))
    return x


def _np(x):
    return x.double().cpu().numpy()


def _check(got, want, slack, kind):
    """|got - want| <= slack + the rounding to `kind`."""
    got = _np(got)
    assert got.shape == want.shape
    off = np.abs(got - want) - (slack + ROUND[kind] * (np.abs(want) + slack) + STEP[kind])
    assert (off <= 0).all(), (float(off.max()), np.unravel_index(off.argmax(), off.shape))


def _same(a, b):
    assert a.dtype == b.dtype and a.shape == b.shape and torch.equal(a.reshape(-1).view(torch.uint8), b.reshape(-1).view(torch.uint8))


# ---- norm ----

def _check_norm_forward(y, x, residual, weight, eps, kind):
    h = _np(x) if residual is None else _np(x) + _np(residual)
    d, w = h.shape[1], _np(weight)
    out, _, rstd = O.norm_forward(h, None, w, eps)
    few = (d + 8) * V                                   # the sum of squares, relative; the root, the quotient, the sum itself
    _check(y.rstd, rstd, few * rstd, "f32")
    _check(y.out, out, few * np.abs(out), kind)
    if residual is None:
        assert y.sum is None
    else:
        _check(y.sum, h, V * np.abs(h), kind)


def _check_norm_backward(dx, dweight, dout, h, rstd, weight, dsum, kind):
    """h and rstd as they were given: what the kernel starts from."""
    dout, h, rstd, w = _np(dout), _np(h), _np(rstd), _np(weight)
    n, d = h.shape
    s = None if dsum is None else _np(dsum)
    want, want_w = O.norm_backward(dout, h, rstd, w, s)
    u, g = np.abs(h * rstd[:, None]), np.abs(dout * w)
    along = (u * g).sum(axis=1, keepdims=True) / d
    slack = rstd[:, None] * (8 * V * g + (d + 12) * V * u * along) + (0 if s is None else V * np.abs(s))
    _check(dx, want, slack, kind)
    if dweight is not None:
        _check(dweight, want_w, (n + 8) * V * (np.abs(dout) * u).sum(axis=0), "f32")


NORM_SHAPES = [(1, 1), (3, 7), (2, 64), (5, 128), (33, 129), (9, 250), (17, 1000), (300, 64), (4, 1365), (2100, 72), (6, 4100), (3, 8192),
               (2, 16383), (5, 16384)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", NORM_SHAPES)
@pytest.mark.parametrize("residual, pad, shift", [(True, 0, 0), (False, 0, 0), (True, 3, 1)])
def test_norm(dev, kind, shape, residual, pad, shift):
    rng = np.random.default_rng(shape[0] * 31 + shape[1])
    n, d = shape
    x = _make(rng, shape, kind, dev, pad=pad, shift=shift)
    r = _make(rng, shape, kind, dev, pad=2 * pad, shift=shift) if residual else None
    weight = torch.from_numpy(rng.normal(size=d) + 1).to(dev).to(KIND[KINDS[(n + d) % 3]])
    y = L.poseidon_norm_forward(x, weight, r, eps=1e-5, keep_out=True, keep_sum=True)
    _check_norm_forward(y, x, r, weight, 1e-5, kind)
    kept = L.poseidon_stash(y.out), L.poseidon_stash(x if r is None else y.sum)
    for got, want in zip((y.kept_out, y.kept_sum), kept):      # the 8-bit form of what was written
        _same(got.codes, want.codes)
        _same(got.scales, want.scales)
    dout = _make(rng, shape, kind, dev, pad=pad, shift=shift)
    dsum = _make(rng, shape, kind, dev, pad=pad) if residual else None
    dx, dweight = L.poseidon_norm_backward(dout, y.kept_sum, y.rstd, weight, dsum)
    h = L.poseidon_restore(y.kept_sum, dtype=torch.float32)
    _check_norm_backward(dx, dweight, dout, h, y.rstd, weight, dsum, kind)
    whole = x if r is None else y.sum
    dx, dweight = L.poseidon_norm_backward(dout, whole, y.rstd, weight, dsum)
    _check_norm_backward(dx, dweight, dout, whole, y.rstd, weight, dsum, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [130, 300, 500, 700, 1030, 1500, 2500, 3500, 4600, 5120, 6100, 7168, 8200, 9216, 12200])
def test_norm_of_widths(dev, kind, d):
    """Teams of every number of waves."""
    test_norm(dev, kind, (7, d), True, 0, 0)


def test_norm_of_many_rows(dev):
    """Teams go through many rows, and the weight's gradient adds up over all of them; into rows with gaps, added to what is there."""
    rng = np.random.default_rng(3)
    for n, d in ((70001, 24), (5003, 640), (2500, 5000)):
        x, dout = (_make(rng, (n, d), "bf16", dev, spread=0.5) for _ in range(2))
        weight = torch.from_numpy(rng.normal(size=d)).to(dev).float()
        out = torch.full((n, d + 3), 7.0, dtype=torch.bfloat16, device=dev)
        y = L.poseidon_norm_forward(x, weight, keep_sum=True, out=out[:, 1:1 + d])
        _check_norm_forward(y, x, None, weight, 1e-6, "bf16")
        assert (out[:, 0] == 7).all() and (out[:, 1 + d:] == 7).all()
        start = torch.randn(d, device=dev)
        total, gaps = start.clone(), torch.full((n, d + 5), 7.0, dtype=torch.bfloat16, device=dev)
        dx, dweight = L.poseidon_norm_backward(dout, y.kept_sum, y.rstd, weight, dx=gaps[:, 2:2 + d], dweight=total, accumulate=True)
        assert dweight is total and (gaps[:, :2] == 7).all() and (gaps[:, 2 + d:] == 7).all()
        h = L.poseidon_restore(y.kept_sum, dtype=torch.float32)
        alone_x, alone = L.poseidon_norm_backward(dout, y.kept_sum, y.rstd, weight)
        _check_norm_backward(dx, alone, dout, h, y.rstd, weight, None, "bf16")
        _same(dx.contiguous(), alone_x)
        assert torch.allclose(total, start + alone, rtol=V, atol=0)       # one rounding each
        frozen_x, none = L.poseidon_norm_backward(dout, y.kept_sum, y.rstd, weight, weight_gradient=False)
        assert none is None
        _same(frozen_x, alone_x)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_norm_of_extreme_rows(dev, kind):
    """Rows whose squares leave the 32-bit range, rows of zeros, and infinities and NaN, which stay in their rows."""
    info, d = torch.finfo(KIND[kind]), 200
    x = torch.randn(9, d, dtype=torch.float64)
    x[1] *= 2.0 ** 90
    x[2] *= 2.0 ** -90
    x[3] = 0
    x[4] = 2.0 ** 125
    x[5, 3] = float("inf")
    x[6, 4] = float("nan")
    x[7] = 0
    x[7, 9] = 2.0 ** 100
    x = x.to(KIND[kind]).to(dev)
    weight = torch.ones(d, device=dev)
    for eps in (1e-6, 0.0, 1e30):
        y = L.poseidon_norm_forward(x, weight, eps=eps)
        fine = [0, 1, 2, 4, 7, 8] + ([3] if eps else [])
        _check_norm_forward(L.Norm(y.out[fine], None, y.rstd[fine], None, None), x[fine], None, weight, eps, kind)
        assert torch.isnan(y.out[6]).all() and torch.isnan(y.out[5, 3]) and (y.out[5, :3] == 0).all()
    assert torch.isinf(y.rstd[3]) or y.rstd[3] > 0
    assert info.bits


# ---- products by expert ----

def _check_product(got, x, w, offsets, transposed, out_kind):
    x, w = _np(x), _np(w)
    want = O.expert_product(x, w, offsets, transposed)
    deep = x.shape[1]
    _check(got, want, (deep + 2) * V * O.expert_product(np.abs(x), np.abs(w), offsets, transposed), out_kind)


def _product_case(rng, dev, kind, offsets, rows, o, i, transposed, out_kind=None, pad=0, shift=0):
    ranges = len(offsets) - 1
    x = _make(rng, (rows, o if transposed else i), kind, dev, pad=pad, shift=shift)
    w = _make(rng, (ranges * o, i), kind, dev, spread=0.5).contiguous().view(ranges, o, i)
    at = torch.tensor(offsets, dtype=torch.int32, device=dev)
    out = L.poseidon_expert_product(x, w, at, transposed=transposed, dtype=None if out_kind is None else KIND[out_kind])
    _check_product(out, x, w, offsets, transposed, out_kind or kind)
    outside = torch.ones(rows, dtype=torch.bool)
    outside[offsets[0]:offsets[-1]] = False
    assert not out.cpu()[outside].any()
    return x, w, at, out


@pytest.mark.parametrize("kind", SHORT)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("o, i", [(1, 1), (8, 8), (7, 9), (64, 32), (65, 40), (130, 136), (200, 333), (96, 264), (300, 5),
                                  (5, 300), (333, 9)])
@pytest.mark.parametrize("rows, offsets", [(1, [0, 1]), (5, [0, 0, 2, 2, 5]), (40, [3, 20, 20, 33]), (300, [0, 130, 131, 300]), (333, [7, 7, 320, 320])])
def test_product(dev, kind, transposed, o, i, rows, offsets):
    rng = np.random.default_rng(rows + o * 7 + i)
    _product_case(rng, dev, kind, offsets, rows, o, i, transposed)
    _product_case(rng, dev, kind, offsets, rows, o, i, transposed, "f32", pad=3, shift=1)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows, o, i, ranges", [(5000, 1024, 1032, 3), (9000, 520, 72, 40), (5000, 1001, 1027, 2), (2600, 2048, 520, 7)])
def test_product_over_large_tiles(dev, transposed, rows, o, i, ranges):
    """256 x 256 tiles, in whole pieces and in odd sizes, over ranges that end anywhere."""
    rng = np.random.default_rng(rows)
    cuts = sorted(rng.integers(0, rows + 1, size=ranges - 1).tolist())
    _product_case(rng, dev, "bf16", [0] + cuts + [rows], rows, o, i, transposed)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("deep", [8, 64, 72, 128, 136, 200, 264, 333, 392, 456, 520])
def test_product_over_small_and_middle_tiles(dev, transposed, deep):
    """64 x 128 and 128 x 128 tiles with one stage of the sum to nine, the last ones of a range and a row part full."""
    rng = np.random.default_rng(deep)
    for rows, offsets, wide in ((150, [0, 150], 264), (600, [5, 230, 230, 231, 590], 136), (2100, [0, 2100], 2000), (4300, [0, 1000, 1001, 2900, 4290], 1000)):
        o, i = (deep, wide) if transposed else (wide, deep)
        _product_case(rng, dev, "bf16", offsets, rows, o, i, transposed)


@pytest.mark.parametrize("kind", SHORT)
def test_product_of_few_rows(dev, kind):
    """One token by experts, the most rows that go the short way, and one range that has them all."""
    rng = np.random.default_rng(8)
    some = np.sort(rng.integers(0, 9, size=63)).tolist()
    for rows, offsets in ((8, [0] + some + [8]), (200, [0] + np.sort(rng.integers(0, 201, size=63)).tolist() + [200]),
                          (100, [0] * 30 + [100] * 35), (256, [0] * 64 + [256]), (64, [0, 64])):
        for o, i in ((48, 264), (33, 1100), (17, 5)):
            _product_case(rng, dev, kind, offsets, rows, o, i, False)


def test_product_of_many_ranges_and_of_one_matrix(dev):
    rng = np.random.default_rng(5)
    cuts = np.sort(rng.integers(0, 3001, size=510)).tolist()
    for transposed in (False, True):
        _product_case(rng, dev, "bf16", [0] + cuts + [3000], 3000, 40, 24, transposed)
    x, w = _make(rng, (700, 128), "bf16", dev), _make(rng, (72, 128), "bf16", dev)
    out = L.poseidon_expert_product(x, w)
    _check_product(out, x, w.view(1, 72, 128), [0, 700], False, "bf16")
    wide = torch.full((700, 80), 7.0, dtype=torch.float32, device=dev)
    L.poseidon_expert_product(x, w, out=wide[:, 3:75])
    _check_product(wide[:, 3:75], x, w.view(1, 72, 128), [0, 700], False, "f32")
    assert (wide[:, :3] == 7).all() and (wide[:, 75:] == 7).all()


def test_offsets_outside_of_the_rows(dev):
    """Bounds are cut to the rows that there are, and offsets that descend touch nothing else."""
    rng = np.random.default_rng(18)
    x, w = _make(rng, (40, 64), "bf16", dev), _make(rng, (2 * 300, 64), "bf16", dev).contiguous().view(2, 300, 64)
    big = _make(rng, (400, 64), "bf16", dev)
    q, k, v, dout = _attention_case(rng, dev, "bf16", 40, 2, 1, 64)
    for given, cut in (([-5, 20, 1000], [0, 20, 40]), ([-2 ** 31, -1, 2 ** 31 - 1], [0, 0, 40]), ([2 ** 31 - 1] * 3, [40, 40, 40])):
        at, inside = (torch.tensor(o, dtype=torch.int32, device=dev) for o in (given, cut))
        _same(L.poseidon_expert_product(x, w, at), L.poseidon_expert_product(x, w, inside))
        _same(L.poseidon_expert_product(big, w, at), L.poseidon_expert_product(big, w, torch.tensor([min(max(o, 0), 400) for o in given], dtype=torch.int32, device=dev)))
        out, lse = L.poseidon_attention_forward(q, k, v, at)
        want = L.poseidon_attention_forward(q, k, v, inside)
        _same(out, want[0])
        _same(lse, want[1])
        for a, b in zip(L.poseidon_attention_backward(dout, q, k, v, out, lse, at), L.poseidon_attention_backward(dout, q, k, v, out, lse, inside)):
            _same(a, b)
    down = torch.tensor([30, 10, 35], dtype=torch.int32, device=dev)
    assert L.poseidon_expert_product(x, w, down).shape == (40, 300)
    assert L.poseidon_attention_forward(q, k, v, down)[0].shape == q.shape
    torch.cuda.synchronize()


def test_product_keeps_infinities_in_their_rows(dev):
    """Rows past a range and values past a row never reach a result, whatever they hold."""
    rng = np.random.default_rng(6)
    for i in (64, 72, 70):
        for transposed in (False, True):
            x, w = _make(rng, (90, i), "bf16", dev, pad=8), _make(rng, (2 * (i if transposed else 40), 40 if transposed else i), "bf16", dev)
            w = w.contiguous().view(2, -1, w.shape[1])
            x[50:] = float("nan")
            x[7, 3] = float("inf")
            at = torch.tensor([0, 30, 50], dtype=torch.int32, device=dev)
            out = L.poseidon_expert_product(x, w, at, transposed=transposed)
            rows = [t for t in range(50) if t != 7]
            assert torch.isfinite(out[rows]).all() and not torch.isfinite(out[7]).any() and not out[50:].any()


# ---- attention ----

def _attention_case(rng, dev, kind, n, heads, kv_heads, dim, layout="joint", spread=1.0):
    """(q, k, v, dout): parts of one product's rows, tensors of their own, head by head, or at odd addresses."""
    t = KIND[kind]
    if layout == "joint":
        rows = torch.from_numpy(rng.normal(size=(n, (heads + 2 * kv_heads) * dim)) * spread).to(dev).to(t)
        q, k, v = (x.view(n, -1, dim) for x in rows.split([heads * dim, kv_heads * dim, kv_heads * dim], dim=1))
    else:
        q, k, v = (torch.from_numpy(rng.normal(size=(n, h, dim)) * spread).to(dev).to(t) for h in (heads, kv_heads, kv_heads))
        if layout == "heads":
            q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
        elif layout == "odd":
            q, k, v = (torch.cat([x.new_zeros(3), x.reshape(-1)])[3:].view(x.shape) for x in (q, k, v))
    return q, k, v, torch.from_numpy(rng.normal(size=(n, heads, dim))).to(dev).to(t)


def _bounds(q, k, v, dout, out, offsets, scale, kind):
    """(slack of out, of lse, of dq, of dk, of dv): p is rounded to `kind` before its products, and so is ds; a score is off by
    `a`, an exponential relatively by a and a few roundings.  The exponential gives 0 for what lies below 2^-126, the least
    normal value in 32 bits, and so do the matrix instructions for such bf16 operands: p and ds are off by that much
    where they are smaller."""
    n, heads, dim = q.shape
    group, r, step = heads // k.shape[1], ROUND[kind], max(STEP[kind], 2.0 ** -126)
    so, sl = np.zeros(q.shape), np.zeros((heads, n))
    sq, sk, sv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)
    for lo, hi in zip(offsets, offsets[1:]):
        if hi <= lo:
            continue
        m = hi - lo
        later = np.triu(np.ones((m, m), bool), 1)
        for h in range(heads):
            j = h // group
            Q, K, X, D, U = q[lo:hi, h], k[lo:hi, j], v[lo:hi, j], dout[lo:hi, h], out[lo:hi, h]
            s = np.where(later, -np.inf, scale * Q @ K.T)
            top = s.max(axis=1, keepdims=True)
            total = np.exp(s - top).sum(axis=1, keepdims=True)
            p = np.exp(s - top) / total
            a = ((dim + 6) * V * abs(scale) * np.abs(Q) @ np.abs(K).T) + 4 * V * (np.abs(np.where(later, 0, s)) + np.abs(top))
            worst = np.where(later, 0, a).max(axis=1, keepdims=True)
            lse = worst + (m + 10) * V + 4 * V * np.abs(top)
            sl[h, lo:hi] = lse[:, 0]
            rel = a + lse + 6 * V                       # of p
            so[lo:hi, h] = ((r + 2 * rel + (m + 8) * V) * p) @ np.abs(X) + step / np.maximum(total, 1) * np.abs(X).sum(axis=0)
            dp = D @ X.T - (D * U).sum(axis=1, keepdims=True)
            edp = (dim + 4) * V * (np.abs(D) @ np.abs(X).T + (np.abs(D) * np.abs(U)).sum(axis=1, keepdims=True))
            ds = p * np.abs(dp)
            eds = np.where(later, 0, (rel + r + (m * group + 8) * V) * (ds + p * edp) + p * edp + step)
            ep = np.where(later, 0, (rel + r + (m * group + 8) * V) * p + step)
            sq[lo:hi, h] = abs(scale) * eds @ np.abs(K)
            sk[lo:hi, j] += abs(scale) * eds.T @ np.abs(Q)
            sv[lo:hi, j] += ep.T @ np.abs(D)
    return so, sl, sq, sk, sv


def _check_attention(dev, q, k, v, dout, offsets, kind, scale=None):
    n, heads, dim = q.shape
    at = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device=dev)
    cuts = [0, n] if offsets is None else offsets
    out, lse = L.poseidon_attention_forward(q, k, v, at, scale=scale)
    dq, dk, dv = L.poseidon_attention_backward(dout, q, k, v, out, lse, at, scale=scale)
    scale = dim ** -0.5 if scale is None else scale
    Q, K, X, D, U = (_np(x) for x in (q, k, v, dout, out))
    want, want_lse = O.attention_forward(Q, K, X, cuts, scale)
    so, sl, sq, sk, sv = _bounds(Q, K, X, D, U, cuts, scale, kind)
    _check(out, want, so, kind)
    inside = np.isfinite(want_lse)
    got = _np(lse)
    assert np.isneginf(got[~inside]).all()
    assert (np.abs(got[inside] - want_lse[inside]) <= sl[inside] + 2 * V * np.abs(want_lse[inside])).all()
    for got, want, slack in zip((dq, dk, dv), O.attention_backward(D, Q, K, X, U, cuts, scale), (sq, sk, sv)):
        _check(got, want, slack, kind)
    return out, lse, dq, dk, dv


LENGTHS = [[0, 1], [0, 1, 2, 3], [0, 0, 5, 5], [0, 64], [0, 65], [2, 129, 256], [0, 130, 130, 131, 200], [3, 3, 33, 97, 160], [0, 300]]


@pytest.mark.parametrize("kind", SHORT)
@pytest.mark.parametrize("offsets", LENGTHS)
@pytest.mark.parametrize("heads, kv_heads, dim", [(1, 1, 64), (2, 2, 128), (6, 2, 72), (4, 1, 8), (3, 3, 120)])
def test_attention(dev, kind, offsets, heads, kv_heads, dim):
    rng = np.random.default_rng(len(offsets) * 100 + offsets[-1] + dim)
    n = offsets[-1] + (5 if len(offsets) > 3 else 0)
    layout = ["joint", "own", "heads", "odd"][(offsets[-1] + heads) % 4]
    q, k, v, dout = _attention_case(rng, dev, kind, n, heads, kv_heads, dim, layout)
    _check_attention(dev, q, k, v, dout, offsets, kind)


@pytest.mark.parametrize("kind", SHORT)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("layout", ["joint", "own", "heads", "odd"])
def test_attention_layouts(dev, kind, dim, layout):
    rng = np.random.default_rng(dim)
    q, k, v, dout = _attention_case(rng, dev, kind, 150, 4, 2, dim, layout)
    _check_attention(dev, q, k, v, dout, None, kind, scale=0.2)


def test_attention_of_sharp_and_of_flat_scores(dev):
    """One key has it all, from anywhere in the row, or all have the same; a negative scale turns them round."""
    rng = np.random.default_rng(4)
    for spread, scale in ((6.0, 0.5), (6.0, -0.5), (1.0, 0.0), (0.01, 1.0)):
        q, k, v, dout = _attention_case(rng, dev, "bf16", 200, 2, 1, 64, spread=spread)
        _check_attention(dev, q, k, v, dout, [0, 200], "bf16", scale=scale)


def test_attention_of_many_sequences(dev):
    """More sequences than two levels of a search hold; with so many blocks a key's heads stay in one."""
    rng = np.random.default_rng(9)
    lengths = rng.integers(0, 3, size=5000)
    offsets = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    n = offsets[-1] + 3
    q, k, v, dout = _attention_case(rng, dev, "bf16", n, 2, 1, 16)
    assert L.lib().poseidon_attention_backward_workspace(n, 2, 1, 16, 5000) == n * 16 + n * 16 * 16   # without offsets: parts
    _check_attention(dev, q, k, v, dout, offsets, "bf16")


def test_attention_of_a_long_sequence(dev):
    """Against the same operator in 64 bits by torch: 3000 tokens, several tiles of each kernel."""
    rng = np.random.default_rng(10)
    n, heads, kv, dim = 3000, 4, 2, 128
    q, k, v, dout = _attention_case(rng, dev, "bf16", n, heads, kv, dim, spread=1.3)
    at = torch.tensor([0, 700, n], dtype=torch.int32, device=dev)
    out, lse = L.poseidon_attention_forward(q, k, v, at)
    got = L.poseidon_attention_backward(dout, q, k, v, out, lse, at)
    Q, K, X = (x.double().detach().requires_grad_() for x in (q, k, v))
    rows = []
    for a, b in ((0, 700), (700, n)):
        later = torch.ones(b - a, b - a, dtype=torch.bool, device=dev).triu(1)
        one = []
        for h in range(heads):
            s = (Q[a:b, h] @ K[a:b, h // 2].t()) * dim ** -0.5
            one.append(torch.softmax(s.masked_fill(later, -float("inf")), 1) @ X[a:b, h // 2])
        rows.append(torch.stack(one, 1))
    want = torch.cat(rows)
    want.backward(dout.double())

    def off(x, y):
        return float((x.double() - y).norm() / y.norm())
    # roundings of 2^-9 of the value at the root mean square each: p and out; p, ds, delta's out and the result
    assert off(out, want.detach()) < 2 * 2.0 ** -9
    assert all(off(x, y.grad) < 3 * 2.0 ** -9 for x, y in zip(got, (Q, K, X)))


def test_attention_keeps_infinities_in_their_sequence(dev):
    rng = np.random.default_rng(11)
    for dim in (64, 128):
        q, k, v, dout = _attention_case(rng, dev, "bf16", 230, 4, 2, dim, "own")
        at = torch.tensor([0, 70, 75, 200], dtype=torch.int32, device=dev)
        clean = L.poseidon_attention_forward(q, k, v, at)
        clean = clean + L.poseidon_attention_backward(dout, q, k, v, *clean, at)
        for x in (q, k, v, dout):
            x[70:75] = float("nan")
            x[200:] = float("inf")
        out, lse = L.poseidon_attention_forward(q, k, v, at)
        got = (out, lse) + L.poseidon_attention_backward(dout, q, k, v, out, lse, at)
        keep = [t for t in range(200) if not 70 <= t < 75]
        for x, y in zip(got, clean):
            if x.dim() == 2:
                x, y = x.t(), y.t()
            _same(x[keep].contiguous(), y[keep].contiguous())
            assert torch.isnan(x[70:75]).any()
            _same(x[200:].contiguous(), y[200:].contiguous())


def test_results_have_the_same_bits_on_every_call(dev):
    rng = np.random.default_rng(12)
    q, k, v, dout = _attention_case(rng, dev, "f16", 700, 8, 2, 64)
    at = torch.tensor([0, 300, 700], dtype=torch.int32, device=dev)
    x, w = _make(rng, (700, 512), "f16", dev), _make(rng, (2 * 96, 512), "f16", dev).contiguous().view(2, 96, 512)

    def run():
        out, lse = L.poseidon_attention_forward(q, k, v, at)
        y = L.poseidon_norm_forward(x, w[0, 0].contiguous(), x, keep_sum=True)
        return (out, lse, *L.poseidon_attention_backward(dout, q, k, v, out, lse, at), L.poseidon_expert_product(x, w, at), y.out,
                *L.poseidon_norm_backward(x, y.kept_sum, y.rstd, w[0, 0].contiguous(), x))
    first = run()
    for _ in range(3):
        for a, b in zip(run(), first):
            _same(a, b)


# ---- addresses, streams, graphs ----

def test_offsets_past_32_bits(dev):
    """Rows more than 2^32 values apart: a token pitch of 2^24 and 300 tokens."""
    n, pitch = 300, 1 << 24
    if torch.cuda.mem_get_info()[0] < (40 << 30):
        pytest.skip("less than 40 GB free")
    rng = np.random.default_rng(13)
    big = torch.empty(n * pitch, dtype=torch.bfloat16, device=dev).view(n, pitch)
    q, k, v, dout = _attention_case(rng, dev, "bf16", n, 2, 1, 64, "own")
    far = [big[:, 64 * i:64 * i + 64 * x.shape[1]].unflatten(1, (x.shape[1], 64)) for i, x in ((0, q), (8, k), (16, v), (24, dout))]
    for x, y in zip(far, (q, k, v, dout)):
        x.copy_(y)
    out, lse = L.poseidon_attention_forward(q, k, v)
    near = L.poseidon_attention_backward(dout, q, k, v, out, lse)
    o2, l2 = L.poseidon_attention_forward(*far[:3], out=big[:, 4096:4096 + 128].unflatten(1, (2, 64)))
    _same(o2.contiguous(), out)
    _same(l2, lse)
    for a, b in zip(L.poseidon_attention_backward(far[3], *far[:3], o2, l2), near):
        _same(a, b)
    x, w = _make(rng, (n, 64), "bf16", dev), _make(rng, (48, 64), "bf16", dev).contiguous()
    big[:, 8192:8256].copy_(x)
    y = L.poseidon_expert_product(x, w)
    _same(L.poseidon_expert_product(big[:, 8192:8256], w, out=big[:, 9000:9048]).contiguous(), y)
    back = L.poseidon_expert_product(y, w, transposed=True)
    _same(L.poseidon_expert_product(big[:, 9000:9048], w, transposed=True), back)
    weight = torch.ones(64, device=dev)
    a, b = L.poseidon_norm_forward(x, weight, keep_sum=True), L.poseidon_norm_forward(big[:, 8192:8256], weight, keep_sum=True)
    _same(a.out, b.out)
    _same(L.poseidon_norm_backward(big[:, 8192:8256], b.kept_sum, b.rstd, weight)[0], L.poseidon_norm_backward(x, a.kept_sum, a.rstd, weight)[0])


def _layer(x, weight, w1, w2, at, heads, stream=None):
    """A layer's parts one after another, forward and backward."""
    n, d = x.shape
    y = L.poseidon_norm_forward(x, weight, x, keep_out=True, keep_sum=True, stream=stream)
    both = L.poseidon_expert_product(y.out, w1, stream=stream)
    q, k, v = (t.view(n, heads, -1) for t in both.split(both.shape[1] // 3, dim=1))
    out, lse = L.poseidon_attention_forward(q, k, v, at, stream=stream)
    z = L.poseidon_expert_product(out.view(n, -1), w2, stream=stream)
    dout = L.poseidon_expert_product(z, w2, transposed=True, stream=stream).view(out.shape)
    dboth = torch.empty_like(both) if stream is None else torch.zeros_like(both)
    parts = [t.view(n, heads, -1) for t in dboth.split(both.shape[1] // 3, dim=1)]
    L.poseidon_attention_backward(dout, q, k, v, out, lse, at, dq=parts[0], dk=parts[1], dv=parts[2], stream=stream)
    dw = L.poseidon_weight_gradient(dboth, y.kept_out, stream=stream)
    dy = L.poseidon_expert_product(dboth, w1, transposed=True, stream=stream)
    dx, dweight = L.poseidon_norm_backward(dy, y.kept_sum, y.rstd, weight, z, stream=stream)
    return z, lse, dw, dx, dweight


def _layer_inputs(rng, dev, n=300, d=128, heads=2):
    x = _make(rng, (n, d), "bf16", dev)
    weight = torch.from_numpy(1 + 0.1 * rng.normal(size=d)).to(dev).bfloat16()
    w1, w2 = (torch.from_numpy(rng.normal(size=s) * d ** -0.5).to(dev).bfloat16() for s in ((3 * d, d), (d, d)))
    return x, weight, w1, w2, torch.tensor([0, 100, n], dtype=torch.int32, device=dev), heads


def test_a_layer_of_them(dev):
    """Norm, product, attention, product and back, against the same layer in 64 bits.  Each of about ten steps rounds to 16
    bits (2^-9 of the value at the root mean square), and what is kept in 8 bits is off by 0.011 of its group's deviation, in two
    places: sqrt(10 * 2^-18 + 2 * 0.011^2) = 0.017, held to 0.05."""
    rng = np.random.default_rng(14)
    x, weight, w1, w2, at, heads = _layer_inputs(rng, dev)
    z, _, dw, dx, dweight = _layer(x, weight, w1, w2, at, heads)
    n, d = x.shape
    X, W, A, B = (t.double().cpu().requires_grad_() for t in (x, weight, w1, w2))
    h = X + X.detach()
    h.retain_grad()
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * W
    q, k, v = (t.view(n, heads, -1) for t in (y @ A.t()).split(d, dim=1))
    rows = []
    for a, b in ((0, 100), (100, n)):
        later = torch.ones(b - a, b - a, dtype=torch.bool).triu(1)
        s = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b]) * (d / heads) ** -0.5
        rows.append(torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(later, -float("inf")), 2), v[a:b]).reshape(b - a, d))
    want = torch.cat(rows) @ B.t()
    want.backward(z.double().cpu())                  # the loss that the layer's backward pass started from

    def off(got, true):
        return float((got.double().cpu() - true).norm() / true.norm())
    assert off(z, want.detach()) < 0.05 and off(dw, A.grad) < 0.05 and off(dweight, W.grad) < 0.05
    assert off(dx, h.grad + z.double().cpu()) < 0.05


def test_capture_and_replay(dev):
    """The layer in a graph, replayed on new inputs with eager work between the replays."""
    rng = np.random.default_rng(15)
    x, weight, w1, w2, at, heads = _layer_inputs(rng, dev)
    _layer(x, weight, w1, w2, at, heads)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _layer(x, weight, w1, w2, at, heads)
    for lengths in ([0, 100, 300], [0, 0, 300], [5, 290, 300], [0, 1, 2]):
        x.copy_(_make(rng, x.shape, "bf16", dev))
        at.copy_(torch.tensor(lengths, dtype=torch.int32))
        want = _layer(x, weight, w1, w2, at, heads)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            _same(a, b)


def test_other_streams(dev):
    """On a stream of the caller's, by argument and as torch's current one."""
    rng = np.random.default_rng(16)
    args = _layer_inputs(rng, dev)
    want = _layer(*args)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for a, b in zip(_layer(*args, stream=stream), want):
        stream.synchronize()
        _same(a, b)
    with torch.cuda.stream(stream):
        got = _layer(*args)
    stream.synchronize()
    for a, b in zip(got, want):
        _same(a, b)
    torch.cuda.synchronize()
    for a, b in zip(_layer(*args, stream=stream.cuda_stream), want):
        stream.synchronize()
        _same(a, b)


def test_threads(dev):
    rng = np.random.default_rng(17)
    inputs = [_layer_inputs(rng, dev, n=200 + 30 * i) for i in range(4)]
    want = [_layer(*args) for args in inputs]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                got = _layer(*inputs[i])
            torch.cuda.current_stream().synchronize()
        return got
    with ThreadPoolExecutor(4) as pool:
        for got, one in zip(pool.map(work, range(4)), want):
            for a, b in zip(got, one):
                _same(a, b)


def test_calls_of_no_rows(dev):
    x, weight = torch.empty(0, 40, dtype=torch.bfloat16, device=dev), torch.ones(40, device=dev)
    y = L.poseidon_norm_forward(x, weight, x, keep_out=True, keep_sum=True)
    assert y.out.shape == y.sum.shape == (0, 40) and y.rstd.shape == (0,)
    dx, dweight = L.poseidon_norm_backward(x, y.kept_sum, y.rstd, weight, x)
    assert dx.shape == (0, 40) and dweight.shape == (40,) and not dweight.any()
    total = torch.full((40,), 3.0, device=dev)
    L.poseidon_norm_backward(x, x, y.rstd, weight, dweight=total, accumulate=True)
    assert (total == 3).all()
    w = torch.ones(2, 24, 40, dtype=torch.bfloat16, device=dev)
    at = torch.zeros(3, dtype=torch.int32, device=dev)
    assert L.poseidon_expert_product(x, w, at).shape == (0, 24)
    h = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=dev)
    out, lse = L.poseidon_attention_forward(h, h, h, at)
    assert out.shape == h.shape and lse.shape == (2, 0)
    assert all(g.shape == h.shape for g in L.poseidon_attention_backward(h, h, h, h, out, lse, at))


def test_refusals_on_the_gpu(dev):
    x, w = torch.zeros(8, 64, dtype=torch.bfloat16, device=dev), torch.zeros(2, 32, 64, dtype=torch.bfloat16, device=dev)
    at, weight = torch.tensor([0, 4, 8], dtype=torch.int32, device=dev), torch.ones(64, device=dev)
    q, k = x.view(8, 4, 16), x[:, :32].reshape(8, 2, 16)
    y = L.poseidon_norm_forward(x, weight, keep_sum=True)
    out, lse = L.poseidon_attention_forward(q, k, k)
    wide = torch.zeros(2, 20000, device=dev)
    refused = [
        lambda: L.poseidon_norm_forward(x, weight[:32]), lambda: L.poseidon_norm_forward(x, weight, x.float()),
        lambda: L.poseidon_norm_forward(x, weight, x[:4]), lambda: L.poseidon_norm_forward(x, weight, eps=-1.0),
        lambda: L.poseidon_norm_forward(x, weight, out=x[:4]), lambda: L.poseidon_norm_forward(wide, torch.ones(20000, device=dev)),
        lambda: L.poseidon_norm_backward(x, y.kept_sum, y.rstd[:4], weight), lambda: L.poseidon_norm_backward(x[:4], y.kept_sum, y.rstd[:4], weight),
        lambda: L.poseidon_norm_backward(x, y.kept_sum, y.rstd, weight, accumulate=True),
        lambda: L.poseidon_norm_backward(x, y.kept_sum, y.rstd, weight, dweight=weight[:32]),
        lambda: L.poseidon_norm_backward(x, y.kept_sum, y.rstd, weight, dweight=weight, weight_gradient=False),
        lambda: L.poseidon_expert_product(x, w), lambda: L.poseidon_expert_product(x, w[0], at), lambda: L.poseidon_expert_product(x.float(), w.float(), at),
        lambda: L.poseidon_expert_product(x, w.half(), at), lambda: L.poseidon_expert_product(x, w, at[:2]), lambda: L.poseidon_expert_product(x, w, at.long()),
        lambda: L.poseidon_expert_product(x, w, at, transposed=True), lambda: L.poseidon_expert_product(x, w, at, dtype=torch.float16),
        lambda: L.poseidon_expert_product(x, w, at, out=x), lambda: L.poseidon_attention_forward(q, k, k[:4]),
        lambda: L.poseidon_attention_forward(q[:, :3], k, k), lambda: L.poseidon_attention_forward(q, k, k.half()),
        lambda: L.poseidon_attention_forward(q.float(), k.float(), k.float()), lambda: L.poseidon_attention_forward(q, k, k, at.long()),
        lambda: L.poseidon_attention_forward(q, k, k, at[:1]), lambda: L.poseidon_attention_forward(x.view(8, 16, 4), x.view(8, 16, 4), x.view(8, 16, 4)),
        lambda: L.poseidon_attention_forward(*[torch.zeros(8, 1, 136, dtype=torch.bfloat16, device=dev)] * 3),
        lambda: L.poseidon_attention_forward(q, k, k, scale=float("nan")), lambda: L.poseidon_attention_forward(q, k, k, out=out[:4]),
        lambda: L.poseidon_attention_forward(q, k, k, out=torch.zeros(8, 4, 17, dtype=torch.bfloat16, device=dev)[:, :, 1:]),
        lambda: L.poseidon_attention_backward(out, q, k, k, out, lse.t()), lambda: L.poseidon_attention_backward(out[:4], q, k, k, out, lse),
        lambda: L.poseidon_attention_backward(out, q, k, k, out, lse, dk=out),
    ]
    for i, f in enumerate(refused):
        with pytest.raises(P.PoseidonError):
            f()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()

"""The layer operators on the GPU against the 64-bit oracle.

Bounds, derived before the first run: ROUND is a rounding to nearest relative to the value (half a unit in the last
place at the lower end of a binade), STEP half of the least step below the normal range, V two roundings in 32 bits.
A sum of n products in 32 bits is off by at most (n + 2) V times the sum of their absolute values, whatever its
order.
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


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def _make(rng, shape, kind, dev, spread=2.0, pad=0, shift=0):
    """Values over a few binades; pad: extra columns of the rows' pitch, shift: values before the first one."""
    n, d = shape
    v = rng.normal(size=shape) * np.exp(rng.normal(size=shape) * spread)
    v = np.clip(v, -2e4, 2e4)
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


def _same(got, want):
    assert np.array_equal(_np(got), want, equal_nan=True)


SHAPES = [(1, 1), (1, 64), (3, 7), (5, 8), (2, 63), (4, 65), (33, 200), (17, 1365), (64, 1024), (700, 130)]
KINDS = ["f32", "f16", "bf16"]


# ---- activations kept in 8 bits ----

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("pad, shift", [(0, 0), (3, 1)])
def test_stash_and_restore(dev, kind, shape, pad, shift):
    x = _make(np.random.default_rng(1), shape, kind, dev, pad=pad, shift=shift)
    s = L.poseidon_stash(x)
    codes, scales = O.stash(_np(x), kind)
    assert np.array_equal(s.codes.cpu().numpy(), codes) and np.array_equal(s.scales.cpu().numpy(), scales)
    want = O.restore(codes, scales, shape[1])
    _same(L.poseidon_restore(s), want)
    _same(L.poseidon_restore(s, dtype=torch.float32), want)
    out = torch.full((shape[0], shape[1] + 5), 7.0, dtype=KIND[kind], device=dev)
    L.poseidon_restore(s, out=out[:, 2:2 + shape[1]])
    _same(out[:, 2:2 + shape[1]], want)
    assert (out[:, :2] == 7).all() and (out[:, 2 + shape[1]:] == 7).all()


@pytest.mark.parametrize("kind", KINDS)
def test_stash_of_extreme_values(dev, kind):
    """Zeros, the largest and smallest values, exact powers and their neighbours, ties, infinities and NaN."""
    info = torch.finfo(KIND[kind])
    rows = torch.zeros(16, 128, dtype=torch.float64)
    rows[1, :] = info.max
    rows[2, :] = -info.max
    rows[3, 0] = info.smallest_normal
    rows[4, 5] = info.smallest_normal * info.eps        # the least value there is
    rows[5, 0], rows[5, 1] = 127.0, 126.5               # the end of a scale's range, a tie
    rows[6, 0], rows[6, 1:8] = 127.5, torch.arange(7) + 0.5
    rows[7, :64] = torch.arange(64) * 0.5 - 16
    rows[8, 3], rows[9, 70], rows[10, 127] = float("inf"), float("-inf"), float("nan")
    rows[11, :] = 1.0
    rows[12, 0], rows[12, 64] = info.max, info.smallest_normal
    rows[13, :] = torch.arange(128) % 2 * -0.0
    rows[14, 0], rows[15, 0] = 2.0 ** -14, 254.0
    x = rows.to(KIND[kind]).to(dev)
    s = L.poseidon_stash(x)
    codes, scales = O.stash(_np(x), kind)
    assert np.array_equal(s.codes.cpu().numpy(), codes) and np.array_equal(s.scales.cpu().numpy(), scales)
    back = L.poseidon_restore(s)
    _same(back, O.restore(codes, scales, 128))
    fine = torch.isfinite(x).view(16, 2, 64).all(2).repeat_interleave(64, 1)
    assert (torch.isfinite(back) == fine).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_gated(dev, kind, shape):
    rng = np.random.default_rng(2)
    n, d = shape
    both = _make(rng, (n, 2 * d), kind, dev, spread=1.0, shift=1)
    gate, up = both[:, :d], both[:, d:]
    dout = _make(rng, shape, kind, dev, spread=1.0, pad=1)
    out, sg, su = L.poseidon_gated_forward(gate, up)
    g, u, w = _np(gate), _np(up), _np(dout)
    want = O.gated_forward(g, u)
    # exp of an argument rounded once: off by |g| 2^-24 relative, as is its share of the sigmoid
    _check(out, want, 8 * V * np.abs(want) * (1 + np.abs(g)), kind)
    assert torch.equal(out, L.poseidon_gated_forward(gate, up, keep=False)[0])
    for s, x in ((sg, g), (su, u)):
        codes, scales = O.stash(x, kind)
        assert np.array_equal(s.codes.cpu().numpy(), codes) and np.array_equal(s.scales.cpu().numpy(), scales)
    g, u = (O.restore(*O.stash(x, kind), d) for x in (g, u))
    dg, du = O.gated_backward(w, g, u)
    a, b = L.poseidon_gated_backward(dout, sg, su)
    s = O.sigmoid(g)
    _check(a, dg, 8 * V * np.abs(w * u * s) * (1 + np.abs(g)) ** 2, kind)
    _check(b, du, 8 * V * np.abs(du) * (1 + np.abs(g)), kind)


@pytest.mark.parametrize("kind", KINDS)
def test_gated_far_below_zero(dev, kind):
    """Gates around -88, where exp(-gate) leaves the range of 32 bits, and far below: silu(gate) is still a normal value there,
    and a large up brings smaller ones back into range.  The bounds of test_gated."""
    big = 2.0 ** 15 if kind == "f16" else 2.0 ** 120
    gates = np.concatenate([np.arange(-70.0, -127.0, -1.0), [-127.0, -60.0, 1.0, 80.0, 127.0]])
    ups = np.array([1.0, -3.0, big, 2.0 ** -10, 1.75 * big])
    g, u = (m.reshape(1, -1) for m in np.meshgrid(gates, ups, indexing="ij"))
    w = np.where(np.arange(g.size) % 2 == 0, 0.75, -big).reshape(1, -1)
    gate, up, dout = (torch.from_numpy(m).to(KIND[kind]).to(dev) for m in (g, u, w))
    # a group of its own for each value, so that what is kept of it is exact
    lone = [torch.zeros(g.size, 64, dtype=KIND[kind], device=dev) for _ in range(3)]
    for m, v in zip(lone, (gate, up, dout)):
        m[:, 5] = v[0]
    top = {"f32": 2.0 ** 128, "f16": 65520.0, "bf16": 2.0 ** 128 * (1 - 2.0 ** -9)}[kind]    # what is rounded to infinity

    def check(got, want, slack):
        fits = (np.abs(want) + slack < top)[0]
        here = torch.from_numpy(fits).to(dev)
        _check(got[:, here], want[:, fits], slack[:, fits], kind)
        assert torch.isinf(got[:, torch.from_numpy((np.abs(want) - slack >= top)[0]).to(dev)]).all()
    out = L.poseidon_gated_forward(gate, up)[0]
    want = O.gated_forward(_np(gate), _np(up))
    check(out, want, 8 * V * np.abs(want) * (1 + np.abs(_np(gate))))
    alone, sg, su = L.poseidon_gated_forward(lone[0], lone[1])
    assert torch.equal(alone[:, 5], out[0]) and alone.count_nonzero() == out.count_nonzero()
    g, u, w = (_np(m)[:, 5:6].T for m in (L.poseidon_restore(sg), L.poseidon_restore(su), lone[2]))
    dg, du = O.gated_backward(w, g, u)
    a, b = L.poseidon_gated_backward(lone[2], sg, su)
    check(a[:, 5:6].t(), dg, 8 * V * np.abs(w * u * O.sigmoid(g)) * (1 + np.abs(g)) ** 2)
    check(b[:, 5:6].t(), du, 8 * V * np.abs(du) * (1 + np.abs(g)))


def test_gated_of_the_lowest_gates(dev):
    """Down to the type's lowest value the product is 0 with its sign; minus infinity gives what the formula gives."""
    x = torch.full((1, 64), 3.0, dtype=torch.float32, device=dev)
    gate = torch.full((1, 64), -1000.5, dtype=torch.float32, device=dev)
    gate[0, 1], gate[0, 2], gate[0, 3] = torch.finfo(torch.float32).min, -400.0, -1e20
    gate[0, 4] = float("-inf")
    up = torch.full_like(gate, torch.finfo(torch.float32).max)
    out = L.poseidon_gated_forward(gate, up)[0]
    assert torch.isnan(out[0, 4]) and out.nan_to_num().count_nonzero() == 0
    gate[0, 4] = -90.0
    _, sg, su = L.poseidon_gated_forward(gate, up)
    a, b = L.poseidon_gated_backward(x, sg, su)
    dg, du = O.gated_backward(_np(x), _np(L.poseidon_restore(sg)), _np(L.poseidon_restore(su)))
    for got, want in ((a, dg), (b, du)):    # the scale of the lowest gate makes the others 0
        assert torch.equal(torch.isinf(got), torch.from_numpy(np.abs(want) > 2.0 ** 128).to(dev)) and not got.isnan().any()


def test_gated_with_infinities(dev):
    """An infinity makes its own output what the formula gives, and its group's gradient NaN; the rest is untouched."""
    x = torch.ones(2, 128, dtype=torch.bfloat16, device=dev)
    gate = x.clone()
    gate[0, 3] = float("inf")
    out, sg, su = L.poseidon_gated_forward(gate, x)
    assert torch.isinf(out[0, 3]) and torch.isfinite(out).sum() == 255
    a, b = L.poseidon_gated_backward(x, sg, su)
    assert torch.isnan(a[0, :64]).all() and torch.isfinite(a).sum() == 192 and torch.isfinite(b).sum() == 192


# ---- weight gradients ----

WIDTHS = [(1, 1), (7, 9), (8, 64), (64, 8), (130, 70), (128, 128), (129, 257), (300, 1365), (1000, 65)]


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("out_kind", KINDS)
@pytest.mark.parametrize("widths", WIDTHS)
@pytest.mark.parametrize("rows", [1, 63, 130, 1100])
def test_weight_gradient(dev, kind, out_kind, widths, rows):
    rng = np.random.default_rng(rows)
    o, i = widths
    dy = _make(rng, (rows, o), kind, dev, spread=0.5, pad=1, shift=1)
    x = _make(rng, (rows, i), kind, dev, spread=0.5)
    s = L.poseidon_stash(x)
    back = O.restore(*O.stash(_np(x), kind), i)
    want = O.weight_gradient(_np(dy), back, [0, rows])[0]
    size = (rows + 2) * V * (np.abs(_np(dy)).T @ np.abs(back))
    got = L.poseidon_weight_gradient(dy, s, dtype=KIND[out_kind])
    _check(got, want, size, out_kind)
    assert torch.equal(got, L.poseidon_weight_gradient(dy, s, dtype=KIND[out_kind]))
    base = _make(rng, (o, i), out_kind, dev, spread=0.5)
    acc = base.clone()
    L.poseidon_weight_gradient(dy, s, out=acc, accumulate=True)
    _check(acc, want + _np(base), size + V * np.abs(_np(base)), out_kind)


RANGES = [[0, 0], [0, 300], [0, 0, 300, 300], [0, 1, 64, 65, 129, 300], [0, 100, 100, 100, 237, 300], [5, 200, 250]]


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("offsets", RANGES)
@pytest.mark.parametrize("widths", [(72, 136), (136, 513)])
def test_weight_gradient_of_ranges(dev, kind, offsets, widths):
    """Ragged ranges, empty ones (zeros), rows outside every range, and NaN rows next to a range, which it must not read."""
    rng = np.random.default_rng(3)
    o, i = widths
    dy, x = _make(rng, (300, o), kind, dev, spread=0.5), _make(rng, (300, i), kind, dev, spread=0.5)
    at = torch.tensor(offsets, dtype=torch.int32, device=dev)
    back = O.restore(*O.stash(_np(x), kind), i)
    want = O.weight_gradient(_np(dy), back, offsets)
    size = np.stack([302 * V * (np.abs(_np(dy)[a:b]).T @ np.abs(back[a:b])) for a, b in zip(offsets, offsets[1:])])
    got = L.poseidon_weight_gradient(dy, L.poseidon_stash(x), offsets=at)
    _check(got, want, size, "f32")
    acc = torch.ones_like(got)
    L.poseidon_weight_gradient(dy, L.poseidon_stash(x), offsets=at, out=acc, accumulate=True)
    _check(acc, want + 1, size + V, "f32")
    for r, (a, b) in enumerate(zip(offsets, offsets[1:])):    # the other ranges' rows spoilt
        dy2, x2 = dy.clone(), x.clone()
        for t in (dy2, x2):
            t[:a] = float("nan")
            t[b:] = float("nan")
        one = L.poseidon_weight_gradient(dy2, L.poseidon_stash(x2), offsets=at)
        assert torch.equal(one[r], got[r])


@pytest.mark.parametrize("rows, offsets", [(300, [0, 300, 0, 300]), (300, [-5, 100, 900, 40]), (20000, [0, 20000, 0, 20000]),
                                           (20000, [0, 64, 19000, 19000, 20000]), (20000, [100, 19900, 19964])])
def test_weight_gradient_of_odd_offsets(dev, rows, offsets):
    """Offsets out of range, out of order or overlapping, and long ranges that are split beside short ones."""
    rng = np.random.default_rng(9)
    dy, x = _make(rng, (rows, 72), "bf16", dev, spread=0.5), _make(rng, (rows, 200), "bf16", dev, spread=0.5)
    s = L.poseidon_stash(x)
    back = L.poseidon_restore(s, dtype=torch.float32).double()
    got = L.poseidon_weight_gradient(dy, s, offsets=torch.tensor(offsets, dtype=torch.int32, device=dev))
    for r, (a, b) in enumerate(zip(offsets, offsets[1:])):
        a, b = min(max(a, 0), rows), min(max(b, 0), rows)
        want = (dy[a:b].double().t().contiguous() @ back[a:b]).cpu().numpy() if b > a else np.zeros((72, 200))
        size = (max(b - a, 0) + 2) * V * (dy[a:b].double().abs().t().contiguous() @ back[a:b].abs()).cpu().numpy() if b > a else 0
        _check(got[r], want, size, "f32")


def test_weight_gradient_of_many_ranges(dev):
    """More ranges than are ordered by length, most of them empty."""
    rng = np.random.default_rng(10)
    ranges, rows = 3000, 2500
    cuts = np.sort(rng.integers(0, rows + 1, size=ranges + 1))
    cuts[0], cuts[-1] = 0, rows
    dy, x = _make(rng, (rows, 8), "f16", dev, spread=0.5), _make(rng, (rows, 24), "f16", dev, spread=0.5)
    got = L.poseidon_weight_gradient(dy, L.poseidon_stash(x), offsets=torch.from_numpy(cuts.astype(np.int32)).to(dev))
    back = O.restore(*O.stash(_np(x), "f16"), 24)
    want = O.weight_gradient(_np(dy), back, cuts)
    _check(got, want, 70 * V * O.weight_gradient(np.abs(_np(dy)), np.abs(back), cuts), "f32")


@pytest.mark.parametrize("ranges", [1, 2, 3, 65, 1023, 1024, 1025])
def test_weight_gradient_of_ranges_in_many_runs(dev, ranges):
    """Long ranges in many runs beside short and empty ones, up to and past the number of runs that are put in order."""
    rng = np.random.default_rng(ranges)
    rows, o, i = 40000, 64, 72
    cuts = np.sort(np.concatenate([[0, rows], rng.integers(0, 700, size=ranges - 1)]))
    g = torch.Generator(device=dev)
    g.manual_seed(ranges)
    dy = torch.randn(rows, o, generator=g, device=dev).bfloat16()
    s = L.poseidon_stash(torch.randn(rows, i, generator=g, device=dev).bfloat16())
    back = L.poseidon_restore(s, dtype=torch.float32).double()
    got = L.poseidon_weight_gradient(dy, s, offsets=torch.from_numpy(cuts.astype(np.int32)).to(dev))
    assert got.shape == (ranges, o, i)
    for r, (a, b) in enumerate(zip(cuts, cuts[1:])):
        left = dy[a:b].double().t().contiguous()
        want, size = left @ back[a:b], (int(b - a) + 2) * V * (left.abs() @ back[a:b].abs())
        assert ((got[r].double() - want).abs() <= size + ROUND["f32"] * want.abs() + STEP["f32"]).all()


def test_weight_gradient_over_tiles_and_splits(dev):
    """Sizes of each tile and of rows in one or more parts, the sums' bound on each; NaN spreads along its row and column
    alone."""
    rng = np.random.default_rng(4)
    for rows, o, i in ((4096, 256, 256), (5000, 257, 383), (2048, 4096, 2048), (700, 4100, 2050), (9000, 64, 64)):
        dy, x = _make(rng, (rows, o), "bf16", dev, 0.5), _make(rng, (rows, i), "bf16", dev, 0.5)
        s = L.poseidon_stash(x)
        back = L.poseidon_restore(s, dtype=torch.float32).double()
        want = (dy.double().t().contiguous() @ back).cpu().numpy()
        size = (rows + 2) * V * (dy.double().abs().t().contiguous() @ back.abs()).cpu().numpy()
        _check(L.poseidon_weight_gradient(dy, s), want, size, "f32")
    dy[100, 3], x[200, 7] = float("nan"), float("inf")
    got = L.poseidon_weight_gradient(dy, L.poseidon_stash(x))
    bad = torch.zeros(64, 64, dtype=torch.bool, device=dev)
    bad[3, :] = True
    bad[:, :64] = True                # the group of the infinity is NaN as a whole
    assert torch.equal(torch.isnan(got), bad)


@pytest.mark.parametrize("out_kind", KINDS)
@pytest.mark.parametrize("rows, o, i, ranges", [(6000, 2040, 1365, 0), (700, 8200, 4099, 0), (12000, 1032, 1030, 24),
                                                (12000, 1024, 1024, 24), (24000, 2040, 2050, 24),
                                                (6000, 2043, 1365, 0), (5000, 2046, 2100, 0), (24000, 2041, 2050, 24),
                                                (9000, 3336, 2049, 0)])
def test_weight_gradient_of_many_large_tiles(dev, out_kind, rows, o, i, ranges):
    """The large tiles at widths that end inside one, with more of them than CUs, alone and added to what is there."""
    g = torch.Generator(device=dev)
    g.manual_seed(rows + i)
    dy = torch.randn(rows, o, generator=g, device=dev).bfloat16()
    s = L.poseidon_stash(torch.randn(rows, i, generator=g, device=dev).bfloat16())
    back = L.poseidon_restore(s, dtype=torch.float32).double()
    cuts = [0, rows]
    if ranges:
        cuts = sorted([0, rows, 1, 65] + torch.randint(0, rows, (ranges - 3,), generator=g, device=dev).tolist())
    at = torch.tensor(cuts, dtype=torch.int32, device=dev) if ranges else None
    got = L.poseidon_weight_gradient(dy, s, offsets=at, dtype=KIND[out_kind])
    acc = torch.full_like(got, 3.0)
    L.poseidon_weight_gradient(dy, s, offsets=at, out=acc, accumulate=True)
    got, acc = got.view(-1, o, i), acc.view(-1, o, i)
    assert got.shape[0] == len(cuts) - 1
    for r, (a, b) in enumerate(zip(cuts, cuts[1:])):
        left = dy[a:b].double().t().contiguous()
        want, size = left @ back[a:b], (b - a + 2) * V * (left.abs() @ back[a:b].abs())
        for have, base in ((got[r], 0.0), (acc[r], 3.0)):
            exact = want + base
            slack = size + V * base
            assert ((have.double() - exact).abs() <= slack + ROUND[out_kind] * (exact.abs() + slack) + STEP[out_kind]).all()


@pytest.mark.parametrize("kind, low, high", [("f16", -24, 10), ("bf16", -133, 100)])
@pytest.mark.parametrize("o", [1, 7, 64])
def test_weight_gradient_of_the_least_values(dev, kind, low, high, o):
    """Gradients below the type's normal range count: every product and sum is exact."""
    dy = torch.full((16, o), 1.0, dtype=torch.float64, device=dev).mul_(2.0 ** low).to(KIND[kind])
    x = torch.full((16, 70), 2.0 ** high, dtype=KIND[kind], device=dev)
    assert (dy != 0).all()
    assert (L.poseidon_weight_gradient(dy, L.poseidon_stash(x)).double() == 16 * 2.0 ** (low + high)).all()


def _brought(x, kind):
    """Kept values x (64 bits) as operands of `kind`: f16 holds what leaves its range to its largest value, and drops what lies
    below its least step."""
    if kind != "f16":
        return x
    x = x.clamp(-65504, 65504)
    return torch.where(x.abs() < 2.0 ** -14, torch.trunc(x * 2.0 ** 24) * 2.0 ** -24, x)


@pytest.mark.parametrize("kind, kept", [("f16", "bf16"), ("f16", "f32"), ("bf16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("o", [72, 67])
def test_weight_gradient_of_rows_kept_from_another_type(dev, kind, kept, o):
    """x over all of its own type's range and beyond f16's, both ends; the sums' bound on the operands as they are defined."""
    rng = np.random.default_rng(11)
    rows, i = 300, 200
    dy, x = _make(rng, (rows, o), kind, dev, spread=0.5), _make(rng, (rows, i), kept, dev, spread=1.0)
    high = 40 if kept != "f16" else 0
    x.mul_(torch.exp2(torch.linspace(-40 if kept != "f16" else -14, high, rows, device=dev)).to(x.dtype).unsqueeze(1))
    s = L.poseidon_stash(x)
    back = _brought(L.poseidon_restore(s, dtype=torch.float32).double(), kind)
    left = dy.double().t().contiguous()
    want, size = (left @ back).cpu().numpy(), (rows + 2) * V * (left.abs() @ back.abs()).cpu().numpy()
    _check(L.poseidon_weight_gradient(dy, s), want, size, "f32")


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("rows, o, i, ranges, pad", [(6000, 2040, 1365, 0, 0), (6000, 2043, 1365, 0, 0), (24000, 2041, 2050, 24, 0),
                                                     (24000, 2040, 2050, 24, 0), (2048, 1408, 1536, 0, 0),
                                                     (2048, 1024, 2048, 0, 0), (6000, 2040, 1365, 0, 1), (2048, 1413, 1536, 0, 1)])
def test_weight_gradient_of_large_calls_by_type(dev, kind, rows, o, i, ranges, pad):
    """Every tile and split in both types, whole and copied dy, and dy on an odd pitch, which no large tile takes."""
    g = torch.Generator(device=dev)
    g.manual_seed(rows + o)
    dy = torch.randn(rows, o + pad, generator=g, device=dev).to(KIND[kind])[:, pad:]
    s = L.poseidon_stash(torch.randn(rows, i, generator=g, device=dev).to(KIND[kind]))
    back = L.poseidon_restore(s, dtype=torch.float32).double()
    cuts = sorted([0, rows, 1, 65] + torch.randint(0, rows, (ranges - 3,), generator=g, device=dev).tolist()) if ranges else [0, rows]
    at = torch.tensor(cuts, dtype=torch.int32, device=dev) if ranges else None
    got = L.poseidon_weight_gradient(dy, s, offsets=at).view(-1, o, i)
    for r, (a, b) in enumerate(zip(cuts, cuts[1:])):
        left = dy[a:b].double().t().contiguous()
        want, size = left @ back[a:b], (b - a + 2) * V * (left.abs() @ back[a:b].abs())
        assert ((got[r].double() - want).abs() <= size + ROUND["f32"] * want.abs() + STEP["f32"]).all()


# ---- experts ----

BATCHES = [(1, 1, 1), (1, 8, 64), (5, 2, 3), (100, 3, 8), (700, 8, 33), (2100, 2, 511), (33000, 4, 256), (300000, 2, 64)]


def _sort64(choice, experts):
    """The oracle's sort, without its lists for long batches."""
    if choice.size < 20000:
        return O.expert_sort(choice, experts)
    key = choice.reshape(-1).astype(np.int64)
    key[(key < 0) | (key >= experts)] = experts
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(experts + 1))
    position = np.full(key.size, -1, np.int64)
    position[order[:offsets[-1]]] = np.arange(offsets[-1])
    return order, position.reshape(choice.shape), offsets


@pytest.mark.parametrize("tokens, k, experts", BATCHES)
@pytest.mark.parametrize("how", ["spread", "dropped", "one", "none"])
def test_expert_sort(dev, tokens, k, experts, how):
    rng = np.random.default_rng(5)
    choice = rng.integers(0, experts, size=(tokens, k))
    if how == "dropped":
        choice = rng.integers(-2, experts + 2, size=(tokens, k))
    if how == "one":
        choice[:] = experts - 1
    if how == "none":
        choice[:] = -1
    plan = L.poseidon_expert_sort(torch.from_numpy(choice.astype(np.int32)).to(dev), experts)
    for got, want in zip((plan.order, plan.position, plan.offsets), _sort64(choice, experts)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_expert_sort_of_nothing(dev):
    plan = L.poseidon_expert_sort(torch.zeros(0, 2, dtype=torch.int32, device=dev), 5)
    assert plan.order.numel() == 0 and (plan.offsets == 0).all()


def test_sort_of_many_blocks(dev):
    """More blocks than add up the counts of the ones before them by themselves."""
    rng = np.random.default_rng(6)
    choice = rng.integers(-1, 300, size=(170000, 4))
    plan = L.poseidon_expert_sort(torch.from_numpy(choice.astype(np.int32)).to(dev), 300)
    for got, want in zip((plan.order, plan.position, plan.offsets), _sort64(choice, 300)):
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens, k, experts, width", [(1, 8, 64, 200), (1, 1, 2, 1), (9, 2, 3, 7), (40, 3, 8, 65),
                                                        (70, 11, 20, 1000), (130, 8, 16, 2056)])
@pytest.mark.parametrize("how", ["all", "dropped", "none"])
def test_experts(dev, kind, tokens, k, experts, width, how):
    rng = np.random.default_rng(7)
    choice = rng.integers(0 if how == "all" else -experts if how == "dropped" else -1, experts if how != "none" else 0,
                          size=(tokens, k))
    order, position, offsets = O.expert_sort(choice, experts)
    plan = L.poseidon_expert_sort(torch.from_numpy(choice.astype(np.int32)).to(dev), experts)
    x = _make(rng, (tokens, width), kind, dev, pad=1, shift=1)
    xs, kept = L.poseidon_expert_gather(x, plan, keep=True)
    want = O.expert_gather(_np(x), position)
    _same(xs, want)
    codes, scales = O.stash(want, kind)
    assert np.array_equal(kept.codes.cpu().numpy(), codes) and np.array_equal(kept.scales.cpu().numpy(), scales)
    assert torch.equal(L.poseidon_expert_gather(x, plan)[0], xs)
    only = L.poseidon_expert_gather(x, plan, keep=True, rows=False)
    assert only[0] is None and torch.equal(only[1].codes, kept.codes) and torch.equal(only[1].scales, kept.scales)

    ys = _make(rng, (tokens * k, width), kind, dev, spread=1.0)
    ys[int(offsets[-1]):] = float("nan")            # places of no choice are not read
    dout = _make(rng, (tokens, width), kind, dev, spread=1.0, pad=3)
    w = torch.from_numpy(rng.uniform(-1, 1, size=(tokens, k)).astype(np.float32)).to(dev)
    y, wn, dn = np.nan_to_num(_np(ys)), _np(w), _np(dout)
    for weights, wv in ((w, wn), (None, np.ones_like(wn))):
        _check(L.poseidon_expert_combine(ys, plan, weights), O.expert_combine(y, position, wv),
               (k + 2) * V * O.expert_combine(np.abs(y), position, np.abs(wv)), kind)
    dys, dw = L.poseidon_expert_combine_backward(dout, ys, plan, w)
    a, b = O.expert_combine_backward(dn, y, position, wn)
    _check(dys, a, V * np.abs(a), kind)
    _check(dw, b, (width + 2) * V * O.expert_combine_backward(np.abs(dn), np.abs(y), position, wn)[1], "f32")


# ---- embedding ----

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out_kind", KINDS)
@pytest.mark.parametrize("tokens, vocab, width", [(1, 1, 1), (1, 100, 64), (3, 2, 7), (50, 1000, 65), (333, 40, 520),
                                                   (5000, 7, 130), (4500, 70000, 24)])
def test_embedding(dev, kind, out_kind, tokens, vocab, width):
    rng = np.random.default_rng(8)
    ids = np.minimum((rng.pareto(0.5, size=tokens)).astype(np.int64), vocab - 1)
    ids[rng.random(tokens) < 0.1] = -1
    ids[rng.random(tokens) < 0.05] = vocab
    at = torch.from_numpy(ids.astype(np.int32)).to(dev)
    table = _make(rng, (vocab, width), kind, dev, pad=1, shift=1)
    dout = _make(rng, (tokens, width), kind, dev, spread=1.0, pad=2)
    want = O.embed(ids, _np(table), 1.25)
    _check(L.poseidon_embed(at, table, 1.25), want, V * np.abs(want), kind)
    dn = _np(dout)
    many = max(1, int(np.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=1).max())) if tokens else 1
    want, size = O.embed_backward(ids, dn, vocab, 1.25), (many + 2) * V * O.embed_backward(ids, np.abs(dn), vocab, 1.25)
    got = L.poseidon_embed_backward(at, dout, vocab, 1.25, dtype=KIND[out_kind])
    _check(got, want, size, out_kind)
    assert torch.equal(got, L.poseidon_embed_backward(at, dout, vocab, 1.25, dtype=KIND[out_kind]))
    base = _make(rng, (vocab, width), out_kind, dev, spread=0.5, pad=1)
    acc = base.clone()
    L.poseidon_embed_backward(at, dout, vocab, 1.25, out=acc, accumulate=True)
    _check(acc, want + _np(base), size + V * np.abs(_np(base)), out_kind)
    rest = np.ones(vocab, bool)
    rest[ids[(ids >= 0) & (ids < vocab)]] = False
    assert np.array_equal(_np(acc)[rest], _np(base)[rest])


@pytest.mark.parametrize("tokens", [8, 9, 4097, 40000])
def test_embedding_gradient_of_one_token(dev, tokens):
    """Every place the same token: its sum crosses every chunk."""
    ids = torch.full((tokens,), 3, dtype=torch.int32, device=dev)
    dout = torch.ones(tokens, 20, dtype=torch.bfloat16, device=dev)
    got = L.poseidon_embed_backward(ids, dout, 5, 0.5)
    assert (got[3] == tokens * 0.5).all() and got.abs().sum() == tokens * 10
    assert (L.poseidon_embed_backward(ids[:0], dout[:0], 5) == 0).all()
    assert (L.poseidon_embed_backward(ids - 9, dout, 5) == 0).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [7, 1000, (1 << 22) + 5, (1 << 23) + 700])
def test_embedding_gradient_into_rows_with_gaps(dev, kind, vocab):
    """Rows of no token become zeros, the gaps between the rows stay: also with more rows than blocks that clear them."""
    wide = torch.full((vocab, 6), 7.0, dtype=KIND[kind], device=dev)
    out = wide[:, 1:4]
    ids = torch.tensor([vocab - 1, 2, -1, vocab - 1, vocab], dtype=torch.int32, device=dev)
    dout = torch.arange(15, device=dev).view(5, 3).to(KIND[kind])
    L.poseidon_embed_backward(ids, dout, vocab, 2.0, out=out)
    assert torch.equal(out[-1], 2 * (dout[0] + dout[3])) and torch.equal(out[2], 2 * dout[1])
    assert out.count_nonzero() == out[-1].count_nonzero() + out[2].count_nonzero()
    assert (wide[:, 0] == 7).all() and (wide[:, 4:] == 7).all()


def test_embedding_gradient_of_a_table_past_32_gib(dev):
    """A table without gaps that takes more than one store a thread to clear."""
    vocab, width = 1 << 23, 1200
    if torch.cuda.mem_get_info(dev)[0] < 60 << 30:
        pytest.skip("not enough memory")
    out = torch.full((vocab, width), 7.0, dtype=torch.float32, device=dev)
    ids = torch.tensor([vocab - 1, 0], dtype=torch.int32, device=dev)
    dout = torch.ones(2, width, dtype=torch.float32, device=dev)
    L.poseidon_embed_backward(ids, dout, vocab, out=out)
    assert (out[-1] == 1).all() and (out[0] == 1).all()
    for a in range(1, vocab - 1, 1 << 20):
        assert not out[a:min(a + (1 << 20), vocab - 1)].any()


def test_calls_of_no_rows(dev):
    """Every operator takes no rows, and writes what depends on none."""
    x, ids = torch.zeros(0, 70, dtype=torch.bfloat16, device=dev), torch.zeros(0, dtype=torch.int32, device=dev)
    s = L.poseidon_stash(x)
    assert L.poseidon_restore(s).shape == (0, 70)
    out, gate, up = L.poseidon_gated_forward(x, x)
    assert out.shape == (0, 70) and all(t.shape == (0, 70) for t in L.poseidon_gated_backward(x, gate, up))
    plan = L.poseidon_expert_sort(ids.view(0, 2), 3)
    w = torch.zeros(0, 2, device=dev)
    xs, kept = L.poseidon_expert_gather(x, plan, keep=True)
    assert xs.shape == (0, 70) and kept.codes.shape == (0, 128) and L.poseidon_expert_combine(xs, plan, w).shape == (0, 70)
    dys, dw = L.poseidon_expert_combine_backward(x, xs, plan, w)
    assert dys.shape == (0, 70) and dw.shape == (0, 2) and L.poseidon_embed(ids, torch.ones(5, 70, device=dev)).shape == (0, 70)
    for offsets, shape in ((None, (70, 70)), (plan.offsets, (3, 70, 70))):
        for value, out in ((0, torch.full(shape, 7.0, device=dev)), (7, torch.full(shape, 7.0, device=dev))):
            L.poseidon_weight_gradient(x, s, offsets=offsets, out=out, accumulate=bool(value))
            assert (out == value).all()


# ---- long calls: the variants that stream, or take several slices a lane or several launches ----

@pytest.mark.parametrize("kind, tokens, width", [("f32", 16301, 1025), ("f32", 40001, 1025), ("bf16", 16301, 1027),
                                                 ("bf16", 70001, 1025), ("f16", 2100003, 3)])
def test_long_lookups(dev, kind, tokens, width):
    """A product of two 32-bit values, rounded to the type, is the same in any order."""
    g = torch.Generator(device=dev)
    g.manual_seed(tokens)
    table = torch.randn(3001, width, generator=g, device=dev).to(KIND[kind])
    ids = torch.randint(-1, 3002, (tokens,), generator=g, device=dev, dtype=torch.int32)
    there = ((ids >= 0) & (ids < 3001)).unsqueeze(1)
    want = torch.where(there, table[ids.clamp(0, 3000).long()].float() * 1.7, torch.zeros((), device=dev)).to(KIND[kind])
    assert torch.equal(L.poseidon_embed(ids, table, 1.7), want)


@pytest.mark.parametrize("kind, width", [("f32", 2501), ("f16", 5003), ("bf16", 5003)])
def test_long_batches_of_experts(dev, kind, width):
    g = torch.Generator(device=dev)
    g.manual_seed(width)
    n, k, e = 9001, 3, 40
    choice = torch.randint(-1, e, (n, k), generator=g, device=dev, dtype=torch.int32)
    plan = L.poseidon_expert_sort(choice, e)
    kept_places, position = int(plan.offsets[-1]), plan.position.long()
    x, dout = (torch.randn(n, width, generator=g, device=dev).to(KIND[kind]) for _ in range(2))
    xs, kept = L.poseidon_expert_gather(x, plan, keep=True)
    want = x[plan.order.long() // k]
    want[kept_places:] = 0
    assert torch.equal(xs, want) and torch.equal(L.poseidon_expert_gather(x, plan)[0], want)
    s = L.poseidon_stash(want)
    assert torch.equal(kept.codes, s.codes) and torch.equal(kept.scales, s.scales)
    ys = torch.randn(n * k, width, generator=g, device=dev).to(KIND[kind])
    ys[kept_places:] = float("nan")
    w = torch.rand(n, k, generator=g, device=dev)
    out, plain = L.poseidon_expert_combine(ys, plan, w), L.poseidon_expert_combine(ys, plan)
    dys, dw = L.poseidon_expert_combine_backward(dout, ys, plan, w)
    rows = torch.where((position >= 0).unsqueeze(2), ys[position.clamp(min=0)], ys.new_zeros(())).double()

    def near(got, want, slack, kind):
        return ((got.double() - want).abs() <= slack + ROUND[kind] * (want.abs() + slack) + STEP[kind]).all()
    for got, by in ((out, w.double()), (plain, torch.ones(n, k, dtype=torch.float64, device=dev))):
        by = by.unsqueeze(2)
        assert near(got, (rows * by).sum(1), (k + 2) * V * (rows * by).abs().sum(1), kind)
    d = dout.double().unsqueeze(1)
    assert near(dw, (rows * d).sum(2), (width + 2) * V * (rows * d).abs().sum(2), "f32")
    flat = plan.order.long()
    want = (w.view(-1)[flat].unsqueeze(1) * dout.float()[flat // k]).to(KIND[kind])    # one product, rounded to the type
    want[kept_places:] = 0
    assert torch.equal(dys, want)


def test_combination_gradient_of_many_places(dev):
    """More places than a launch takes, of one value each: every result is one product."""
    n = (1 << 25) + 3
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    choice = torch.randint(-1, 2, (n, 1), generator=g, device=dev, dtype=torch.int32)
    plan = L.poseidon_expert_sort(choice, 2)
    ys, dout, w = (torch.randn(n, 1, generator=g, device=dev) for _ in range(3))
    dys, dw = L.poseidon_expert_combine_backward(dout, ys, plan, w)
    here, flat = int(plan.offsets[-1]), plan.order.long()
    assert torch.equal(dys[:here], (w * dout)[flat[:here]]) and dys[here:].count_nonzero() == 0
    assert torch.equal(dw, torch.where(plan.position >= 0, dout * ys[plan.position.clamp(min=0).long().view(-1)], torch.zeros((), device=dev)))


@pytest.mark.parametrize("kind, vocab, width", [("bf16", 1000, 230), ("f32", 70000, 120)])
def test_embedding_gradient_of_many_tokens(dev, kind, vocab, width):
    """Two passes of the sort over more blocks than add up the counts before them, beside a clear in parts."""
    tokens = 600001
    g = torch.Generator(device=dev)
    g.manual_seed(vocab)
    ids = torch.randint(-1, vocab + 1, (tokens,), generator=g, device=dev, dtype=torch.int32)
    ids[torch.rand(tokens, generator=g, device=dev) < 0.3] = vocab - 7      # a frequent one
    dout = torch.randn(tokens, width, generator=g, device=dev).to(KIND[kind])
    got = L.poseidon_embed_backward(ids, dout, vocab, 1.25, out=torch.full((vocab, width), 7.0, device=dev))
    assert torch.equal(got, L.poseidon_embed_backward(ids, dout, vocab, 1.25))
    fine = (ids >= 0) & (ids < vocab)
    at = ids[fine].long()

    def sums(rows):
        return torch.zeros(vocab, width, dtype=torch.float64, device=dev).index_add_(0, at, rows)
    d = dout[fine].double() * 1.25
    want, size = sums(d), (torch.bincount(at, minlength=vocab).unsqueeze(1) + 2) * V * sums(d.abs())
    assert ((got.double() - want).abs() <= size + ROUND["f32"] * want.abs()).all()


# ---- addresses, streams, graphs ----

def test_offsets_past_32_bits(dev):
    """More than 2^32 values in a matrix: the last rows are the right ones."""
    rows, width = 70001, 65536
    x = torch.zeros(rows, width, dtype=torch.bfloat16, device=dev)
    tail = torch.randn(3, width, device=dev).bfloat16()
    x[-3:] = tail
    s, few = L.poseidon_stash(x), L.poseidon_stash(tail)
    assert torch.equal(s.codes[-3:], few.codes) and torch.equal(s.scales[-3:], few.scales)
    back = L.poseidon_restore(s)
    assert torch.equal(back[-3:], L.poseidon_restore(few)) and back[:-3].count_nonzero() == 0
    del back
    out, sg, su = L.poseidon_gated_forward(x, x)
    a, b = L.poseidon_gated_forward(tail, tail)[:2]
    assert torch.equal(out[-3:], a) and torch.equal(sg.codes[-3:], b.codes)
    del out, sg, su
    ids = torch.tensor([rows - 1, 0, rows - 2], dtype=torch.int32, device=dev)
    assert torch.equal(L.poseidon_embed(ids, x)[0], tail[2])
    L.poseidon_embed_backward(ids, tail, rows, out=x, accumulate=True)
    assert torch.equal(x[-1], tail[2] + tail[0]) and torch.equal(x[-2], tail[1] + tail[2]) and torch.equal(x[0], tail[1])
    # a weight gradient whose last rows lie past 2^32 codes: 62 zero rows and the last three
    offsets = torch.tensor([rows - 65, rows], dtype=torch.int32, device=dev)
    dy = torch.zeros(rows, 8, dtype=torch.bfloat16, device=dev)
    dy[-3:] = 1.0
    grad = L.poseidon_weight_gradient(dy, s, offsets=offsets)
    want = L.poseidon_restore(few, dtype=torch.float32).double().sum(0)
    assert (grad[0].double() - want).abs().max() <= 8 * V * L.poseidon_restore(few).double().abs().sum(0).max()


def _block(x, ids, table, choice, weights, experts):
    """A small block: embed, sort, gather and keep, gated activation, combine, and everything back."""
    h = L.poseidon_embed(ids, table, 2.0)
    plan = L.poseidon_expert_sort(choice, experts)
    xs, kept = L.poseidon_expert_gather(h + x, plan, keep=True)
    a, g, u = L.poseidon_gated_forward(xs, xs)
    y = L.poseidon_expert_combine(a, plan, weights)
    dys, dw = L.poseidon_expert_combine_backward(y, a, plan, weights)
    dg, du = L.poseidon_gated_backward(dys, g, u)
    grad = L.poseidon_weight_gradient(dg, kept, offsets=plan.offsets)
    dx = L.poseidon_expert_combine(du, plan)
    return [h, plan.order, xs, a, y, dys, dw, dg, du, grad, dx, L.poseidon_embed_backward(ids, dx, table.shape[0], 2.0),
            L.poseidon_restore(kept)]


def _block_inputs(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    n, d, k, e, v = 200, 136, 2, 6, 50
    return (torch.randn(n, d, generator=g, device=dev).bfloat16(),
            torch.randint(-1, v, (n,), generator=g, device=dev, dtype=torch.int32),
            torch.randn(v, d, generator=g, device=dev).bfloat16(),
            torch.randint(-1, e, (n, k), generator=g, device=dev, dtype=torch.int32),
            torch.rand(n, k, generator=g, device=dev), e)


def test_other_streams(dev):
    """On a stream of its own, named or current, with inputs made on another: the same bits."""
    args = _block_inputs(dev, 1)
    want = _block(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _block(*args)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for stream in (side, side.cuda_stream, 0):
        s = L.poseidon_stash(args[0], stream=stream)
        back = L.poseidon_restore(s, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(back, L.poseidon_restore(L.poseidon_stash(args[0])))


def _with_workspaces(x, ids, choice, e, **kw):
    """The operators that bring a workspace of their own."""
    plan = L.poseidon_expert_sort(choice, e, **kw)
    kept = L.poseidon_stash(x, **kw)
    half = torch.tensor([0, x.shape[0] // 3, x.shape[0]], dtype=torch.int32, device=x.device)
    return [plan.order, plan.position, plan.offsets, L.poseidon_weight_gradient(x, kept, **kw),
            L.poseidon_weight_gradient(x, kept, offsets=half, **kw), L.poseidon_embed_backward(ids, x, 50, 2.0, **kw)]


def _long_inputs(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    n = 9000
    return (torch.randn(n, 136, generator=g, device=dev).bfloat16(),
            torch.randint(-1, 50, (n,), generator=g, device=dev, dtype=torch.int32),
            torch.randint(-1, 6, (n, 2), generator=g, device=dev, dtype=torch.int32), 6)


def test_workspaces_on_named_streams(dev):
    """Two streams at once, each call with a workspace that belongs to its stream."""
    batches = [_long_inputs(dev, seed) for seed in (1, 2)]
    want = [_with_workspaces(*b) for b in batches]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in batches]
    for _ in range(3):
        got = [_with_workspaces(*b, stream=s) for b, s in zip(batches, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_threads(dev):
    """Calls from several threads, each with a stream of its own, give what they give alone."""
    batches = [_long_inputs(dev, seed) for seed in range(4)]
    want = [_with_workspaces(*b) for b in batches]
    torch.cuda.synchronize()

    def work(batch):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            got = [_with_workspaces(*batch) for _ in range(5)]
        stream.synchronize()
        return got
    with ThreadPoolExecutor(max_workers=4) as pool:
        results = list(pool.map(work, batches))
    for got, w in zip(results, want):
        assert all(torch.equal(x, y) for one in got for x, y in zip(one, w))


def test_capture_and_replay(dev):
    """The block in a graph, replayed on new inputs with eager work between the replays."""
    args = _block_inputs(dev, 2)
    _block(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _block(*args)
    for seed in (3, 4, 5):
        new = _block_inputs(dev, seed)
        for a, b in zip(args[:5], new[:5]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, _block(*new)):
            assert torch.equal(a, b)


def test_refusals_on_the_gpu(dev):
    """Shapes, types and layouts that do not fit each other."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device=dev)
    s = L.poseidon_stash(x)
    plan = L.poseidon_expert_sort(torch.zeros(4, 2, dtype=torch.int32, device=dev), 2)
    w = torch.zeros(4, 2, device=dev)
    ids = torch.zeros(4, dtype=torch.int32, device=dev)
    calls = [
        lambda: L.poseidon_stash(x[0]), lambda: L.poseidon_stash(x.double()), lambda: L.poseidon_stash(x[:, :0]),
        lambda: L.poseidon_restore(s, dtype=torch.int8), lambda: L.poseidon_restore(s, out=x[:3]),
        lambda: L.poseidon_gated_forward(x, x[:3]), lambda: L.poseidon_gated_forward(x, x.half()),
        lambda: L.poseidon_gated_backward(x[:3], s, s), lambda: L.poseidon_weight_gradient(x.float(), s),
        lambda: L.poseidon_weight_gradient(x[:3], s), lambda: L.poseidon_weight_gradient(x, s, accumulate=True),
        lambda: L.poseidon_weight_gradient(x, s, offsets=ids.long()),
        lambda: L.poseidon_weight_gradient(x, s, out=torch.zeros(64, 128, device=dev)[:, ::2]),
        lambda: L.poseidon_expert_sort(ids, 2), lambda: L.poseidon_expert_sort(ids.view(2, 2).long(), 2),
        lambda: L.poseidon_expert_sort(ids.view(2, 2), 0), lambda: L.poseidon_expert_sort(ids.view(2, 2), 512),
        lambda: L.poseidon_expert_gather(x[:3], plan), lambda: L.poseidon_expert_gather(x, plan, rows=False),
        lambda: L.poseidon_expert_combine(x, plan, w), lambda: L.poseidon_expert_combine_backward(x, x, plan, w),
        lambda: L.poseidon_embed(ids.long(), x), lambda: L.poseidon_embed(ids.cpu(), x),
        lambda: L.poseidon_embed_backward(ids[:3], x, 8), lambda: L.poseidon_embed_backward(ids, x, 8, accumulate=True),
    ]
    for f in calls:
        with pytest.raises(P.PoseidonError) as ei:
            f()
        assert ei.value.status in (P.POSEIDON_E_INVAL, P.POSEIDON_E_RANGE)


def test_layouts_that_are_copied(dev):
    """Transposed, broadcast and strided inputs give what their copies give."""
    x = torch.randn(96, 80, device=dev).bfloat16()
    for view in (x.t(), x[:, ::2], x[:1].expand(40, 80), x[::3], x[5:6, 3:]):
        s, c = L.poseidon_stash(view), L.poseidon_stash(view.contiguous())
        assert torch.equal(s.codes, c.codes) and torch.equal(s.scales, c.scales)

"""Attention's gradients in f16 where p and ds lie outside of what f16 holds well: small and large gradients, and keys that get
little of a row.

Bounds, derived before the first run: a rounding is 2^-12 of the value at the root mean square (half a unit of 2^-10 at most, a
binade's mean below that), and what a gradient depends on is rounded three times on its way: p or ds, delta's out, the result,
which below 2^-14 is off by up to 2^-25 besides.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_06086_amd import layers as L  # noqa: E402
from test_gpu_transformer import _check_attention, dev  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def _gradients64(q, k, v, dout, scale):
    """One sequence in 64 bits, a head at a time."""
    Q, K, X = (x.double().detach().requires_grad_() for x in (q, k, v))
    n, heads = q.shape[:2]
    group = heads // k.shape[1]
    later = torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1)
    rows = []
    for h in range(heads):
        s = (Q[:, h] @ K[:, h // group].t().contiguous()) * scale
        rows.append(torch.softmax(s.masked_fill(later, -float("inf")), 1) @ X[:, h // group])
    torch.stack(rows, 1).backward(dout.double())
    return Q.grad, K.grad, X.grad


def _near(got, want):
    off = float((got.double() - want).norm())
    assert off <= 3 * 2.0 ** -12 * float(want.norm()) + 2.0 ** -25 * want.numel() ** 0.5, (off, float(want.norm()))


def _case(dev, n, heads, kv, dim, dout):  # noqa: F811
    g = torch.Generator(device=dev)
    g.manual_seed(n + dim)
    q, k = (torch.randn(n, h, dim, generator=g, device=dev) * dim ** -0.25 for h in (heads, kv))
    v, d = torch.randn(n, kv, dim, generator=g, device=dev), torch.randn(n, heads, dim, generator=g, device=dev) * dout
    return [x.half() for x in (q, k, v, d)]


@pytest.mark.parametrize("heads, kv, dim", [(2, 1, 128), (4, 2, 64), (3, 3, 72)])
@pytest.mark.parametrize("spread", [1.0, 1e-3, 1e-4])
def test_small_gradients(dev, spread, heads, kv, dim):  # noqa: F811
    """ds down to 2^-30, where f16's least value is 2^-24."""
    q, k, v, dout = _case(dev, 2048, heads, kv, dim, spread)
    out, lse = L.poseidon_attention_forward(q, k, v, scale=1.0)
    got = L.poseidon_attention_backward(dout, q, k, v, out, lse, scale=1.0)
    for x, want in zip(got, _gradients64(q, k, v, dout, 1.0)):
        _near(x, want)


@pytest.mark.parametrize("heads, kv, dim", [(2, 1, 128), (3, 1, 64)])
def test_keys_that_get_little(dev, heads, kv, dim):  # noqa: F811
    """The first key has all but a few millionths of every row; the gradients of the others' values are held as well."""
    q, k, v, dout = _case(dev, 1500, heads, kv, dim, 1.0)
    q[:, :, 0], k[:, :, 0], k[0, :, 0] = 4, 0, 3
    out, lse = L.poseidon_attention_forward(q, k, v, scale=1.0)
    got = L.poseidon_attention_backward(dout, q, k, v, out, lse, scale=1.0)[2]
    want = _gradients64(q, k, v, dout, 1.0)[2]
    _near(got[:1], want[:1])
    _near(got[1:], want[1:])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [3, 40, 200])
def test_large_gradients(dev, n, dim):  # noqa: F811
    """ds above 65504, the largest value of f16, where the gradients are far below it."""
    rng = np.random.default_rng(n + dim)
    q, k, v, dout = (torch.from_numpy(rng.normal(size=(n, h, dim)) * spread).to(dev).half()
                     for h, spread in ((4, 0.01), (2, 0.01), (2, 200.0), (4, 200.0)))
    got = _check_attention(dev, q, k, v, dout, [0, n], "f16", scale=0.1)
    assert all(torch.isfinite(x).all() for x in got)
    dp = (dout[:, 0].double() @ v[:, 0].double().t().contiguous()).abs().max()
    assert dp / n > 65504 or n > 3                # the case is what it is meant to be
    for spread in (1e-5, 1.0):                    # a tile of small ones before it, or after
        some = dout.clone()
        some[n // 2:] *= spread
        some[:n // 2] *= 1e-5 / spread
        _check_attention(dev, q, k, v, some, [0, n], "f16", scale=0.1)

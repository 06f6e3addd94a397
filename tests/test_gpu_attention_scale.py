"""Attention's scale: the largest ones, and those past 2^127 refused (their base-2 exponents leave 32 bits)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_06086_amd import layers as L  # noqa: E402
from paper_2609_06086_amd import poseidon as P  # noqa: E402
from oracle import layers as O  # noqa: E402
from test_gpu_transformer import _bounds, _check, _np, dev  # noqa: E402, F401
from test_transformer_cpu import AB, AF, _good  # noqa: E402


@pytest.mark.parametrize("name, at", [(AF, 14), (AB, 21)])
@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 2.0 ** 127 * (1 + 2.0 ** -23)])
def test_scales_past_the_largest(name, at, scale):
    args = _good()[name]
    args[at] = scale
    assert getattr(L.lib(), name)(*args) == P.POSEIDON_E_RANGE


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [2.0 ** 127, -2.0 ** 127, 2.0 ** -120])
def test_the_largest_and_a_small_scale(dev, scale):  # noqa: F811
    """Scores of 64 to 256 (of almost none for the small scale) from one product of q and k each, far from order 1 themselves."""
    rng = np.random.default_rng(21)
    n, power = 70, 2.0 ** -60 if abs(scale) > 1 else 1.0
    q, k = (np.zeros((n, h, 64)) for h in (2, 1))
    q[:, :, 5], k[:, :, 5] = rng.uniform(1, 2, size=(n, 2)) * power, rng.uniform(1, 2, size=(n, 1)) * power / 2
    v, dout = rng.normal(size=(n, 1, 64)), rng.normal(size=(n, 2, 64))
    q, k, v, dout = (torch.from_numpy(x).to(dev).bfloat16() for x in (q, k, v, dout))
    out, lse = L.poseidon_attention_forward(q, k, v, scale=scale)
    got = (out, *L.poseidon_attention_backward(dout, q, k, v, out, lse, scale=scale))
    assert all(torch.isfinite(x).all() for x in (lse, *got))
    q, k, v, dout, out = (_np(x) for x in (q, k, v, dout, out))
    bounds = _bounds(q, k, v, dout, out, [0, n], scale, "bf16")
    want, want_lse = O.attention_forward(q, k, v, [0, n], scale)
    assert (np.abs(_np(lse) - want_lse) <= bounds[1] + 2.0 ** -22 * np.abs(want_lse)).all()
    # Sums of ds k and ds q lie before `scale` stretches them: each of up to 2 n products of 16-bit values, and each sum on the
    # way, counts as 0 below 2^-126, the least normal value in 32 bits.  Of gradients of 2^67 that is 2^-58.
    lost = 4 * n * 2.0 ** -126 * abs(scale)
    for x, y, slack, least in zip(got, (want, *O.attention_backward(dout, q, k, v, out, [0, n], scale)), (bounds[0], *bounds[2:]),
                                  (0, lost, lost, 0)):
        _check(x, y, slack + least, "bf16")

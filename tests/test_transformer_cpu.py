"""Norm, products by expert and attention on the CPU: refusals before any GPU call, workspaces, and the oracle's gradients
against differences of its forward functions."""
import os
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layers as O  # noqa: E402
from paper_2609_06086_amd import layers as L  # noqa: E402
from paper_2609_06086_amd import poseidon as P  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "poseidon_layers.h")).read()
BAD, BIG, NONE = P.POSEIDON_E_INVAL, P.POSEIDON_E_RANGE, 2 ** 64 - 1
A = 1 << 20    # an aligned address that no refused call reads
NAN, INF = float("nan"), float("inf")


def test_limits_match_the_header():
    for name in ("NORM_WIDTH_MAX", "HEAD_MAX", "HEADS_MAX"):
        assert int(re.search(rf"#define POSEIDON_{name} (\d+)u", HEADER).group(1)) == getattr(L, name)


def _good():
    """Arguments that pass every check, by operator; a refusal changes one of them."""
    heads = [A, 32, 8]
    return {
        "poseidon_norm_forward": [A, 8, A, 8, 2, 4, 8, A, 0, 1e-6, A, 8, A, 8, A, A, A, A, A, None],
        "poseidon_norm_backward": [A, 8, 2, 4, 8, None, 0, A, A, A, A, 0, A, 8, A, 8, A, 0, A, 1 << 20, None],
        "poseidon_expert_product": [A, 8, 2, 4, A, 16, 8, 0, A, 3, A, 16, 2, None],
        "poseidon_attention_forward": heads * 3 + [2, 16, 4, 2, 8, 0.5, A, 2] + heads + [A, None],
        "poseidon_attention_backward": heads * 5 + [A, 2, 16, 4, 2, 8, 0.5, A, 2] + heads * 3 + [A, 1 << 20, None],
    }


F, B, X, AF, AB = _good()
REFUSED = [
    # null pointers
    *[(F, i, None, BAD) for i in (0, 7, 15, 16, 17, 18)], *[(B, i, None, BAD) for i in (0, 7, 8, 9, 10, 14, 18)],
    *[(X, i, None, BAD) for i in (0, 4, 8, 10)], *[(AF, i, None, BAD) for i in (0, 3, 6, 15, 17, 20)],
    *[(AB, i, None, BAD) for i in (0, 3, 6, 9, 12, 15, 22, 24, 27, 30, 33)],
    (B, 5, A, BAD),                                      # the sum as it is and in 8 bits
    # types: unknown ones, 32 bits for the matrix instructions, an output of another 16-bit type
    (F, 4, 3, BAD), (F, 8, 3, BAD), (B, 2, 3, BAD), (B, 11, 3, BAD), (X, 2, 0, BAD), (X, 2, 3, BAD), (X, 12, 1, BAD),
    (X, 12, 3, BAD), (AF, 9, 0, BAD), (AF, 9, 3, BAD), (AB, 16, 0, BAD), (AB, 16, 3, BAD),
    # widths of 0, pitches below the width, addresses and pitches off their boundaries
    (F, 6, 0, BAD), (F, 1, 7, BAD), (F, 3, 7, BAD), (F, 11, 7, BAD), (F, 13, 7, BAD), (F, 0, A + 1, BAD), (F, 15, A + 8, BAD),
    (F, 17, A + 8, BAD), (F, 14, A + 2, BAD), (B, 4, 0, BAD), (B, 1, 7, BAD), (B, 13, 7, BAD), (B, 15, 7, BAD), (B, 9, A + 2, BAD),
    (B, 16, A + 2, BAD), (B, 18, A + 128, BAD), (B, 19, 8, BAD), (X, 5, 0, BAD), (X, 6, 0, BAD), (X, 1, 7, BAD), (X, 11, 15, BAD),
    (X, 0, A + 1, BAD), (X, 8, A + 2, BAD), (AF, 1, 0, BAD), (AF, 1, 36, BAD), (AF, 2, 4, BAD), (AF, 5, 0, BAD), (AF, 0, A + 8, BAD),
    (AF, 6, A + 2, BAD), (AF, 15, A + 2, BAD), (AF, 17, A + 8, BAD), (AF, 20, A + 2, BAD), (AB, 1, 12, BAD), (AB, 13, 0, BAD),
    (AB, 24, A + 8, BAD), (AB, 28, 4, BAD), (AB, 33, A + 16, BAD), (AB, 34, 16, BAD),
    # flags, counts, what is no number
    (F, 9, -1.0, BAD), (F, 9, NAN, BAD), (F, 9, INF, BAD), (B, 17, 2, BAD), (X, 7, 2, BAD), (X, 9, 0, BAD), (AF, 11, 0, BAD),
    (AF, 12, 0, BAD), (AF, 12, 3, BAD), (AF, 13, 0, BAD), (AF, 13, 12, BAD), (AF, 14, NAN, BAD), (AF, 14, INF, BAD), (AF, 16, 0, BAD),
    (AB, 18, 0, BAD), (AB, 19, 3, BAD), (AB, 20, 4, BAD), (AB, 21, NAN, BAD), (AB, 23, 0, BAD),
    # sizes above the limits
    (F, 5, 1 << 31, BIG), (F, 6, 16385, BIG), (F, 1, 1 << 33, BIG), (B, 3, 1 << 31, BIG), (B, 4, 16385, BIG), (X, 3, 1 << 31, BIG),
    (X, 5, 1 << 21, BIG), (X, 6, 1 << 21, BIG), (X, 9, 512, BIG), (X, 11, 1 << 25, BIG), (AF, 10, 1 << 31, BIG), (AF, 13, 136, BIG),
    (AF, 11, 2048, BIG), (AF, 1, 1 << 25, BIG), (AF, 16, 1 << 31, BIG), (AB, 17, 1 << 31, BIG), (AB, 20, 256, BIG),
]


@pytest.mark.parametrize("name, at, value, status", REFUSED)
def test_refusals(name, at, value, status):
    args = _good()[name]
    args[at] = value
    assert getattr(L.lib(), name)(*args) == status


def test_one_range_without_offsets_only():
    lib, good = L.lib(), _good()
    args = good[X]
    args[8], args[9] = None, 2
    assert lib.poseidon_expert_product(*args) == BAD
    args = good[AF]
    args[15], args[16] = None, 2
    assert lib.poseidon_attention_forward(*args) == BAD


def test_a_norm_without_any_output_is_refused():
    args = _good()[F]
    args[10] = args[15] = args[16] = None
    assert L.lib().poseidon_norm_forward(*args) == BAD


def test_empty_calls_need_no_buffers():
    lib, no = L.lib(), [None, 8, 8]
    assert lib.poseidon_norm_forward(None, 8, None, 8, 2, 0, 8, None, 0, 1e-6, None, 8, None, 8, None, None, None, None, None,
                                     None) == P.POSEIDON_OK
    assert lib.poseidon_norm_backward(None, 8, 2, 0, 8, None, 0, None, None, None, None, 0, None, 8, None, 8, None, 0, None, 0,
                                      None) == P.POSEIDON_OK
    assert lib.poseidon_expert_product(None, 8, 2, 0, None, 16, 8, 0, None, 3 - 2, None, 16, 2, None) == P.POSEIDON_OK
    assert lib.poseidon_attention_forward(*no * 3, 2, 0, 1, 1, 8, 0.5, None, 1, *no, None, None) == P.POSEIDON_OK
    assert lib.poseidon_attention_backward(*no * 5, None, 2, 0, 1, 1, 8, 0.5, None, 1, *no * 3, None, 0, None) == P.POSEIDON_OK


def test_workspaces():
    lib = L.lib()
    norm, attention = lib.poseidon_norm_backward_workspace, lib.poseidon_attention_backward_workspace
    assert norm(0, 64) == 0 and norm(1, 64) == 64 * 4 and norm(1 << 31, 64) == NONE and norm(64, 16385) == NONE
    assert norm((1 << 31) - 1, 16384) == 256 * 16384 * 4
    assert attention(1 << 31, 8, 8, 64, 1) == NONE and attention(64, 8, 3, 64, 1) == NONE and attention(64, 8, 8, 136, 1) == NONE
    assert attention(0, 8, 8, 64, 1) == 0
    assert attention(1000, 8, 8, 64, 1) == 1000 * 8 * 8        # every head has keys of its own: no parts
    assert attention(1000, 8, 2, 64, 1) == 1000 * 8 * 8 + 4 * 1000 * 2 * 64 * 8


def test_the_workspace_of_an_attention_is_bounded():
    """Parts of the heads that share a key take at most 1 GB, and calls without offsets fit the workspace of any number of
    sequences."""
    f, rng = L.lib().poseidon_attention_backward_workspace, np.random.default_rng(0)
    for _ in range(5000):
        kv, group, dim = int(2 ** rng.uniform(0, 5)), int(2 ** rng.uniform(0, 5)), 8 * int(rng.integers(1, 17))
        tokens, sequences = int(2 ** rng.uniform(0, 30)), int(2 ** rng.uniform(0, 20))
        need = f(tokens, kv * group, kv, dim, sequences)
        assert tokens * kv * group * 8 <= need <= tokens * kv * group * 8 + (1 << 30)
        assert need >= f(tokens, kv * group, kv, dim, 1) or sequences > 1 and need == f(tokens, kv * group, kv, dim, sequences)


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(2, 32, 64, dtype=torch.bfloat16)
    h, v = x.view(4, 1, 64), torch.zeros(4)
    for f, args in ((L.poseidon_norm_forward, (x, x[0])), (L.poseidon_norm_backward, (x, x, v, x[0])),
                    (L.poseidon_expert_product, (x, w, torch.zeros(3, dtype=torch.int32))),
                    (L.poseidon_attention_forward, (h, h, h)), (L.poseidon_attention_backward, (h, h, h, h, h, v.view(1, 4)))):
        with pytest.raises(P.PoseidonError) as ei:
            f(*args)
        assert ei.value.status == BAD


def _difference(f, h=1e-6):
    return (f(h) - f(-h)) / (2 * h)


def test_gradients_against_differences():
    """Central differences of step 1e-6 on functions of order 1 to 10: an error of about 1e-11 / 1e-6, held to 1e-6."""
    rng = np.random.default_rng(1)
    n, d = 7, 5
    x, r, dx, w, dsum = rng.normal(size=(5, n, d))
    weight, dweight = rng.normal(size=(2, d))

    def loss(t):
        out, h, _ = O.norm_forward(x + t * dx, r, weight + t * dweight, 1e-3)
        return (w * out).sum() + (dsum * h).sum()
    _, h, rstd = O.norm_forward(x, r, weight, 1e-3)
    a, b = O.norm_backward(w, h, rstd, weight, dsum)
    assert abs((a * dx).sum() + (b * dweight).sum() - _difference(loss)) < 1e-6

    W, offsets = rng.normal(size=(2, 6, d)), [1, 3, n]
    dy = rng.normal(size=(n, 6))
    want = _difference(lambda t: (dy * O.expert_product(x + t * dx, W, offsets, False)).sum())
    assert abs((O.expert_product(dy, W, offsets, True) * dx).sum() - want) < 1e-6

    heads, kv, dim, cuts = 4, 2, 3, [0, 4, 4, 6]
    q, tq, dout = rng.normal(size=(3, n, heads, dim))
    k, v, tk, tv = rng.normal(size=(4, n, kv, dim))

    def attended(t):
        return (dout * O.attention_forward(q + t * tq, k + t * tk, v + t * tv, cuts, 0.7)[0]).sum()
    out, lse = O.attention_forward(q, k, v, cuts, 0.7)
    assert np.isneginf(lse[:, 6]).all() and not out[6].any()
    dq, dk, dv = O.attention_backward(dout, q, k, v, out, cuts, 0.7)
    assert abs((dq * tq).sum() + (dk * tk).sum() + (dv * tv).sum() - _difference(attended)) < 1e-6

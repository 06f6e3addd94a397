"""The layer operators on the CPU: the library exports them and refuses bad arguments before any GPU call, and the
oracle's gradients agree with differences of its forward functions."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layers as O  # noqa: E402
from paper_2609_06086_amd import layers as L  # noqa: E402
from paper_2609_06086_amd import poseidon as P  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = open(os.path.join(ROOT, "include", "poseidon_layers.h")).read()
BAD, BIG = P.POSEIDON_E_INVAL, P.POSEIDON_E_RANGE


def test_library_exports_every_declared_operator():
    declared = set(re.findall(r"\b(poseidon_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", HEADER, flags=re.S)))
    out = subprocess.run(["nm", "-D", "--defined-only", P.LIB_PATH], capture_output=True, text=True, check=True).stdout
    assert declared <= set(re.findall(r"\bT (poseidon_[a-z_]+)", out))
    assert declared == set(L.EXPORTS)


def test_limits_match_the_header():
    def value(name):
        return int(re.search(rf"#define POSEIDON_{name} \(?([0-9a-fx<u ]+)\)?", HEADER).group(1).replace("u", "")
                   .split("<<")[0], 0) << {"WIDTH_MAX": 20, "PITCH_MAX": 24}.get(name, 0)
    assert value("GROUP") == L.GROUP == O.GROUP
    assert value("WIDTH_MAX") == L.WIDTH_MAX and value("PITCH_MAX") == L.PITCH_MAX
    for name in ("ROWS_MAX", "EXPERTS_MAX", "RANGES_MAX", "VOCAB_MAX", "TILES_MAX"):
        assert value(name) == getattr(L, name)


A = 1 << 20    # an aligned address that no refused call reads


def _good():
    """Arguments that pass every check, by operator; a refusal changes one of them."""
    return {
        "poseidon_stash": [A, 8, 2, 4, 8, A, A, None],
        "poseidon_restore": [A, A, 4, 8, A, 8, 2, None],
        "poseidon_gated_forward": [A, 8, A, 8, 2, 4, 8, A, 8, A, A, A, A, None],
        "poseidon_gated_backward": [A, 8, 2, 4, 8, A, A, A, A, A, 8, A, 8, None],
        "poseidon_weight_gradient": [A, 8, 2, 4, 8, A, A, 8, None, 1, A, 0, 0, None, 0, None],
        "poseidon_expert_sort": [A, 4, 2, 8, A, A, A, None, 0, None],
        "poseidon_expert_gather": [A, 8, 2, 4, 8, A, 2, A, A, A, A, None],
        "poseidon_expert_combine": [A, 2, 4, 8, A, 2, A, A, 8, None],
        "poseidon_expert_combine_backward": [A, 8, A, 2, 4, 8, A, 2, A, A, A, A, None],
        "poseidon_embed": [A, 4, A, 8, 2, 16, 8, 1.0, A, 8, None],
        "poseidon_embed_backward": [A, 4, A, 8, 2, 16, 8, 1.0, A, 8, 0, 0, A, 1 << 30, None],
    }


REFUSED = [
    # null pointers
    *[("poseidon_stash", i, None, BAD) for i in (0, 5, 6)],
    *[("poseidon_restore", i, None, BAD) for i in (0, 1, 4)],
    *[("poseidon_gated_forward", i, None, BAD) for i in (0, 2, 7, 9, 10, 11, 12)],
    *[("poseidon_gated_backward", i, None, BAD) for i in (0, 5, 6, 7, 8, 9, 11)],
    *[("poseidon_weight_gradient", i, None, BAD) for i in (0, 5, 6, 10)],
    *[("poseidon_expert_sort", i, None, BAD) for i in (0, 4, 5, 6)],
    *[("poseidon_expert_gather", i, None, BAD) for i in (0, 5, 7, 9, 10)],
    *[("poseidon_expert_combine", i, None, BAD) for i in (0, 4, 7)],
    *[("poseidon_expert_combine_backward", i, None, BAD) for i in (0, 2, 6, 8, 9, 10, 11)],
    *[("poseidon_embed", i, None, BAD) for i in (0, 2, 8)],
    *[("poseidon_embed_backward", i, None, BAD) for i in (0, 2, 8, 12)],
    # unknown types, a 32-bit gradient for the 16-bit matrix instructions
    ("poseidon_stash", 2, 3, BAD), ("poseidon_restore", 6, 3, BAD), ("poseidon_gated_forward", 4, 9, BAD),
    ("poseidon_gated_backward", 2, 3, BAD), ("poseidon_weight_gradient", 2, 3, BAD),
    ("poseidon_weight_gradient", 2, 0, BAD), ("poseidon_weight_gradient", 11, 3, BAD),
    ("poseidon_expert_gather", 2, 3, BAD), ("poseidon_expert_combine", 1, 3, BAD),
    ("poseidon_expert_combine_backward", 3, 3, BAD), ("poseidon_embed", 4, 3, BAD),
    ("poseidon_embed_backward", 4, 3, BAD), ("poseidon_embed_backward", 10, 3, BAD),
    # widths of 0, pitches below the width, addresses between values, codes and workspaces off their boundary
    ("poseidon_stash", 4, 0, BAD), ("poseidon_stash", 1, 7, BAD), ("poseidon_stash", 0, A + 1, BAD),
    ("poseidon_stash", 5, A + 8, BAD), ("poseidon_restore", 5, 7, BAD), ("poseidon_gated_forward", 3, 7, BAD),
    ("poseidon_gated_backward", 10, 7, BAD), ("poseidon_weight_gradient", 1, 7, BAD),
    ("poseidon_weight_gradient", 7, 0, BAD), ("poseidon_weight_gradient", 10, A + 2, BAD),
    ("poseidon_expert_combine", 8, 7, BAD), ("poseidon_embed", 3, 7, BAD), ("poseidon_embed_backward", 9, 7, BAD),
    ("poseidon_embed_backward", 12, A + 128, BAD), ("poseidon_embed_backward", 13, 64, BAD),
    # flags, counts
    ("poseidon_weight_gradient", 12, 2, BAD), ("poseidon_weight_gradient", 9, 0, BAD),
    ("poseidon_weight_gradient", 9, 2, BAD),    # two ranges without offsets
    ("poseidon_embed_backward", 11, 2, BAD), ("poseidon_expert_sort", 2, 0, BAD), ("poseidon_expert_sort", 3, 0, BAD),
    ("poseidon_expert_gather", 6, 0, BAD), ("poseidon_expert_combine", 5, 0, BAD),
    ("poseidon_expert_combine_backward", 7, 0, BAD),
    # sizes above the limits
    ("poseidon_stash", 3, 1 << 31, BIG), ("poseidon_stash", 4, (1 << 20) + 1, BIG), ("poseidon_stash", 1, 1 << 33, BIG),
    ("poseidon_restore", 2, 1 << 31, BIG), ("poseidon_gated_forward", 5, 1 << 40, BIG),
    ("poseidon_gated_backward", 4, 1 << 21, BIG), ("poseidon_weight_gradient", 3, 1 << 31, BIG),
    ("poseidon_weight_gradient", 9, 65536, BIG), ("poseidon_expert_sort", 1, 1 << 30, BIG),
    ("poseidon_expert_sort", 3, 512, BIG), ("poseidon_expert_gather", 6, 1 << 30, BIG),
    ("poseidon_expert_combine", 2, 1 << 62, BIG), ("poseidon_expert_combine_backward", 4, 1 << 31, BIG),
    ("poseidon_embed", 5, 1 << 26, BIG), ("poseidon_embed_backward", 5, 1 << 26, BIG),
    ("poseidon_embed_backward", 1, 1 << 31, BIG),
]


@pytest.mark.parametrize("name, at, value, status", REFUSED)
def test_refusals(name, at, value, status):
    args = _good()[name]
    args[at] = value
    assert getattr(L.lib(), name)(*args) == status


def test_empty_calls_need_no_buffers():
    lib = L.lib()
    assert lib.poseidon_stash(None, 8, 2, 0, 8, None, None, None) == P.POSEIDON_OK
    assert lib.poseidon_restore(None, None, 0, 8, None, 8, 2, None) == P.POSEIDON_OK
    assert lib.poseidon_gated_forward(None, 8, None, 8, 2, 0, 8, None, 8, None, None, None, None, None) == P.POSEIDON_OK
    assert lib.poseidon_expert_gather(None, 8, 2, 0, 8, None, 2, None, None, None, None, None) == P.POSEIDON_OK
    assert lib.poseidon_expert_combine(None, 2, 0, 8, None, 2, None, None, 8, None) == P.POSEIDON_OK
    assert lib.poseidon_embed(None, 0, None, 8, 2, 0, 8, 1.0, None, 8, None) == P.POSEIDON_OK
    # an embedding gradient of no rows and no tokens
    assert lib.poseidon_embed_backward(None, 0, None, 8, 2, 0, 8, 1.0, None, 8, 0, 0, None, 0, None) == P.POSEIDON_OK


def test_workspaces():
    lib, none = L.lib(), 2 ** 64 - 1
    assert lib.poseidon_weight_gradient_workspace(1 << 31, 64, 64, 1) == none
    assert lib.poseidon_weight_gradient_workspace(64, 1 << 20, 1 << 20, 1) == none      # more than 2^22 tiles
    assert lib.poseidon_weight_gradient_workspace(64, 64, 64, 0) == none
    assert lib.poseidon_weight_gradient_workspace(64, 64, 64, 1) == 0
    assert lib.poseidon_expert_sort_workspace(64, 0, 8) == none
    assert lib.poseidon_expert_sort_workspace(64, 2, 512) == none
    assert lib.poseidon_expert_sort_workspace(1, 8, 64) == 0
    assert lib.poseidon_embed_backward_workspace(64, 1 << 26, 64) == none
    assert lib.poseidon_embed_backward_workspace(0, 100, 64) == 0
    assert lib.poseidon_embed_backward_workspace(64, 100, 64) > 0


def test_the_workspace_of_a_weight_gradient_is_bounded():
    """Parts of the rows take at most 1 GB however large the gradient is, and a copy of dy at most 8 GB."""
    f, rng = L.lib().poseidon_weight_gradient_workspace, np.random.default_rng(0)
    sizes = [(1 << 20, 32776, 32776, 1), (65536, 8200, 8200, 1), (65536, 16640, 16640, 1), (1 << 20, 2048, 2048, 64)]
    sizes += [(int(2 ** rng.uniform(0, 21)), 8 * int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 16)),
               int(2 ** rng.uniform(0, 8)) if rng.random() < 0.5 else 1) for _ in range(20000)]
    for size in sizes:
        need, tables = f(*size), 32 * (size[3] + 2 * 1024) + 1024
        assert need == 2 ** 64 - 1 or need <= (1 << 30) + tables, size
        odd = f(size[0], size[1] + 3, *size[2:])
        assert odd == 2 ** 64 - 1 or odd <= (1 << 30) + tables + (8 << 30), size
    assert f(8192, 5120, 3584, 1) == 2 * 5120 * 3584 * 4        # in two parts


def test_the_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros(4, 64)
    s = L.Stash(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 64, torch.float32)
    plan = L.ExpertPlan(torch.zeros(8, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32),
                        torch.zeros(3, dtype=torch.int32))
    for f, args in ((L.poseidon_stash, (x,)), (L.poseidon_restore, (s,)), (L.poseidon_gated_forward, (x, x)),
                    (L.poseidon_gated_backward, (x, s, s)), (L.poseidon_weight_gradient, (x, s)),
                    (L.poseidon_expert_sort, (plan.position, 2)), (L.poseidon_expert_gather, (x, plan)),
                    (L.poseidon_expert_combine, (x, plan)), (L.poseidon_expert_combine_backward, (x, x, plan, x)),
                    (L.poseidon_embed, (plan.order, x)), (L.poseidon_embed_backward, (plan.order, x, 10))):
        with pytest.raises(P.PoseidonError) as ei:
            f(*args)
        assert ei.value.status == BAD


def test_the_binding_refuses_a_stream_of_another_gpu(monkeypatch):
    """Work would be enqueued on the tensors' GPU's current stream, and not on the one that was asked for."""
    class Tensor:                              # what the binding asks of the memory that a stash holds
        is_cuda, device, streams = True, torch.device("cuda", 0), []

        def record_stream(self, stream):
            self.streams.append(stream)

    class Stash(L.Stash):
        def tensors(self):
            return (Tensor(),)

    class Stream:
        def __init__(self, index):
            self.device = torch.device("cuda", index)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    s = Stash(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), 64, torch.float32)
    calls = []
    f = L._streamed(lambda stash: calls.append(stash))
    own = Stream(0)
    f(s, stream=own)
    assert calls == [s] and Tensor.streams == [own]
    with pytest.raises(P.PoseidonError) as ei:
        f(s, stream=Stream(1))
    assert ei.value.status == BAD and len(calls) == 1


# ---- the oracle against itself ----

def test_the_8_bit_form_holds_its_bounds():
    """|x - restored| <= 2^e / 2 with 127 2^e < 2 max |x|: below max |x| / 127; the ends of every type stay finite."""
    rng = np.random.default_rng(0)
    x = rng.normal(size=(40, 200)) * np.exp(rng.normal(size=(40, 200)) * 3)
    codes, scales = O.stash(x, "f32")
    back = O.restore(codes, scales, 200)
    for b in range(4):
        part, err = x[:, b * 64:(b + 1) * 64], np.abs(back - x)[:, b * 64:(b + 1) * 64]
        assert (err.max(axis=1) <= np.abs(part).max(axis=1) / 127).all()
    top = {"f32": float(np.finfo(np.float32).max), "bf16": 2.0 ** 128 * (1 - 2.0 ** -8), "f16": 65504.0}
    for kind, most in top.items():
        back = O.restore(*O.stash(np.array([[most, -most, 0.0]]), kind), 3)
        assert (np.abs(back) <= most).all() and abs(back[0, 0] - most) <= most / 127


def _difference(f, x, dx, h=1e-6):
    return (f(x + h * dx) - f(x - h * dx)) / (2 * h)


def test_gradients_against_differences():
    """Central differences of step 1e-6 on functions of order 1: an error of about 1e-12 / 1e-6 + 1e-12, held to 1e-7."""
    rng = np.random.default_rng(1)
    n, d, k, e = 7, 5, 3, 4
    g, u, w, dg, du = (rng.normal(size=(n, d)) for _ in range(5))
    want = _difference(lambda t: (w * O.gated_forward(g + t * dg, u + t * du)).sum(), 0.0, 1.0)
    a, b = O.gated_backward(w, g, u)
    assert abs((a * dg).sum() + (b * du).sum() - want) < 1e-7

    x, W, dW, offsets = rng.normal(size=(n, d)), rng.normal(size=(2, 6, d)), rng.normal(size=(2, 6, d)), [0, 3, n]
    dy = rng.normal(size=(n, 6))

    def loss(V):
        return sum((dy[a:b] * (x[a:b] @ V[r].T)).sum() for r, (a, b) in enumerate(zip(offsets, offsets[1:])))
    assert abs((O.weight_gradient(dy, x, offsets) * dW).sum() - _difference(loss, W, dW)) < 1e-7

    choice = rng.integers(-1, e, size=(n, k))
    _, position, _ = O.expert_sort(choice, e)
    ys, dys = rng.normal(size=(2, n * k, d))
    ws, dws = rng.normal(size=(2, n, k))
    want = _difference(lambda t: (w * O.expert_combine(ys + t * dys, position, ws + t * dws)).sum(), 0.0, 1.0)
    a, b = O.expert_combine_backward(w, ys, position, ws)
    assert abs((a * dys).sum() + (b * dws).sum() - want) < 1e-7
    back = rng.normal(size=(n * k, d))
    want = _difference(lambda v: (back * O.expert_gather(v, position)).sum(), x, dg)
    assert abs((O.expert_combine(back, position, np.ones((n, k))) * dg).sum() - want) < 1e-7

    ids = rng.integers(-1, 6, size=n)
    table, dtable = rng.normal(size=(2, 5, d))
    want = _difference(lambda v: (w * O.embed(ids, v, 1.5)).sum(), table, dtable)
    assert abs((O.embed_backward(ids, w, 5, 1.5) * dtable).sum() - want) < 1e-7

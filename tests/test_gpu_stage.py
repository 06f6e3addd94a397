"""The stage's layers: their gradients against a 64-bit model, and a plan from measured layers."""
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import coracle  # noqa: E402
from paper_2609_06086_amd import poseidon as P  # noqa: E402
from paper_2609_06086_amd import stage as S  # noqa: E402

SHAPE = S.Shape(vocab=300, width=128, experts=5, chosen=2, inner=192, tokens=200)


def _profiles():
    return S.LayerProfile(40.2, 71.7, 10 ** 8, 10 ** 4), S.LayerProfile(900.0, 1800.4, 2 * 10 ** 8, 3 * 10 ** 7)


def test_plan_problem_fills_the_tables():
    """Times by device type, rounded; memory of weights and of min(S, M) micro-batches, rounded up to whole MB."""
    prob = S.plan_problem(*_profiles(), blocks=5, stages=3, micro_batches=2, slower=(1.0, 2.0), caps_mb=(1000, 900))
    assert P.poseidon_validate(prob) == 10 * 8
    assert prob.fwd.tolist() == [[40] + [900] * 5, [80] + [1800] * 5]
    assert prob.bwd.tolist() == [[72] + [1800] * 5, [143] + [3601] * 5]
    assert prob.mem.tolist() == [101] + [260] * 5 and prob.cap.tolist() == [1000, 900]


def test_plan_problem_leaves_room_for_a_pass():
    """What the largest pass works with is free on every device, once; a device that has less holds nothing."""
    first, block = (S.LayerProfile(p.fwd_us, p.bwd_us, p.weight_bytes, p.kept_bytes, work_bytes=w)
                    for p, w in zip(_profiles(), (10 ** 6, 150 * 10 ** 6 + 1)))
    prob = S.plan_problem(first, block, blocks=5, stages=3, micro_batches=2, caps_mb=(1000, 90))
    assert prob.cap.tolist() == [849, 0] and prob.mem.tolist() == [101] + [260] * 5


@pytest.mark.gpu
def test_the_measured_memory_of_a_pass():
    """At least what the block's backward pass holds at once: the restored outputs and their gradient, then both
    gradients of the gated activation, dact and the activation, in 16 bits; at most a few times that, and no weights."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    shape = S.Shape(vocab=300, width=256, experts=5, chosen=2, inner=192, tokens=4000)
    first, block = S.measure(shape, repeats=2)
    rows, least = shape.tokens * shape.chosen, 2 * shape.tokens * shape.chosen * (2 * shape.width + 4 * shape.inner)
    assert least <= block.work_bytes <= 3 * least + rows * 200 + (64 << 20)
    assert shape.tokens * shape.width * 2 <= first.work_bytes <= (64 << 20)


@pytest.mark.gpu
def test_gradients_of_the_block_and_the_embedding():
    """Against a model in 64 bits on the same weights and the same choices.  A kept value is off by 0.011 of its
    group's deviation at the root mean square (a step of 2.5 deviations / 63.5 over the root of 12, for the largest of 64
    normal values), a gradient holds up to three such factors and bf16 roundings of 0.004 / 2 each:
    sqrt(3 * 0.011^2 + 8 * 0.002^2) = 0.02; held to 0.05."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    first, block = S.Embedding(SHAPE, dev, 1), S.ExpertBlock(SHAPE, dev, 2)
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    ids = torch.randint(-1, SHAPE.vocab, (SHAPE.tokens,), generator=g, device=dev, dtype=torch.int32)
    first.table.mul_(4)
    x, _ = first.forward(ids)
    out, kept = block.forward(x)
    dout = torch.randn(out.shape, generator=g, device=dev).bfloat16()
    for _ in range(2):                        # two micro-batches: the gradients add up
        dx = block.backward(dout, kept)
        first.backward(dx, ids)

    table, router, w1, w2 = (t.double().cpu().requires_grad_() for t in (first.table, block.router, block.w1, block.w2))
    there = (ids >= 0).cpu()
    h = table[ids.clamp(min=0).long().cpu()] * first.scale * there.unsqueeze(1)
    h.retain_grad()
    choice = kept.choice.long().cpu()
    probs = torch.softmax(torch.gather(h @ router.t(), 1, choice), 1)
    y = h
    for j in range(SHAPE.chosen):
        a = torch.bmm(w1[choice[:, j]], h.unsqueeze(2)).squeeze(2)
        act = torch.nn.functional.silu(a[:, :SHAPE.inner]) * a[:, SHAPE.inner:]
        y = y + probs[:, j:j + 1] * torch.bmm(w2[choice[:, j]], act.unsqueeze(2)).squeeze(2)
    y.backward(dout.double().cpu())

    def off(got, want):
        return float((got.double().cpu() - want).norm() / want.norm())
    assert off(out, y.detach()) < 0.05
    assert off(dx, h.grad) < 0.05
    assert off(block.dw1, 2 * w1.grad) < 0.05 and off(block.dw2, 2 * w2.grad) < 0.05
    assert off(block.drouter, 2 * router.grad) < 0.05 and off(first.grad, 2 * table.grad) < 0.05


@pytest.mark.gpu
def test_a_plan_from_measured_layers():
    """Measured tables go through the planner: its optimum is the oracle's; 8 bits keep about half of 16."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    first, block = S.measure(SHAPE, repeats=2)
    _, plain = S.measure(SHAPE, keep_8_bits=False, repeats=2)
    assert 0 < block.kept_bytes < 0.62 * plain.kept_bytes
    prob = S.plan_problem(first, block, blocks=7, stages=3, micro_batches=8, caps_mb=(64, 64))
    ctx = P.poseidon_load_costs(prob, 0)
    best, _ = P.poseidon_search(ctx, rows_per_chunk=0)
    ctx.close()
    assert (best.index, best.makespan) == coracle.search(prob, 2 ** 31 - 1, rows_per_chunk=0)["best"]


@pytest.mark.gpu
def test_the_command_says_whose_times_it_plans_with(monkeypatch, capsys):
    """Layers run with activations in 8 bits only: a plan for 16 bits has the same times, and says so."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    monkeypatch.setattr("sys.argv", "stage --tokens 200 --width 128 --experts 5 --inner 192 --blocks 7 --stages 3 "
                                    "--micro-batches 8 --cap-mb 200".split())
    S.main()
    eight, sixteen = capsys.readouterr().out.splitlines()
    assert "in 8 bits" in eight and "in 16 bits" in sixteen and "times of 8 bits" in sixteen

    def times(line):
        return re.search(r"block (\d+ \+ \d+) us", line).group(1)

    def kept(line):
        return float(re.search(r"keeps ([\d.]+) MB", line).group(1))
    assert times(eight) == times(sixteen) and kept(eight) < 0.62 * kept(sixteen)
    assert times(eight) == times(sixteen) and kept(eight) < 0.62 * kept(sixteen)


def test_the_command_explains_its_options(monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["stage", "--help"])
    with pytest.raises(SystemExit) as ei:
        S.main()
    text = " ".join(capsys.readouterr().out.split())
    assert ei.value.code == 0 and "default: 5% above an even share" in text and "argparse" not in text

"""The stage's attention block and whole layers: their gradients against a 64-bit model, and a plan from measured layers."""
import re

import pytest

torch = pytest.importorskip("torch")

from oracle import coracle  # noqa: E402
from paper_2609_06086_amd import poseidon as P  # noqa: E402
from paper_2609_06086_amd import stage as S  # noqa: E402

SHAPE = S.Shape(vocab=300, width=128, experts=5, chosen=2, inner=192, tokens=200, heads=4, kv_heads=2)


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def test_heads_share_the_width():
    for heads in (0, 3):
        with pytest.raises(ValueError):
            S.AttentionBlock(S.Shape(width=128, heads=heads), torch.device("cpu"))


def _attention(x, norm, wqkv, wo, cuts):
    """The block in 64 bits, from its weights."""
    n, d = x.shape
    dim, kv = d // SHAPE.heads, SHAPE.kv_heads
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6) * norm
    q, k, v = (t.reshape(n, -1, dim) for t in (y @ wqkv.t()).split([d, kv * dim, kv * dim], dim=1))
    k, v = (t.repeat_interleave(SHAPE.heads // kv, 1) for t in (k, v))
    rows = []
    for a, b in zip(cuts, cuts[1:]):
        later = torch.ones(b - a, b - a, dtype=torch.bool).triu(1)
        s = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b]) * dim ** -0.5
        rows.append(torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(later, -float("inf")), 2), v[a:b]).reshape(b - a, d))
    return x + torch.cat(rows) @ wo.t()


def _off(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("cuts", [None, [0, 1, 70, 70, 200]])
def test_gradients_of_the_attention_block(cuts):
    """Against a model in 64 bits on the same weights.  About twelve roundings of 2^-9 of the value at the root mean square, and
    two times what 8 bits are off, 0.011 of their group's deviation: sqrt(12 * 2^-18 + 2 * 0.011^2) = 0.017; held to 0.05."""
    dev = _gpu()
    block = S.AttentionBlock(SHAPE, dev, 1)
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    block.norm.copy_(1 + 0.2 * torch.randn(SHAPE.width, generator=g, device=dev))
    block.wqkv.mul_(1.5)
    x = torch.randn(SHAPE.tokens, SHAPE.width, generator=g, device=dev).bfloat16()
    dout = torch.randn(x.shape, generator=g, device=dev).bfloat16()
    offsets = None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device=dev)
    out, kept = block.forward(x, offsets)
    for _ in range(2):                        # two micro-batches: the gradients add up
        dx = block.backward(dout, kept)
    X, norm, wqkv, wo = (t.double().cpu().requires_grad_() for t in (x, block.norm, block.wqkv, block.wo))
    want = _attention(X, norm, wqkv, wo, [0, SHAPE.tokens] if cuts is None else cuts)
    want.backward(dout.double().cpu())
    assert _off(out, want.detach()) < 0.05 and _off(dx, X.grad) < 0.05
    assert _off(block.dnorm, 2 * norm.grad) < 0.05 and _off(block.dwqkv, 2 * wqkv.grad) < 0.05 and _off(block.dwo, 2 * wo.grad) < 0.05
    assert kept.kept_bytes < kept.plain_bytes


@pytest.mark.gpu
def test_gradients_of_a_layer():
    """The attention block's and, after it, the experts', whose choices the model takes over; bounds as above, with twice as many
    steps: sqrt(30 * 2^-18 + 5 * 0.011^2) = 0.027; held to 0.08."""
    dev = _gpu()
    layer = S.Layer(SHAPE, dev, 5)
    g = torch.Generator(device=dev)
    g.manual_seed(6)
    x = torch.randn(SHAPE.tokens, SHAPE.width, generator=g, device=dev).bfloat16()
    dout = torch.randn(x.shape, generator=g, device=dev).bfloat16()
    out, kept = layer.forward(x)
    dx = layer.backward(dout, kept)
    at, ex = layer.attention, layer.experts
    X, norm, wqkv, wo, router, w1, w2 = (t.double().cpu().requires_grad_() for t in (x, at.norm, at.wqkv, at.wo, ex.router, ex.w1, ex.w2))
    h = _attention(X, norm, wqkv, wo, [0, SHAPE.tokens])
    choice = kept.experts.choice.long().cpu()
    probs = torch.softmax(torch.gather(h @ router.t(), 1, choice), 1)
    y = h
    for j in range(SHAPE.chosen):
        a = torch.bmm(w1[choice[:, j]], h.unsqueeze(2)).squeeze(2)
        act = torch.nn.functional.silu(a[:, :SHAPE.inner]) * a[:, SHAPE.inner:]
        y = y + probs[:, j:j + 1] * torch.bmm(w2[choice[:, j]], act.unsqueeze(2)).squeeze(2)
    y.backward(dout.double().cpu())
    assert _off(out, y.detach()) < 0.08 and _off(dx, X.grad) < 0.08
    for got, want in ((at.dwqkv, wqkv), (at.dwo, wo), (at.dnorm, norm), (ex.dw1, w1), (ex.dw2, w2), (ex.drouter, router)):
        assert _off(got, want.grad) < 0.08


@pytest.mark.gpu
def test_experts_in_32_bits_run_forward():
    dev = _gpu()
    block = S.ExpertBlock(SHAPE, dev, 2, dtype=torch.float32)
    x = torch.randn(60, SHAPE.width, device=dev)
    out, kept = block.forward(x)
    choice, y = kept.choice.long(), x.double()
    for j in range(SHAPE.chosen):
        a = torch.matmul(block.w1[choice[:, j]].double(), x.double().unsqueeze(2)).squeeze(2)
        act = torch.nn.functional.silu(a[:, :SHAPE.inner]) * a[:, SHAPE.inner:]
        y = y + kept.probs[:, j:j + 1] * torch.matmul(block.w2[choice[:, j]].double(), act.unsqueeze(2)).squeeze(2)
    assert _off(out, y.cpu()) < 1e-5          # sums of 128 and 192 products in 32 bits


@pytest.mark.gpu
def test_a_plan_from_measured_layers():
    _gpu()
    first, layer = S.measure(SHAPE, repeats=2)
    assert 0 < layer.kept_bytes < layer.plain_bytes
    prob = S.plan_problem(first, layer, blocks=7, stages=3, micro_batches=8, caps_mb=(64, 64))
    ctx = P.poseidon_load_costs(prob, 0)
    best, _ = P.poseidon_search(ctx, rows_per_chunk=0)
    ctx.close()
    assert (best.index, best.makespan) == coracle.search(prob, 2 ** 31 - 1, rows_per_chunk=0)["best"]


@pytest.mark.gpu
def test_the_command_plans_layers_with_attention(monkeypatch, capsys):
    _gpu()
    monkeypatch.setattr("sys.argv", "stage --tokens 200 --width 128 --experts 5 --inner 192 --blocks 7 --stages 3 --micro-batches 8 "
                                    "--heads 4 --kv-heads 2 --sequence 64 --cap-mb 200".split())
    S.main()
    eight, sixteen = capsys.readouterr().out.splitlines()
    keeps = [float(re.search(r"keeps ([\d.]+) MB", line).group(1)) for line in (eight, sixteen)]
    assert "best plan" in eight and keeps[0] < keeps[1]

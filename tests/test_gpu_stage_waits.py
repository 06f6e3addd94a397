"""How often a pass of the stage's layers waits for the GPU: only the 32-bit experts do, once, for their ranges."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_06086_amd import stage as S  # noqa: E402

pytestmark = pytest.mark.gpu
SHAPE = S.Shape(width=128, experts=40, chosen=2, inner=64, heads=4)


@pytest.mark.parametrize("dtype, waits, products", [(torch.float32, 1, 2), (torch.bfloat16, 0, 0)])
def test_waits_and_products_of_a_forward_pass(monkeypatch, dtype, waits, products):
    """Of 3 tokens by 2 of 40 experts at most 6 experts have rows, for which the library is asked for two products each."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    block = S.ExpertBlock(SHAPE, dev, 2, dtype=dtype)
    x = torch.randn(3, SHAPE.width, device=dev).to(dtype)
    block.forward(x)
    count = {"tolist": 0, "matmul": 0}

    def counted(name, f):
        def g(*args, **kw):
            count[name] += 1
            return f(*args, **kw)
        return g
    monkeypatch.setattr(torch.Tensor, "tolist", counted("tolist", torch.Tensor.tolist))
    monkeypatch.setattr(torch, "matmul", counted("matmul", torch.matmul))
    _, kept = block.forward(x)
    monkeypatch.undo()
    busy = len(kept.choice.unique())
    assert count == {"tolist": waits, "matmul": products * busy}


def test_a_layer_does_not_wait():
    """Forward and backward in 16 bits, with torch told to raise where it would wait for the GPU."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dev = torch.device("cuda:0")
    layer = S.Layer(SHAPE, dev, 4)
    x = torch.randn(100, SHAPE.width, device=dev).bfloat16()
    offsets = torch.tensor([0, 30, 100], dtype=torch.int32, device=dev)
    torch.cuda.set_sync_debug_mode("error")
    try:
        out, kept = layer.forward(x, offsets)
        dx = layer.backward(out, kept)
    finally:
        torch.cuda.set_sync_debug_mode("default")
    assert torch.isfinite(dx).all()

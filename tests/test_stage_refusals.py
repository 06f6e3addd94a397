"""Sizes that a stage's attention cannot have are refused before anything is allocated or run."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_06086_amd import stage as S  # noqa: E402

REFUSED = [dict(width=2048, heads=8), dict(width=96, heads=8), dict(width=1152, heads=8), dict(width=512, heads=8, kv_heads=3),
           dict(width=512, heads=8, kv_heads=16), dict(width=512, heads=8, kv_heads=-2), dict(width=16392, heads=2049),
           dict(width=32768, heads=256), dict(width=512, heads=-8), dict(width=512, heads=8, sequence=-1)]
CPU = torch.device("cpu")


@pytest.mark.parametrize("sizes", REFUSED)
def test_sizes_of_an_attention_block(sizes):
    with pytest.raises(ValueError):
        S.AttentionBlock(S.Shape(**sizes), CPU)
    with pytest.raises(ValueError):
        S.Layer(S.Shape(**sizes), CPU)


def test_attention_is_in_16_bits():
    for block in (S.AttentionBlock, S.Layer):
        with pytest.raises(ValueError):
            block(S.Shape(width=128, heads=2, experts=2, inner=64), CPU, dtype=torch.float32)


@pytest.mark.parametrize("sizes", [dict(width=128, heads=16), dict(width=128, heads=1), dict(width=240, heads=2, kv_heads=1)])
def test_sizes_that_an_attention_block_takes(sizes):
    block = S.AttentionBlock(S.Shape(**sizes), CPU)
    assert block.dim * block.heads == sizes["width"] and block.wqkv.shape == (sum(block.parts), sizes["width"])


@pytest.mark.parametrize("args, named", [("--heads 8", "8 heads"), ("--heads 16 --kv-heads 3", "3 heads of keys"),
                                         ("--width 2000 --heads 20", "width of 2000"), ("--heads 16 --sequence -5", "-5 tokens")])
def test_the_command_names_what_it_does_not_take(monkeypatch, capsys, args, named):
    monkeypatch.setattr("sys.argv", ["stage"] + args.split())
    with pytest.raises(SystemExit) as e:
        S.main()
    assert e.value.code == 2 and named in capsys.readouterr().err.splitlines()[-1]

"""The workspace of attention's backward pass, value by value: two words a query and head, and the parts of the query heads that
share a key, of the split that a call with these sequences takes or a call without offsets, whichever needs more."""
import numpy as np
import pytest

pytest.importorskip("torch")

from paper_2609_06086_amd import layers as L  # noqa: E402
from test_gpu_transformer_variants import _split  # noqa: E402


def test_the_workspace_fits_both_kinds_of_calls():
    f, rng = L.lib().poseidon_attention_backward_workspace, np.random.default_rng(3)
    for _ in range(3000):
        kv, group, dim = int(2 ** rng.uniform(0, 6)), int(2 ** rng.uniform(0, 4)), 8 * int(rng.integers(1, 17))
        tokens, sequences = int(2 ** rng.uniform(0, 26)), int(2 ** rng.uniform(0, 16))
        parts = max(_split(tokens, n, kv * group, kv, dim) for n in (sequences, 0))
        want = tokens * kv * group * 8 + (parts > 1) * parts * tokens * kv * dim * 8
        assert f(tokens, kv * group, kv, dim, sequences) == want
        assert group % parts == 0 and (parts == 1 or parts * tokens * kv * dim * 8 <= 1 << 30)

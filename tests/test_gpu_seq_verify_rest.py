"""What is left of p less q where a draft's logits are the target's: nothing, wherever the rows lie in memory."""
import numpy as np
import pytest
import torch

from test_gpu_seq_verify import _compare, _logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [997, 5003, 50021])
def test_refused_where_the_draft_is_the_target(dtype, V):
    """A drafted token that neither gives any weight is refused, and the next is drawn from p.  Rows of an odd number of logits are summed in another order where they begin at another alignment."""
    g = np.random.default_rng(V)
    B, n = 6, 5
    logits = _logits(g, B, n, V, dtype)
    tokens = g.integers(0, V, (B, n))
    for b in range(B):
        for i in range(n - 1):
            logits[b, i, tokens[b, i + 1]] = -float("inf")
    draft = logits[:, :n - 1].clone()
    for temperatures in (None, g.uniform(0.5, 1.5, B)):
        for _ in range(3):
            assert _compare(logits, tokens, g.random((B, n + 1)), draft=draft, temperatures=temperatures) == [1] * B
    for first in range(1, 8):   # every alignment of the draft against the target
        wide = torch.zeros((B, n - 1, V + 11), dtype=logits.dtype, device="cuda")
        wide[..., first:first + V] = draft
        _compare(logits, tokens, g.random((B, n + 1)), draft=wide[..., first:first + V])

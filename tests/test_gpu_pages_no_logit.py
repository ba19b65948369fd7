"""Attention over pages: rows whose logits are all -infinity are zeros, whatever values lie in the slots that they see."""
import numpy as np
import pytest
import torch

from pages_helpers import Case, bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("counts,lengths", [((3, 2), (90, 700)), ((40, 33), (300, 64)), ((1, 1), (5000, 40)), ((60, 1), (5000, 2049))])
def test_zeros_over_values_that_are_no_numbers(counts, lengths, dh):
    rng = np.random.default_rng(dh + counts[0])
    inf, nan, T = float("inf"), float("nan"), max(lengths)
    k, v = bf16(rng, 2, T, 1, dh), bf16(rng, 2, T, 1, dh)
    v[:, 7, 0, 3], v[:, 8, 0, 4], v[:, 9, 0, 5] = inf, nan, -inf           # (slots that every row sees, and the last ones)
    for b, t in enumerate(lengths):
        v[b, t - 1, 0, dh - 1], v[b, t - 1, 0, 0] = nan, inf
    c = Case(rng, 2, 1, dh, 16, 16, lengths, counts, k=k, v=v)
    c.cache.k.fill_(-inf)
    c.q.copy_(c.q.abs() + 0.5)
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=max(counts), max_length=T, with_lse=True)
    assert not out.any() and torch.all(lse == -inf)

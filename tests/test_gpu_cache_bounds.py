"""Lengths beyond max_length, and a bound far above the lengths: in every path of the attention, with weights."""
import numpy as np
import pytest
import torch

from answer_helpers import ints
from test_gpu_cache_attention import build, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n_q,H,H_kv", [(1, 2, 2), (3, 8, 2), (40, 2, 2), (60, 1, 1), (130, 2, 1)])
def test_lengths_and_their_bound(n_q, H, H_kv, dh):
    rng = np.random.default_rng(n_q)
    ctx, cache, q = build(rng, 3, H, H_kv, dh, n_q, (1500, 1500, 1500), cap=1504)
    start = cache.weight.clone()
    for asked, bound, counts in (((1500, 700, 2 ** 31 - 1), 333, None), ((5, 1, 0), 1504, None), ((1500, 2, -2 ** 31), 1499, (n_q, 1, n_q)),
                                 ((33, 32, 31), 32, (0, n_q + 5, -3))):
        cache.weight.copy_(start)
        out = torch.full_like(q, 9.0)
        print("case", n_q, H, H_kv, dh, asked, bound, counts, flush=True)
        ctx.cache_attention(cache, q, ints(*asked), None if counts is None else ints(*counts), max_length=bound, accumulate=True, out=out)
        lengths = [min(max(t, 0), bound) for t in asked]
        check(cache, q, out, start, lengths, [min(max(c, 0), n_q) for c in counts or (n_q,) * 3], dh ** -0.5)
    ctx.close()

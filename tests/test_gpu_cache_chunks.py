"""One context for a chunk of queries and for the single ones behind it."""
import numpy as np
import pytest
import torch

from answer_helpers import bf16, context, fill, garbage_cache, ints
from test_gpu_cache_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,H_kv,dh,length,calls", [(1, 32, 32, 128, 700, (49, 1, 16, 48, 4)),
                                                      (2, 8, 2, 64, 1500, (128, 1, 16, 48, 96, 4))])
def test_a_context_for_a_chunk_takes_fewer_queries(B, H, H_kv, dh, length, calls):
    rng = np.random.default_rng(H)
    ctx = context(B, H, H_kv, max(calls), length, dh)
    cap = (length + 31) // 32 * 32
    cache = garbage_cache(B, H_kv, dh, cap)
    fill(ctx, cache, bf16(rng, B, length, H_kv, dh), bf16(rng, B, length, H_kv, dh), (length,) * B)
    for n_q in calls:
        q = bf16(rng, B, n_q, H, dh, scale=1.3).cuda()
        before = cache.weight.clone()
        out = ctx.cache_attention(cache, q, ints(*(length,) * B), max_length=length, accumulate=True)
        check(cache, q, out, before, (length,) * B, (n_q,) * B, dh ** -0.5)
    ctx.close()

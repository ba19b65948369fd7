"""Caches and rows that lie anywhere: weights and positions at every 4 bytes."""
import numpy as np
import pytest
import torch

from answer_helpers import bf16, context, fill, ints
from paper_2604_09244_amd import binding as mv
from test_gpu_cache_attention import check

pytestmark = pytest.mark.gpu


def shifted_cache(B, H_kv, dh, cap, shift):
    """A cache whose weights and positions start `shift` values behind an aligned address, and the whole arrays."""
    n = B * H_kv * cap
    weight, pos = torch.full((n + 8,), 3.0, device="cuda"), torch.full((n + 8,), -7, dtype=torch.int32, device="cuda")
    u8 = lambda k: torch.zeros(B, H_kv, cap, k, dtype=torch.uint8, device="cuda")  # noqa: E731
    view = lambda t: t[shift:shift + n].view(B, H_kv, cap)  # noqa: E731
    return mv.Cache4(u8(dh // 2), u8(dh // 2), u8(dh // 32), u8(dh // 32), view(pos), view(weight)), weight, pos


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("B,H,H_kv,dh,n_q,T", [(1, 2, 2, 64, 1, 40), (1, 1, 1, 128, 1, 5003), (1, 4, 2, 64, 3, 4098),
                                               (2, 2, 2, 128, 40, 333), (1, 1, 1, 64, 130, 301)])
def test_weights_at_any_four_bytes(B, H, H_kv, dh, n_q, T, shift):
    rng = np.random.default_rng(T)
    cap = (T + 31) // 32 * 32
    cache, weight, pos = shifted_cache(B, H_kv, dh, cap, shift)
    ctx = context(B, H, H_kv, n_q, cap, dh)
    fill(ctx, cache, bf16(rng, B, T, H_kv, dh), bf16(rng, B, T, H_kv, dh), (T,) * B)
    cache.weight[:, :, :T] = torch.rand(B, H_kv, T, device="cuda")
    q, before = bf16(rng, B, n_q, H, dh).cuda(), cache.weight.clone()
    print("case", B, H, H_kv, dh, n_q, T, shift, flush=True)
    out = ctx.cache_attention(cache, q, ints(*(T,) * B), max_length=T, accumulate=True)
    check(cache, q, out, before, (T,) * B, (n_q,) * B, dh ** -0.5)
    assert torch.equal(cache.weight[:, :, T:], before[:, :, T:])
    assert (weight[:shift] == 3).all() and (weight[shift + before.numel():] == 3).all()
    kept, new = ctx.cache_evict(cache, cache, ints(*(T,) * B), max(1, T // 2))
    assert (new == max(1, T // 2)).all() and (pos[:shift] == -7).all() and (pos[shift + before.numel():] == -7).all()
    ctx.close()

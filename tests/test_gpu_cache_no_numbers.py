"""Blocks that are no numbers in used slots: in every path of the attention they reach the rows that see them, and those
alone, outputs and weights."""
import numpy as np
import pytest
import torch

from answer_helpers import bf16, context, fill, garbage_cache, held, ints
from oracle import answering as A

pytestmark = pytest.mark.gpu
PATHS = [(1, 4, 2), (6, 2, 2), (30, 2, 2), (60, 2, 2), (20, 8, 2), (130, 2, 2), (300, 2, 2), (70, 6, 2)]   # n_q, H, H_kv


def build(rng, n_q, H, H_kv, dh, T, bad, keys):
    k, v = bf16(rng, 1, T, H_kv, dh), bf16(rng, 1, T, H_kv, dh)
    for slot, head, dim in bad:
        (k if keys else v)[0, slot, head, dim] = float("nan") if slot % 2 else float("inf")
    cap = (T + 31) // 32 * 32
    ctx, cache = context(1, H, H_kv, n_q, cap, dh), garbage_cache(1, H_kv, dh, cap)
    fill(ctx, cache, k, v, (T,))
    cache.weight[:, :, :T] = 0.5
    return ctx, cache, bf16(rng, 1, n_q, H, dh).cuda()


def sees(T, n_q):
    return np.arange(T)[None] <= (T - n_q + np.arange(n_q))[:, None]     # [query, slot]


def slots(T, n_q):
    """One slot that everybody sees, and some of the new ones: in several tiles, at tiles' ends and the last one."""
    new = {T - n_q + i for i in (1, 2, n_q // 2, n_q - 1) if 0 < i < n_q} | {T - 1}
    return [[s] for s in sorted({5} | new)] + [sorted(new)]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n_q,H,H_kv", PATHS)
def test_values(n_q, H, H_kv, dh):
    rng = np.random.default_rng(n_q + dh)
    T = n_q + 77
    for at in slots(T, n_q):
        bad = [(s, 1, (11 * s) % dh) for s in at]              # (of the second key head)
        ctx, cache, q = build(rng, n_q, H, H_kv, dh, T, bad, False)
        out = ctx.cache_attention(cache, q, ints(T), max_length=T, accumulate=True)[0]
        none = np.zeros((n_q, H, dh), bool)
        for s, g, d in bad:
            for h in range(g * H // H_kv, (g + 1) * H // H_kv):
                none[sees(T, n_q)[:, s], h, d // 32 * 32:d // 32 * 32 + 32] = True
        assert np.array_equal(out.isnan().cpu().numpy(), none), at
        kk, vv = held(cache, 0, T)
        ref, p = A.cache_attention(q[0].double().cpu().numpy(), kk, np.nan_to_num(vv), n_q, dh ** -0.5)
        reach = np.einsum("iht,htd->ihd", p, np.abs(np.repeat(np.nan_to_num(vv), H // H_kv, 0)))
        off = np.abs(out.double().cpu().numpy() - ref)
        assert np.all((off <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -7.9 * reach)[~none]), at
        add = p.reshape(n_q, H_kv, H // H_kv, T).sum((0, 2))
        got = cache.weight[0, :, :T].double().cpu().numpy() - 0.5
        assert np.all(np.abs(got - add) <= 1e-4 * add + 1e-6), at
        ctx.close()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n_q,H,H_kv", PATHS)
def test_keys(n_q, H, H_kv, dh):
    rng = np.random.default_rng(n_q + dh)
    T, group = n_q + 77, H // H_kv
    for at in slots(T, n_q):
        bad = [(s, 0, (7 * s) % dh) for s in at]
        ctx, cache, q = build(rng, n_q, H, H_kv, dh, T, bad, True)
        out = ctx.cache_attention(cache, q, ints(T), max_length=T, accumulate=True)[0]
        spoiled = sees(T, n_q)[:, at].any(-1)                  # queries whose sum of weights is none
        none = np.zeros((n_q, H, dh), bool)
        none[spoiled, :group] = True
        assert np.array_equal(out.isnan().cpu().numpy(), none), at
        weight = cache.weight[0, :, :T].isnan().cpu().numpy()
        assert np.array_equal(weight[0], sees(T, n_q)[spoiled].any(0)), at
        assert not weight[1:].any(), at
        ctx.close()

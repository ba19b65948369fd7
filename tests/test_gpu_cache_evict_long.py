"""Eviction from caches whose keys do not fit in LDS: by workgroups that copy their rows themselves, and by a second launch."""
import numpy as np
import pytest
import torch

from answer_helpers import context, ints
from test_gpu_cache_evict import NAMES, check, random_cache

pytestmark = pytest.mark.gpu


def parts(c):
    return {n: getattr(c, n).clone().cpu() for n in NAMES}


def some_heads(tensors, heads):
    return {n: t[:, heads] for n, t in tensors.items()}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "broken"])
@pytest.mark.parametrize("dh,length,budget", [(64, 17000, 300), (128, 16385, 512), (64, 33000, 1000), (128, 20000, 15000)])
def test_few_heads(dh, length, budget, kind, in_place):
    rng = np.random.default_rng(length)
    cap = (length + 31) // 32 * 32
    ctx = context(1, 1, 1, 1, cap, dh)
    src = random_cache(rng, 1, 1, dh, cap, kind)
    dst = src if in_place else random_cache(rng, 1, 1, dh, (budget + 31) // 32 * 32, "equal")
    before = parts(src)
    print("case", dh, length, budget, kind, in_place, flush=True)
    kept, new = ctx.cache_evict(src, dst, ints(length), budget, 40, ints(4 * cap - 100))
    check(before, parts(dst), kept.cpu(), new.cpu(), (length,), budget, 40, (4 * cap - 100,), in_place)
    if not in_place:
        assert all(torch.equal(t.nan_to_num(-3), before[n].nan_to_num(-3)) for n, t in parts(src).items())
    ctx.close()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
def test_many_heads(dh, in_place):
    """Enough workgroups that each copies its rows itself, whatever their number; some heads are looked at."""
    rng = np.random.default_rng(dh)
    H, length, budget = 224, 16500, 4000
    cap = (length + 31) // 32 * 32
    ctx = context(1, H, H, 1, cap, dh)
    src = random_cache(rng, 1, H, dh, cap, "ties")
    dst = src if in_place else random_cache(rng, 1, H, dh, 4000, "equal")
    before = parts(src)
    print("case", dh, in_place, flush=True)
    kept, new = ctx.cache_evict(src, dst, ints(length), budget, 7)
    heads = [0, 1, 100, 223]
    check(some_heads(before, heads), some_heads(parts(dst), heads), kept.cpu()[:, heads], new.cpu(), (length,), budget, 7, None,
          in_place)
    ctx.close()

"""Eviction at the ends of its arguments: positions up to the largest number."""
import numpy as np
import pytest
import torch

from answer_helpers import context, ints
from test_gpu_cache_evict import NAMES, check, random_cache

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("recent", [None, (MOST,), (MOST - 1,), (-2 ** 31,)])
@pytest.mark.parametrize("cap,budget", [(96, 40), (1056, 1000)])
def test_positions_up_to_the_largest_number(cap, budget, recent):
    """Without recent positions none is recent, the largest one neither."""
    rng = np.random.default_rng(cap)
    c = random_cache(rng, 1, 2, 64, cap, "spread")
    c.pos[:, :, ::3] = MOST
    c.pos[:, :, 1::7] = MOST - 1
    c.weight[:, :, ::3] *= 1e-6                 # (those would go)
    before = {n: getattr(c, n).clone().cpu() for n in NAMES}
    ctx = context(1, 2, 2, 1, cap, 64)
    kept, new = ctx.cache_evict(c, c, ints(cap), budget, 5, None if recent is None else ints(*recent))
    check(before, {n: getattr(c, n).cpu() for n in NAMES}, kept.cpu(), new.cpu(), (cap,), budget, 5, recent, True)
    ctx.close()

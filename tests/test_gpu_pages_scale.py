"""Attention over pages: the largest scale, and those beyond it, whose product with log2(e) fp32 does not hold."""
import numpy as np
import pytest
import torch

from pages_helpers import Case, f64
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EINVAL = -1


@pytest.mark.parametrize("count", [2, 40])
def test_largest_scale(count):
    c = Case(np.random.default_rng(count), 2, 1, 64, 16, 16, (80,), (count,))
    for scale in (2.4e38, 3.0e38, 3.4e38):
        with pytest.raises(mv.MvlaError) as e:
            c.ctx.pages_attention(c.cache, c.batch, c.q, scale=scale)
        assert e.value.code == EINVAL, scale
    # queries of zeros: every logit is zero, and all slots that a row sees count alike (one rounding of 1 / n, bf16's own)
    c.q.zero_()
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, scale=2.3e38, with_lse=True)
    _, v, _ = c.held(0)
    for i in range(count):
        sees = 80 - count + i + 1
        want, reach = v[0, :sees].mean(0), np.abs(v[0, :sees]).mean(0)
        assert np.all(np.abs(f64(out[i]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -16 * reach)
        assert torch.all((lse[i].double() - np.log(sees)).abs() <= 2.0 ** -22 * np.log(sees))

"""Log probabilities at the ends of their arguments' ranges (bars: test_gpu_logprobs)."""
import numpy as np
import pytest
import torch

from pages_helpers import ints
from paper_2604_09244_amd import binding as mv
from test_gpu_logprobs import check, ctx                            # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("half", [True, False])
def test_infinite_temperature(ctx, half):                           # noqa: F811
    """All logits above -infinity count alike; where some are +infinity, these alone."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((4, 3001)) * 3
    x[1, [5, 2000]] = INF
    x[2, ::2] = -INF
    x[3, :2990] = -INF
    x[3, 2995] = INF
    x = torch.from_numpy(x).to(torch.bfloat16 if half else torch.float32).cuda()
    tokens = np.tile([0, 5, 2000, 2995, 3000], (4, 1))
    check(ctx, x, tokens, [INF] * 4, 0)
    check(ctx, x, tokens, [INF] * 4, 7)


def test_no_rows(ctx):                                              # noqa: F811
    """A step with nothing to score: empty results, as of the other calls without rows."""
    x = torch.zeros(0, 100, device="cuda")
    lp, ent, tt, tl = ctx.logprobs(x, ints([]).view(0, 3), torch.zeros(0, device="cuda"), top=4)
    assert lp.shape == (0, 3) and ent.shape == (0,) and tt.shape == tl.shape == (0, 4)
    assert lp.dtype == ent.dtype == tl.dtype == torch.float32 and tt.dtype == torch.int32
    lp, ent, tt, tl = ctx.logprobs(x.bfloat16(), None)
    assert lp is None and ent.shape == (0,) and tt is None and tl is None
    with pytest.raises(AssertionError):
        ctx.logprobs(x, ints([1]))
    for logits, top in ((torch.zeros(2, 0, device="cuda"), 0), (x, 33)):      # (of no tokens; more than there are)
        with pytest.raises(mv.MvlaError):
            ctx.logprobs(logits, None, top=top)

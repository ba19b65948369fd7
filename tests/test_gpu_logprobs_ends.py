"""Log probabilities at the ends of their arguments' ranges (bars: test_gpu_logprobs)."""
import numpy as np
import pytest
import torch

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

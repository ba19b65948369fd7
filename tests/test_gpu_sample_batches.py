"""Token choice of more rows than its scratch holds at once: later turns take their own logits, settings and places."""
import numpy as np
import pytest
import torch

from answer_helpers import context

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("half", [True, False])
def test_many_long_rows(half):
    B, V = 1700, 33003
    g = torch.Generator(device="cuda").manual_seed(4)
    x = 2.0 * torch.randn(B, V, generator=g, device="cuda")
    x[torch.arange(B, device="cuda"), torch.arange(B, device="cuda") * 19] += 9.0
    x = x.to(torch.bfloat16 if half else torch.float32)
    row = torch.arange(B, device="cuda")
    u = torch.rand(B, generator=g, device="cuda")
    settings = (0.5 + 0.001 * row.float(), (row % 5 * 20).int(), torch.where(row % 3 == 0, 1.0, 0.6 + 0.0002 * row),
                torch.where(row % 4 == 0, 0.0, 1e-5 * row.float()))
    ctx = context(1, 1)
    token, prob = ctx.sample(x, u, *settings)
    for b in list(range(0, B, 83)) + [849, 850, 851, B - 1]:
        again, share = ctx.sample(x[b:b + 1], u[b:b + 1], *(s[b:b + 1] for s in settings))
        assert torch.equal(again, token[b:b + 1]) and torch.equal(share, prob[b:b + 1]), b
    few = ctx.sample(x, u, *settings, out=(torch.empty_like(token), None))
    assert torch.equal(few[0], token) and few[1] is None
    ctx.close()

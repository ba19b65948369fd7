"""Sums of weights are exact: neither token nor probability depends on where a row lies, on what is chosen beside it, or on
how its sums were formed."""
import numpy as np
import pytest
import torch

from answer_helpers import context
from test_gpu_sample import logits_of

pytestmark = pytest.mark.gpu
SETTINGS = [(1.0, 0, 0.0), (0.9, 0, 0.0), (0.999, 0, 0.0), (1.0, 1500, 0.0), (0.95, 1500, 0.0), (1.0, 0, 0.01), (0.97, 0, 0.001),
            (0.98, 3000, 0.0005), (1.0, 50, 0.0)]      # top_p, top_k, min_p


def choose(ctx, t, u, p, k, least, temperature=None):
    B = len(t)
    full = lambda v, dt=torch.float32: torch.full((B,), v, dtype=dt, device="cuda")  # noqa: E731
    return [x.clone() for x in ctx.sample(t, u, full(temperature or 1.0), full(k, torch.int32), full(p), full(least))]


@pytest.mark.parametrize("kind", ["plain", "ties"])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("p,k,least", SETTINGS)
def test_one_row_as_in_a_batch(p, k, least, half, kind):
    """Slices are shorter where rows are few, and top_k of 1500 takes a list of tokens there, the whole row here."""
    rng = np.random.default_rng(29)
    B, V = 90, 100003
    t = torch.from_numpy(logits_of(rng, B, V, kind)).to(torch.bfloat16 if half else torch.float32).cuda()
    ctx, u = context(1, 1), torch.rand(B, generator=torch.Generator().manual_seed(5)).cuda()
    token, prob = choose(ctx, t, u, p, k, least)
    for b in range(0, B, 7):
        again, share = choose(ctx, t[b:b + 1], u[b:b + 1], p, k, least)
        assert torch.equal(again, token[b:b + 1]) and torch.equal(share, prob[b:b + 1]), b
    ctx.close()


@pytest.mark.parametrize("V", [5003, 20011, 50021])
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("p,k,least", SETTINGS)
def test_a_row_that_lies_elsewhere(p, k, least, half, V):
    """The 16 bytes that are read together start at another token."""
    rng = np.random.default_rng(V)
    B, dt = 12, torch.bfloat16 if half else torch.float32
    rows = torch.from_numpy(logits_of(rng, B, V, "plain")).to(dt).cuda()
    ctx, u = context(1, 1), torch.rand(B, generator=torch.Generator().manual_seed(7)).cuda()
    want = choose(ctx, rows, u, p, k, least)
    for offset in range(1, 8 if half else 4):
        wide = torch.zeros(B, V + 8, dtype=dt, device="cuda")      # (rows start at different places of 16 bytes)
        wide[:, offset:offset + V] = rows
        got = choose(ctx, wide[:, offset:offset + V], u, p, k, least)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), offset
    ctx.close()


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("p,k,least", SETTINGS)
def test_tokens_that_cannot_be_chosen_change_nothing(p, k, least, half):
    """One workgroup's row, and the same one with forbidden tokens behind it, which several take."""
    rng = np.random.default_rng(31)
    B, V = 16, 30011
    rows = torch.from_numpy(logits_of(rng, B, V, "plain")).to(torch.bfloat16 if half else torch.float32).cuda()
    longer = torch.full((B, 90000), -float("inf"), dtype=rows.dtype, device="cuda")
    longer[:, :V] = rows
    ctx, u = context(1, 1), torch.rand(B, generator=torch.Generator().manual_seed(9)).cuda()
    a, b = choose(ctx, rows, u, p, k, least), choose(ctx, longer, u, p, k, least)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ctx.close()


def test_weights_down_to_the_last_unit():
    """Weights near 2^-40 of the largest, thousands of them: each counts as the nearest whole number of units, so sums that
    are formed here and there agree."""
    B, V = 8, 40009
    octaves = torch.linspace(38.0, 42.5, V, dtype=torch.float64)
    x = (-octaves * np.log(2.0)).float().repeat(B, 1)
    x[:, 17] = 0.0
    x = x.cuda()
    u = torch.tensor([0.0, 0.5, 0.99, 0.999999, 1.0, 0.25, 0.75, 0.9], device="cuda")
    ctx = context(1, 1)
    for p, k, least in ((1.0, 0, 0.0), (0.99999994, 0, 0.0), (1.0, 30000, 0.0), (0.99999994, 39000, 0.0)):
        token, prob = choose(ctx, x, u, p, k, least)
        for b in range(B):
            again, share = choose(ctx, x[b:b + 1], u[b:b + 1], p, k, least)
            assert torch.equal(again, token[b:b + 1]) and torch.equal(share, prob[b:b + 1]), (p, k, b)
        short = x[:, :32000].clone()
        longer = torch.full((B, 90000), -float("inf"), device="cuda")
        longer[:, :32000] = short
        a, c = choose(ctx, short, u, p, min(k, 31000), least), choose(ctx, longer, u, p, min(k, 31000), least)
        assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1]), (p, k)
    ctx.close()

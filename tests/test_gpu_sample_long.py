"""Token choice on rows that are dealt out over several workgroups (bounds as in test_gpu_sample.py)."""
import numpy as np
import pytest
import torch

from answer_helpers import context
from test_gpu_sample import logits_of, run_and_check, settle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["plain", "masked", "ties", "signs"])
@pytest.mark.parametrize("V,half", [(32769, False), (65537, True), (131077, True), (200003, False)])
def test_settings_by_row(V, half, kind):
    rng = np.random.default_rng(V + len(kind))
    B = 14
    t = torch.from_numpy(logits_of(rng, B, V, kind)).to(torch.bfloat16 if half else torch.float32)
    rows = t.double().numpy()
    f32 = np.float32
    temperature = np.array([0.0] + [0.3, 0.8, 1.0, 2.5] * 3 + [1.0], f32)
    top_k = np.array([0, 0, 0, 0, 0, 1, 7, 300, 2000, 0, 0, 0, V, 50])
    top_p = np.array([1.0, 0.1, 0.55, 0.9, 0.997, 1.0, 0.9, 0.8, 0.99, 1.0, 1.0, 0.9, 0.95, 1.0], f32)
    min_p = np.array([0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.01, 0.0, 0.013, 0.5, 0.02, 0.0, 0.1], f32)
    u = settle(rows, rng.random(B), temperature, top_k, top_p, min_p)
    ctx = context(1, 1)
    run_and_check(ctx, t.cuda(), rows, u, temperature, top_k, top_p, min_p)
    ctx.close()


@pytest.mark.parametrize("half", [True, False])
def test_the_longest_rows(half):
    """A slice's threads walk several times over their share."""
    rng = np.random.default_rng(5)
    B, V = 4, 1 << 22
    t = torch.from_numpy(rng.standard_normal((B, V)).astype(np.float32) * 2)
    t[:, ::V // 97] += 14.0
    t = t.to(torch.bfloat16) if half else t
    rows = t.double().numpy()
    temperature, top_k = np.array([1.0, 0.7, 1.0, 0.5], np.float32), np.array([0, 100, 0, 0])
    top_p, min_p = np.array([0.6, 0.9, 1.0, 1.0], np.float32), np.array([0.0, 0.0, 0.0, 0.02], np.float32)
    u = settle(rows, np.array([0.1, 0.5, 0.02, 0.7]), temperature, top_k, top_p, min_p)
    ctx = context(1, 1)
    run_and_check(ctx, t.cuda(), rows, u, temperature, top_k, top_p, min_p)
    ctx.close()


def test_infinities_and_no_numbers_in_some_slices():
    inf, nan, V = float("inf"), float("nan"), 70001
    x = torch.zeros(8, V, device="cuda")
    x[0] = -inf
    x[1] = nan
    x[2], x[2, 69000] = nan, 1.0
    x[3, 5] = x[3, 68000] = inf                    # the infinite ones alone, whatever the others are
    x[4], x[4, 40000] = -inf, -5.0
    x[5, :30000], x[5, 30000:], x[5, 66000] = nan, -inf, inf
    x[6, :60000], x[6, 60000:] = -3e38, -inf       # weights that are none beside the largest
    x[6, 59999] = 3e38
    x[7, :35000] = nan
    x[7, 35000:] = -inf
    x[7, 35001] = x[7, 70000] = -1.0
    u = torch.tensor([0.5, 0.5, 0.5, 0.7, 0.99, 0.3, 0.9, 0.6], device="cuda")
    k = torch.full((8,), 2, dtype=torch.int32, device="cuda")
    p, some = torch.full((8,), 0.9, device="cuda"), torch.full((8,), 0.1, device="cuda")
    ctx = context(1, 1)
    for t in (x, x.to(torch.bfloat16)):
        for args in ((), (None, k), (None, None, p), (None, k, p, some), (None, None, None, some), (None, None, p, some)):
            token, prob = ctx.sample(t, u, *args)
            assert token.tolist() == [-1, -1, 69000, 68000, 40000, 66000, 59999, 70000], args
            assert prob.tolist() == [0.0, 0.0, 1.0, 0.5, 1.0, 1.0, 1.0, 0.5], args
        token, prob = ctx.sample(t, u, torch.zeros(8, device="cuda"))
        assert token.tolist() == [-1, -1, 69000, 5, 40000, 66000, 59999, 35001]
        # every token weighs the same
        hot = torch.full((8,), inf, device="cuda")
        token, prob = ctx.sample(t[6:], u[6:], hot[6:])
        assert token.tolist() == [int(float(np.float32(0.9)) * 60000), 70000] and np.allclose(prob.tolist(), [1 / 60000, 0.5])
    ctx.close()


def test_the_same_choice_every_time_whatever_the_batch():
    """Slices are shorter while rows are few: nothing that is chosen depends on them."""
    rng = np.random.default_rng(17)
    t = torch.from_numpy(logits_of(rng, 90, 100003, "plain")).to(torch.bfloat16).cuda()
    ctx = context(1, 1)
    u = torch.rand(90, generator=torch.Generator().manual_seed(3)).cuda()
    for p, k in ((0.9, 0), (0.97, 40), (1.0, 0)):
        p, k = torch.full((90,), p, device="cuda"), torch.full((90,), k, dtype=torch.int32, device="cuda")
        token, prob = [x.clone() for x in ctx.sample(t, u, None, k, p)]
        for b0, b1 in ((0, 1), (1, 7), (30, 90)):
            again, share = ctx.sample(t[b0:b1], u[b0:b1], None, k[b0:b1], p[b0:b1])
            assert torch.equal(again, token[b0:b1]) and torch.equal(share, prob[b0:b1])
    ctx.close()

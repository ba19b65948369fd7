"""Attention over pages where logits are finite and far from zero.

Inputs whose logits fp32 holds exactly.  Near ones: a constant from dim 0 (2^10 times 2^7 to 2560, either sign), and from dim 32
(another block of the cache in 8 bits) 1 times a number of at most four bits between -7 and 7; the sum is a multiple of a
quarter below 2^24 of them.  Apart ones: one dim alone, a product of two bf16 numbers.

Bars.  A logit is exact, its distance from a reference too (14 at most; the reference only rises, so all its moves together are
as much).  The power's argument has the roundings of log2 e and of the product, 2 2^-24 of 14 log2(e) either way, and the power
2^-20: an exponential is off by a share of 2^-17.5 at most, and an output by twice that, 2^-16, beside the rounding of each probability
to bf16 and its own.  A log-sum adds its own roundings, as pages_helpers has them.  Where logits are apart, one (or its
equals) has everything."""
import numpy as np
import pytest
import torch

from oracle import many_prompts as M
from pages_helpers import Case, bf16, f64

pytestmark = pytest.mark.gpu
SHARE = 2.0 ** -16


def near(case, out, lse, scale):
    q, got, got_lse = f64(case.q), f64(out), f64(lse)
    for b, (t, c) in enumerate(zip(case.lengths, case.counts)):
        k, v, there = case.held(b)
        k, v, there = k[:, :t], v[:, :t], there[:t]
        at = slice(case.starts[b], case.starts[b] + c)
        want, want_lse, p = M.attention(q[at], k, v, t, scale, there)
        reach = np.einsum("iht,htd->ihd", p, np.abs(np.repeat(v, case.H // case.H_kv, 0)))
        err = np.abs(got[at] - want)
        assert np.all(err <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + SHARE) * reach + 2.0 ** -126), (b, err.max())
        err = np.abs(got_lse[at] - want_lse)
        assert np.all(err <= SHARE + 2.0 ** -22 * np.abs(want_lse)), (b, err.max())


FEW = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("counts,lengths", [((3, 1), (90, 700)), ((40, 33), (300, 64)), ((1, 1), (5000, 40)), ((60, 1), (5000, 2049))])
@pytest.mark.parametrize("far", [2.0 ** 7, -2.0 ** 11, 2560.0])
def test_near_each_other(far, counts, lengths, dh, bits):
    rng = np.random.default_rng(dh + bits + counts[0])
    H, T = 2, max(lengths)
    k = np.zeros((2, T, 1, dh))
    k[..., 0] = far
    k[..., 32] = rng.choice(FEW, (2, T, 1)) * rng.choice([-1.0, 1.0], (2, T, 1))
    k = torch.from_numpy(k).to(torch.bfloat16)
    # (values all of one sign: that nothing cancels what is off)
    c = Case(rng, H, 1, dh, 16, bits, lengths, counts, k=k, v=bf16(rng, 2, T, 1, dh).abs())
    c.q.zero_()
    c.q[..., 0], c.q[..., 32] = 1024.0, 1.0
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=max(counts), max_length=T, scale=1.0, with_lse=True)
    near(c, out, lse, 1.0)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("counts,lengths", [((3, 1), (90, 700)), ((40, 33), (300, 64)), ((60, 1), (5000, 2049))])
@pytest.mark.parametrize("size", [3.0e10, 1.0e12, 1.0e30])
def test_apart(size, counts, lengths, dh, bits):
    """Either sign; a tenth of the keys are the same one."""
    rng = np.random.default_rng(dh + bits + counts[0])
    T, scale = max(lengths), dh ** -0.5
    k = np.zeros((2, T, 2, dh))
    k[..., 5] = rng.uniform(1.0, 2.0, (2, T, 2)) * rng.choice([-1.0, 1.0], (2, T, 2))
    k[..., 5] = np.where(rng.random((2, T, 2)) < 0.1, 1.9375, k[..., 5])
    k = torch.from_numpy(k).to(torch.bfloat16)
    c = Case(rng, 4, 2, dh, 16, bits, lengths, counts, k=k, v=bf16(rng, 2, T, 2, dh).abs())
    q = rng.uniform(1.0, 2.0, (c.n, 4)) * size * rng.choice([-1.0, 1.0], (c.n, 4))
    c.q.zero_()
    c.q[..., 5] = torch.from_numpy(q).to(torch.bfloat16).cuda()
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=max(counts), max_length=T, with_lse=True)
    near(c, out, lse, scale)

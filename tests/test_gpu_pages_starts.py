"""Attention over pages with starts that do not ascend or lie outside: rows of one sequence alone are right, rows of none stay
as they were; sequences that share rows and all else write what each would alone."""
import numpy as np
import pytest
import torch

from oracle import many_prompts as M
from pages_helpers import Case, check, f64, ints
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,dh", [(16, 64), (8, 128)])
@pytest.mark.parametrize("start", [[0, 20, 10, 60], [60, 40, 20, 0], [-5, 20, 40, 99], [0, 2 ** 31 - 1, -2 ** 31, 60], [0, 3, 1, 60], [55, 60, 50, 58]])
def test_rows_of_one_sequence(start, bits, dh):
    rng = np.random.default_rng(5)
    c = Case(rng, 2, 2, dh, 16, bits, (40, 50, 60), (20, 20, 20))
    out = torch.full((60, 2, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((60, 2), 7.0, device="cuda")
    c.ctx.pages_attention(c.cache, mv.PageBatch(ints(start), c.batch.length, c.batch.table), c.q, with_lse=True, out=(out, lse))
    begin, end = np.clip(start[:-1], 0, 60), np.clip(start[1:], 0, 60)
    owners = np.array([[b <= i < e for b, e in zip(begin, end)] for i in range(60)]).sum(1)
    assert torch.all(out[owners == 0] == 7) and torch.all(lse[owners == 0] == 7)
    q, seen = f64(c.q), 0
    for b in range(3):
        rows = [i for i in range(begin[b], end[b]) if owners[i] == 1]
        if not rows:
            continue
        k, v, there = (x[..., :c.lengths[b], :] if x.ndim > 1 else x[:c.lengths[b]] for x in c.held(b))
        at = np.array(rows) - begin[b]
        want, want_lse, p = (x[at] for x in M.attention(q[begin[b]:end[b]], k, v, c.lengths[b], dh ** -0.5, there))
        # (bars: pages_helpers)
        size = dh ** -0.5 * np.max(np.einsum("ihd,htd->iht", np.abs(q[rows]), np.abs(k)))
        share = 2 * size * (dh + 4) * 2.0 ** -24 + 2.0 ** -20
        reach = np.einsum("iht,htd->ihd", p, np.abs(v))
        assert np.all(np.abs(f64(out[rows]) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + share) * reach + 2.0 ** -126), b
        none, got = np.isneginf(want_lse), f64(lse[rows])
        assert np.array_equal(np.isneginf(got), none) and np.all(np.abs(got - want_lse)[~none] <= share + 2.0 ** -22 * np.abs(want_lse[~none]))
        seen += len(rows)
    assert seen == (owners == 1).sum()


@pytest.mark.parametrize("bits", [16, 8])
def test_more_blocks_of_rows_than_workgroups(bits):
    """Six sequences that are one and the same, in the same rows: more blocks than the rows of the call make, so that
    workgroups take several, one behind the other."""
    rng = np.random.default_rng(8)
    n, T, H = 300, 320, 64
    c = Case(rng, H, H, 64, 16, bits, (T,), (n,))
    start = [0, n] * 6 + [0]
    batch = mv.PageBatch(ints(start), ints([T] * 12), c.batch.table.repeat(12, 1))
    ctx = mv.Context.for_pages(12, H, H, n, n, T, 64)
    out, lse = ctx.pages_attention(c.cache, batch, c.q, max_q=n, max_length=T, with_lse=True)
    check(c, out, lse, 0.125)

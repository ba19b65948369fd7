"""Shared plumbing of the tests of the cache in pages (no arithmetic of the HIP path)."""
import numpy as np
import torch

from oracle import many_prompts as M
from paper_2604_09244_amd import binding as mv


def bf16(rng, *shape, scale=1.0):
    """Normal values that bf16 holds, as a CPU tensor."""
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def garbage_pool(n_pages, H_kv, dh, page, bits):
    """A pool whose every byte is 0xff: values, codes and powers that are no numbers."""
    c = mv.PagedCache.empty(n_pages, H_kv, dh, page, bits)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(255)
    return c


def deal(rng, lengths, page, spare=2, entries=None):
    """Pages for sequences of these lengths in any order: (pages in the pool, table [B, entries] with -1 behind)."""
    per = [-(-t // page) for t in lengths]
    n = sum(per) + spare
    order = rng.permutation(n)
    table = np.full((len(lengths), entries or max(max(per), 1)), -1, np.int32)
    at = 0
    for b, m in enumerate(per):
        table[b, :m] = order[at:at + m]
        at += m
    return n, table


class Case:
    """Sequences of `lengths` slots, the last `counts` of them new, their rows written into a pool of garbage."""

    def __init__(self, rng, H, H_kv, dh, page, bits, lengths, counts, entries=None, k=None, v=None, spread=1.0, front=0, behind=0):
        self.lengths, self.counts, self.dh, self.H, self.H_kv = lengths, counts, dh, H, H_kv
        B, T = len(lengths), max(max(lengths), 1)
        self.n_pages, self.table = deal(rng, lengths, page, entries=entries)
        self.cache = garbage_pool(self.n_pages, H_kv, dh, page, bits)
        starts = front + np.concatenate([[0], np.cumsum(counts)])
        self.n = int(starts[-1]) + behind
        self.starts = starts.astype(int)
        self.batch = mv.PageBatch(ints(starts.tolist()), ints(lengths), torch.from_numpy(self.table).cuda())
        self.ctx = mv.Context.for_pages(B, H, H_kv, max(self.n, 1), max(max(counts), 1), T, dh)
        self.k = bf16(rng, B, T, H_kv, dh, scale=spread) if k is None else k
        self.v = bf16(rng, B, T, H_kv, dh) if v is None else v
        # every row by one append, packed
        at = np.concatenate([[0], np.cumsum(lengths)])
        if at[-1]:
            rows = lambda x: torch.cat([x[b, :t] for b, t in enumerate(lengths)]).cuda()
            self.ctx.pages_append(self.cache, mv.PageBatch(ints(at.tolist()), self.batch.length, self.batch.table), rows(self.k), rows(self.v))
        self.q = bf16(rng, max(self.n, 1), H, dh, scale=1.3).cuda()[:self.n]

    def held(self, b):
        """What the pool holds of sequence b: k, v [H_kv, slots, dh] (slots of all table entries), which slots have a page."""
        c, page = self.cache, self.cache.page
        out, there = [], np.repeat((self.table[b] >= 0) & (self.table[b] < self.n_pages), page)
        at = torch.from_numpy(np.clip(self.table[b], 0, self.n_pages - 1).astype(np.int64)).cuda()
        for x, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
            rows = x[at].transpose(0, 1).flatten(1, 2)
            out.append(f64(rows) if s is None else M.fp8_decode(rows.cpu().numpy(), s[at].transpose(0, 1).flatten(1, 2).cpu().numpy()))
        return out[0], out[1], there


def check(case, out, lse, scale, max_q=None, starts=None):
    """Bars, from the arithmetic: products of bf16 queries with the cache's exact values, summed in fp32 (dh additions), put a
    logit off by at most dh 2^-24 of scale sum |q k|, its exponential by twice that as a share; exp2 and its argument
    add 2^-20.  A log-sum is off by that share and by its own rounding.  An output adds the rounding of each probability to
    bf16 (2^-8 of sum p |v|) and its own (2^-8 of itself); what lies below the smallest normal number may be lost."""
    starts = case.starts if starts is None else starts
    q, got, got_lse = f64(case.q), f64(out), f64(lse)
    group, dh = case.H // case.H_kv, case.dh
    for b, (t, c) in enumerate(zip(case.lengths, case.counts)):
        if c == 0:
            continue
        k, v, there = case.held(b)
        rows = slice(starts[b], starts[b] + min(c, max_q or c))
        k, v = np.where(there[None, :, None], k, 0.0), np.where(there[None, :, None], v, 0.0)
        qb = q[starts[b]:starts[b] + c]
        want, want_lse, p = M.attention(qb, k, v, t, scale, there)
        want, want_lse, p = want[:rows.stop - rows.start], want_lse[:rows.stop - rows.start], p[:rows.stop - rows.start]
        kk, vv = np.repeat(k[:, :t], group, 0), np.repeat(v[:, :t], group, 0)
        size = scale * np.max(np.einsum("ihd,htd->iht", np.abs(qb), np.abs(np.nan_to_num(kk))), initial=0.0)
        share = 2 * size * (dh + 4) * 2.0 ** -24 + 2.0 ** -20
        reach = np.einsum("iht,htd->ihd", p[..., :t], np.abs(np.nan_to_num(vv)))
        lost = 2.0 ** -126 * (1 + np.abs(np.nan_to_num(vv)).sum(1))
        fine = np.isfinite(want)
        err = np.where(fine, np.abs(got[rows] - want), 0.0)
        assert np.all(err <= np.where(fine, 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + share) * reach + lost, 1.0)), (b, err.max())
        assert np.array_equal(np.isnan(got[rows]), np.isnan(want)) and np.array_equal(np.isinf(got[rows]), np.isinf(want)), b
        none = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse[rows]), none) and not got[rows][none].any(), b
        ok = np.isfinite(want_lse)
        err = np.abs(got_lse[rows][ok] - want_lse[ok])
        assert np.all(err <= share + 2.0 ** -22 * np.abs(want_lse[ok])), (b, err.max())

"""Attention over pages against its definition in fp64 on the values that the pool's bytes stand for (bars: pages_helpers)."""
import numpy as np
import pytest
import torch

from oracle import many_prompts as M
from pages_helpers import Case, bf16, check, f64, ints
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EINVAL, EUNSUPPORTED = -1, -4

CASES = [  # H, H_kv, dh, page, lengths, counts
    (1, 1, 64, 16, (1,), (1,)), (1, 1, 128, 16, (1,), (1,)), (4, 4, 128, 16, (0, 3, 31), (0, 1, 1)),
    (2, 1, 128, 32, (33, 127, 129, 16), (1, 1, 1, 1)), (8, 1, 64, 64, (257, 5), (2, 1)), (16, 1, 128, 16, (300, 64), (1, 1)),
    (3, 3, 64, 16, (5, 40), (5, 7)),
    (2, 2, 128, 16, (3, 100), (9, 16)),                     # more new rows than rows: the first see nothing
    (2, 2, 64, 16, (17, 200), (17, 17)),                    # one row more than a wave's 16
    (34, 2, 64, 32, (90, 1), (1, 1)),                       # a group of 17: many rows for one token
    (1, 1, 128, 64, (64, 65, 63, 128), (64, 65, 63, 100)),
    (4, 2, 128, 16, (200, 7, 333, 0, 90), (130, 1, 3, 0, 33)),   # a chunk beside next tokens
    (2, 1, 64, 128, (700, 129), (300, 129)), (1, 1, 128, 256, (520,), (257,)),
    (6, 2, 128, 32, (40, 41, 42), (8, 40, 5)),
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,H_kv,dh,page,lengths,counts", CASES)
def test_attention(H, H_kv, dh, page, lengths, counts, bits):
    rng = np.random.default_rng(sum(lengths) + dh + bits)
    c = Case(rng, H, H_kv, dh, page, bits, lengths, counts)
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=max(counts), max_length=max(max(lengths), 1), with_lse=True)
    check(c, out, lse, dh ** -0.5)
    again = c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=max(counts), max_length=max(max(lengths), 1))
    assert torch.equal(out, again)
    # bounds that are not tight, another scale
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, scale=0.3, with_lse=True)
    check(c, out, lse, 0.3)


@pytest.mark.parametrize("bits,dh,count", [(16, 128, 1), (8, 64, 1), (16, 128, 40), (8, 128, 40), (16, 64, 200), (8, 64, 40)])
def test_long_sequences_in_parts(bits, dh, count):
    """Sequences that are split over workgroups, lengths that differ, logits of tens."""
    rng = np.random.default_rng(count + dh)
    c = Case(rng, 2, 1, dh, 64, bits, (5000, 1300, 64, 2049), (count, 1, 1, count), spread=3.0)
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=count, max_length=5000, with_lse=True)
    check(c, out, lse, dh ** -0.5)
    # a context with the least workspace: the same call, in as many parts as fit
    small = mv.Context.for_pages(1, 1, 1, 1, 1, 1, 64)
    again, lse = small.pages_attention(c.cache, c.batch, c.q, max_q=count, max_length=5000, with_lse=True)
    check(c, again, lse, dh ** -0.5)


def test_more_sequences_than_a_wave_counts():
    """150 sequences: next tokens, chunks and none, in one call."""
    rng = np.random.default_rng(7)
    lengths = [int(x) for x in rng.integers(0, 120, 150)]
    counts = [min(t, int(rng.choice([0, 1, 1, 2, 30, 70]))) for t in lengths]
    c = Case(rng, 2, 1, 64, 16, 16, lengths, counts)
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=max(counts), with_lse=True)
    check(c, out, lse, 0.125)


@pytest.mark.parametrize("count", [3, 50])
def test_rows_that_are_nobodys(count):
    """Rows before the first and behind the last sequence, and rows from max_q on, stay as they were; logits of lengths
    beyond max_length do not exist."""
    rng = np.random.default_rng(count)
    c = Case(rng, 2, 2, 64, 16, 16, (90, 70), (count, count), front=3, behind=4)
    out = torch.full((c.n, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.n, 2), 7.0, device="cuda")
    c.ctx.pages_attention(c.cache, c.batch, c.q, with_lse=True, out=(out, lse))
    check(c, out, lse, 0.125)
    for t in (out, lse):
        assert torch.all(t[:3] == 7) and torch.all(t[-4:] == 7)
    most = count - 2
    out.fill_(7), lse.fill_(7)
    c.ctx.pages_attention(c.cache, c.batch, c.q, max_q=most, with_lse=True, out=(out, lse))
    check(c, out, lse, 0.125, max_q=most)
    for b in range(2):
        assert torch.all(out[c.starts[b] + most:c.starts[b + 1]] == 7)
    out.fill_(7), lse.fill_(7)
    c.ctx.pages_attention(c.cache, c.batch, c.q, max_length=64, with_lse=True, out=(out, lse))
    c.lengths = [64, 64]
    check(c, out, lse, 0.125)


@pytest.mark.parametrize("count", [2, 40])
@pytest.mark.parametrize("bits", [16, 8])
def test_pages_that_are_none(count, bits):
    """Numbers out of range within a sequence: its slots have no part; a sequence with no page at all gives zeros."""
    rng = np.random.default_rng(bits + count)
    c = Case(rng, 2, 1, 128, 16, bits, (200, 150, 90), (count, count, count))
    bad = c.table.copy()
    bad[0, 3], bad[0, 12], bad[1, 1], bad[1, 9] = -1, c.n_pages, 2 ** 31 - 1, -2 ** 31
    bad[2] = -5
    c.table = bad
    c.batch = mv.PageBatch(c.batch.start, c.batch.length, torch.from_numpy(bad).cuda())
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, with_lse=True)
    check(c, out, lse, 128 ** -0.5)
    assert not out[c.starts[2]:].any() and torch.all(lse[c.starts[2]:] == -float("inf"))


@pytest.mark.parametrize("count", [4, 70])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("bits", [16, 8])
def test_values_that_are_no_numbers(count, dh, bits):
    """An infinity or NaN among the new tokens' values reaches the rows that see it, in its dims, and not the rows before."""
    rng = np.random.default_rng(count + dh)
    lengths = (100, 130)
    k, v = bf16(rng, 2, 130, 2, dh), bf16(rng, 2, 130, 2, dh)
    inf = float("inf")
    v[0, 98, 0, 5], v[0, 99, 1, 33], v[1, 128, 0, 2], v[1, 129, 0, 2] = inf, float("nan"), inf, -inf
    v[0, 97, 1, dh - 1] = -inf
    if count > 60:
        v[1, 75, 1, 40], v[0, 40, 0, 11] = -inf, inf
    c = Case(rng, 4, 2, dh, 16, bits, lengths, (count, count), k=k, v=v)
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, with_lse=True)
    check(c, out, lse, dh ** -0.5)
    assert torch.isnan(out).any() and torch.isfinite(out[c.starts[1] - 4]).any()


@pytest.mark.parametrize("count", [4, 70])
def test_keys_that_are_no_numbers(count):
    """A key of NaN makes the rows that see it NaN; logits of -infinity alone give zeros, +infinity NaN, as a softmax has it."""
    rng = np.random.default_rng(count)
    k, v = bf16(rng, 3, 90, 1, 64), bf16(rng, 3, 90, 1, 64)
    k[0, 89] = float("nan")
    c = Case(rng, 1, 1, 64, 16, 16, (90, 90, 90), (count, count, count), k=k, v=v)
    c.q[c.starts[1]:] = c.q[c.starts[1]:].abs()
    pool = c.cache.k.view(c.n_pages, 16, 64)
    for b, x in ((1, -float("inf")), (2, float("inf"))):
        for p in c.table[b][c.table[b] >= 0]:
            pool[int(p)] = x
    out, lse = c.ctx.pages_attention(c.cache, c.batch, c.q, with_lse=True)
    last = c.starts[1] - 1
    assert torch.isnan(out[last]).all() and torch.isnan(lse[last]).all() and torch.isfinite(out[:last]).all()
    assert not out[c.starts[1]:c.starts[2]].any() and torch.all(lse[c.starts[1]:c.starts[2]] == -float("inf"))
    assert torch.isnan(out[c.starts[2]:]).all()


@pytest.mark.parametrize("count", [3, 40])
def test_views_and_shared_pages(count):
    """Queries inside a projection's rows, outputs transposed; sequences that share their first pages."""
    rng = np.random.default_rng(count)
    c = Case(rng, 4, 2, 64, 16, 16, (80, 80), (count, count))
    c.table[1, :2] = c.table[0, :2]
    c.batch = mv.PageBatch(c.batch.start, c.batch.length, torch.from_numpy(c.table).cuda())
    wide = torch.zeros(c.n, 8, 64, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:6] = c.q
    out = torch.zeros(4, c.n, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    lse = torch.zeros(c.n, 4, device="cuda")
    c.ctx.pages_attention(c.cache, c.batch, wide[:, 2:6], with_lse=True, out=(out, lse))
    check(c, out, lse, 0.125)


def test_far_pages():
    """A pool of more than 2^32 bytes: rows behind it are read and written where they are."""
    dh, page, H_kv = 128, 256, 8
    n_pages = (1 << 32) // (H_kv * page * dh * 2) + 40
    cache = mv.PagedCache.empty(n_pages, H_kv, dh, page, 16)
    rng = np.random.default_rng(1)
    table = np.array([[n_pages - 1, n_pages - 3], [n_pages - 2, n_pages - 5]], np.int32)
    batch = mv.PageBatch(ints([0, 40, 41]), ints([300, 290]), torch.from_numpy(table).cuda())
    ctx = mv.Context.for_pages(2, H_kv, H_kv, 41, 40, 512, dh)
    k, v = (bf16(rng, 590, H_kv, dh).cuda() for _ in range(2))
    ctx.pages_append(cache, mv.PageBatch(ints([0, 300, 590]), batch.length, batch.table), k, v)
    kr, vr = ctx.pages_read(cache, batch, None, 290)
    assert torch.equal(kr[0].transpose(0, 1), k[:290]) and torch.equal(vr[1].transpose(0, 1), v[300:])
    q = bf16(rng, 41, H_kv, dh).cuda()
    out = ctx.pages_attention(cache, batch, q, max_q=40)
    near = mv.PagedCache(cache.k[n_pages - 8:].clone(), cache.v[n_pages - 8:].clone())
    moved = mv.PageBatch(batch.start, batch.length, torch.from_numpy(table - (n_pages - 8)).cuda())
    assert torch.equal(out, ctx.pages_attention(near, moved, q, max_q=40))


def test_starts_out_of_order():
    """Starts that do not ascend or lie outside: no fault, and sequences that are whole are right."""
    rng = np.random.default_rng(5)
    c = Case(rng, 2, 2, 64, 16, 16, (40, 50, 60), (20, 20, 20))
    for start in ([0, 20, 10, 60], [60, 40, 20, 0], [-5, 20, 40, 99], [0, 2 ** 31 - 1, -2 ** 31, 60]):
        batch = mv.PageBatch(ints(start), c.batch.length, c.batch.table)
        out, lse = c.ctx.pages_attention(c.cache, batch, c.q, with_lse=True)
        torch.cuda.synchronize()
        assert out.shape == c.q.shape


def test_empty_calls_and_refusals():
    rng = np.random.default_rng(6)
    c = Case(rng, 4, 2, 64, 16, 16, (40,), (4,))
    assert c.ctx.pages_attention(c.cache, c.batch, c.q[:0]).shape == (0, 4, 64)
    for kw, code in ((dict(max_q=0), EINVAL), (dict(max_length=0), EINVAL), (dict(max_length=100), EINVAL), (dict(scale=0.0), EINVAL),
                     (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=-1.0), EINVAL)):
        with pytest.raises(mv.MvlaError) as e:
            c.ctx.pages_attention(c.cache, c.batch, c.q, **kw)
        assert e.value.code == code, kw
    odd = torch.zeros(4 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    for q in (odd[1:1 + 4 * 4 * 64].view(4, 4, 64), odd[:4 * 4 * 64].view(4, 64, 4).transpose(1, 2), c.q[:, :3]):
        with pytest.raises(mv.MvlaError) as e:
            c.ctx.pages_attention(c.cache, c.batch, q)
        assert e.value.code == EINVAL
    for q in (c.q.float(), c.q.cpu(), c.q[..., :32]):
        with pytest.raises(AssertionError):
            c.ctx.pages_attention(c.cache, c.batch, q)

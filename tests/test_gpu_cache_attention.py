"""Attention over the 4-bit cache against its definition in fp64 on the values that the cache's bytes stand for.

Bars, from the arithmetic: products of bf16 queries with the cache's exact values, summed in fp32 (dh additions), put a
logit off by at most dh 2^-24 of scale sum |q k|, its exponential by twice that as a share; exp2 and its argument add
2^-20.  A weight is a sum of probabilities: it is off by that share.  An output adds the rounding of each probability to
bf16 (2^-8 of sum p |v|) and its own (2^-8 of itself); what lies below the smallest normal number, 2^-126, may be lost."""
import numpy as np
import pytest
import torch

from answer_helpers import bf16, context, fill, garbage_cache, held, ints
from oracle import answering as A
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EINVAL, ENOMEM, EUNSUPPORTED = -1, -2, -4


def check(cache, q, out, weight_before, lengths, counts, scale):
    """out [B, n_q, H, dh], and the cache's weights where weight_before is given."""
    B, n_q, H, dh = q.shape
    H_kv = cache.H_kv
    for b in range(B):
        T = lengths[b]
        k, v = held(cache, b, T)
        qb = q[b].double().cpu().numpy()
        want, p = A.cache_attention(qb, k, v, counts[b], scale)
        got = out[b].double().cpu().numpy()
        kk, vv = np.repeat(k, H // H_kv, 0), np.repeat(v, H // H_kv, 0)
        size = scale * np.max(np.einsum("ihd,htd->iht", np.abs(qb), np.abs(kk)), initial=0.0)
        share = 2 * size * (dh + 4) * 2.0 ** -24 + 2.0 ** -20
        reach = np.einsum("iht,htd->ihd", p, np.abs(vv))
        lost = 2.0 ** -126 * (1 + np.abs(vv).sum(1))
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + share) * reach + lost), b
        empty = p.sum(-1) == 0
        assert not got[empty].any()
        if weight_before is not None:
            add = p.reshape(n_q, H_kv, H // H_kv, T).sum((0, 2))
            before = weight_before[b, :, :T].double().cpu().numpy()
            after = cache.weight[b, :, :T].double().cpu().numpy()
            assert np.all(np.abs(after - before - add) <= share * add + 2.0 ** -23 * (before + add)), b
            assert torch.equal(cache.weight[b, :, T:].isnan(), weight_before[b, :, T:].isnan())


def build(rng, B, H, H_kv, dh, n_q, lengths, cap=None, spread=1.0):
    T = max(max(lengths), 1)
    cap = cap or (T + 31) // 32 * 32
    ctx = context(B, H, H_kv, n_q, cap, dh)
    cache = garbage_cache(B, H_kv, dh, cap)
    fill(ctx, cache, bf16(rng, B, T, H_kv, dh, scale=spread), bf16(rng, B, T, H_kv, dh), lengths)
    for b in range(B):
        cache.weight[b, :, :lengths[b]] = torch.rand(H_kv, lengths[b], device="cuda")
    return ctx, cache, bf16(rng, B, n_q, H, dh, scale=1.3).cuda()


CASES = [  # B, H, H_kv, dh, n_q, lengths, counts
    (1, 1, 1, 64, 1, (1,), None), (1, 1, 1, 128, 1, (1,), None), (2, 4, 4, 128, 1, (0, 3), None),
    (1, 2, 2, 128, 1, (31,), None), (1, 2, 2, 64, 1, (32,), None), (3, 2, 1, 128, 1, (33, 127, 129), None),
    (2, 8, 1, 64, 1, (257, 5), None), (2, 16, 1, 128, 1, (300, 64), None), (1, 3, 3, 64, 5, (5,), None),
    (2, 3, 3, 128, 5, (3, 100), None),                      # more new rows than rows: the first see nothing
    (2, 2, 2, 128, 16, (64, 65), (16, 7)), (2, 6, 2, 64, 3, (90, 61), (2, 0)),
    (1, 17, 1, 128, 1, (77,), None), (1, 2, 2, 128, 17, (17,), None), (2, 2, 2, 64, 33, (33, 95), (33, 20)),
    (2, 4, 2, 128, 40, (70, 200), (40, 0)), (1, 1, 1, 128, 130, (130,), None), (1, 2, 1, 64, 130, (300,), None),
    (3, 3, 1, 128, 50, (0, 20, 321), (10, 50, 43)), (1, 24, 1, 64, 9, (190,), None),
    (1, 1, 1, 128, 1, (5000,), None), (1, 1, 1, 64, 70, (4100,), None), (1, 1, 1, 128, 300, (2050,), None),
]


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("B,H,H_kv,dh,n_q,lengths,counts", CASES)
def test_attention(B, H, H_kv, dh, n_q, lengths, counts, accumulate):
    rng = np.random.default_rng(H * n_q + dh)
    ctx, cache, q = build(rng, B, H, H_kv, dh, n_q, lengths)
    before = cache.weight.clone()
    out = torch.full((B, n_q, H, dh), 9.0, dtype=torch.bfloat16, device="cuda")
    print("case", B, H, H_kv, dh, n_q, lengths, counts, accumulate, flush=True)
    ctx.cache_attention(cache, q, ints(*lengths), None if counts is None else ints(*counts), accumulate=accumulate, out=out)
    check(cache, q, out, before if accumulate else None, lengths, counts or (n_q,) * B, dh ** -0.5)
    if not accumulate:
        assert torch.equal(cache.weight.nan_to_num(-1.0), before.nan_to_num(-1.0))
    # the same bits again, whatever the sums were formed by
    cache.weight.copy_(before)
    again = ctx.cache_attention(cache, q, ints(*lengths), None if counts is None else ints(*counts), accumulate=accumulate)
    first = cache.weight.clone()
    assert torch.equal(again, out)
    cache.weight.copy_(before)
    ctx.cache_attention(cache, q, ints(*lengths), None if counts is None else ints(*counts), accumulate=accumulate)
    assert torch.equal(cache.weight.nan_to_num(-1.0), first.nan_to_num(-1.0))
    ctx.close()


@pytest.mark.parametrize("n_q,H,H_kv", [(1, 2, 2), (1, 4, 1), (20, 2, 1), (140, 1, 1)])
def test_large_logits_of_both_signs(n_q, H, H_kv):
    """Weights that differ by hundreds of powers of two, maxima that move late."""
    rng = np.random.default_rng(n_q)
    ctx, cache, q = build(rng, 2, H, H_kv, 128, n_q, (400, 211), spread=6.0)
    before = cache.weight.clone()
    out = ctx.cache_attention(cache, 4 * q, ints(400, 211), accumulate=True, scale=0.3)
    check(cache, 4 * q, out, before, (400, 211), (n_q, n_q), float(np.float32(0.3)))
    ctx.close()


@pytest.mark.parametrize("n_q,H,H_kv,dh", [(1, 2, 1, 128), (6, 2, 1, 64), (40, 2, 2, 128)])
def test_strided_queries_and_outputs(n_q, H, H_kv, dh):
    """Queries as a layer's projection leaves them (beside keys and values), outputs heads first."""
    rng = np.random.default_rng(3)
    ctx, cache, q = build(rng, 2, H, H_kv, dh, n_q, (150, 97))
    wide = torch.full((2, n_q, 3 * H + 1, dh), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :, 1:H + 1] = q
    out = torch.full((2, H, n_q + 1, dh), 9.0, dtype=torch.bfloat16, device="cuda")
    ctx.cache_attention(cache, wide[:, :, 1:H + 1], ints(150, 97), out=out[:, :, 1:].transpose(1, 2))
    check(cache, q, out[:, :, 1:].transpose(1, 2), None, (150, 97), (n_q, n_q), dh ** -0.5)
    assert (out[:, :, 0] == 9).all()
    ctx.close()


@pytest.mark.parametrize("n_q", [4, 40])
def test_a_value_row_that_is_no_number_reaches_only_those_who_see_it(n_q):
    rng = np.random.default_rng(2)
    H, T, dh = 2, 70, 128
    k, v = bf16(rng, 1, T, H, dh), bf16(rng, 1, T, H, dh)
    bad = T - n_q + 2                          # seen by queries 2 and on
    v[0, bad, 1, 40] = float("inf")            # block 1 of head 1
    ctx, cache = context(1, H, H, n_q, 96, dh), garbage_cache(1, H, dh, 96)
    fill(ctx, cache, k, v, (T,))
    cache.weight[:, :, :T] = 0.5
    q = bf16(rng, 1, n_q, H, dh).cuda()
    out = ctx.cache_attention(cache, q, ints(T), accumulate=True)[0]
    none = out.isnan()
    want = torch.zeros_like(none)
    want[2:, 1, 32:64] = True
    assert torch.equal(none, want)
    kk, vv = held(cache, 0, T)
    ref, p = A.cache_attention(q[0].double().cpu().numpy(), kk, np.nan_to_num(vv), n_q, dh ** -0.5)
    reach = np.einsum("iht,htd->ihd", p, np.abs(np.nan_to_num(vv)))
    fine = ~none.cpu().numpy()
    assert np.all((np.abs(out.double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -7.9 * reach)[fine])
    assert not cache.weight[0, :, :T].isnan().any()
    ctx.close()


@pytest.mark.parametrize("n_q", [4, 40])
def test_a_key_row_that_is_no_number_spoils_only_the_rows_that_see_it(n_q):
    rng = np.random.default_rng(4)
    H, T, dh = 2, 70, 64
    k, v = bf16(rng, 1, T, H, dh), bf16(rng, 1, T, H, dh)
    k[0, T - n_q + 3, 0, 1] = float("nan")
    ctx, cache = context(1, H, H, n_q, 96, dh), garbage_cache(1, H, dh, 96)
    fill(ctx, cache, k, v, (T,))
    q = bf16(rng, 1, n_q, H, dh).cuda()
    none = ctx.cache_attention(cache, q, ints(T))[0].isnan()
    want = torch.zeros_like(none)
    want[3:, 0] = True
    assert torch.equal(none, want)
    ctx.close()


def test_lengths_beyond_the_bound_are_cut_to_it():
    rng = np.random.default_rng(6)
    ctx, cache, q = build(rng, 2, 2, 2, 64, 1, (96, 96))
    a = ctx.cache_attention(cache, q, ints(1 << 30, -5), max_length=70)
    b = ctx.cache_attention(cache, q, ints(70, 0), max_length=96)
    assert torch.equal(a[1], torch.zeros_like(a[1])) and torch.equal(b[1], torch.zeros_like(b[1]))
    check(cache, q, a, None, (70, 0), (1, 1), 64 ** -0.5)
    check(cache, q, b, None, (70, 0), (1, 1), 64 ** -0.5)
    ctx.close()


def test_far_offsets():
    """A cache whose last rows lie beyond 2^32 bytes: all rows are alike but four, which have the larger logits."""
    cap, dh = (1 << 26) + 64, 128
    z = lambda *s, dt=torch.uint8: torch.zeros(1, 1, cap, *s, dtype=dt, device="cuda")  # noqa: E731
    cache = mv.Cache4(z(64), z(64), z(4), z(4), z(dt=torch.int32), z(dt=torch.float32))
    ctx = context(1, 1, 1, 1, cap, dh)
    T = cap - 7
    rng = np.random.default_rng(9)
    k, v = torch.ones(1, 4, 1, dh).bfloat16(), bf16(rng, 1, 4, 1, dh)
    ctx.cache_append(cache, k.cuda(), v.cuda(), torch.zeros(1, 4, dtype=torch.int32, device="cuda"), ints(T))
    q = torch.full((1, 1, 1, dh), 2.0, dtype=torch.bfloat16, device="cuda")
    out = ctx.cache_attention(cache, q, ints(T), accumulate=True)[0, 0, 0].double().cpu().numpy()
    x = 2.0 * dh * dh ** -0.5                  # their logit; all others 0
    p = np.exp(x) / (4 * np.exp(x) + (T - 4))
    vv = A.fp4_decode(*A.fp4_encode(v[0, :, 0].double().numpy()))
    assert np.all(np.abs(out - p * vv.sum(0)) <= 2.0 ** -7 * p * np.abs(vv).sum(0))
    w = cache.weight[0, 0].double()
    assert abs(float(w[T - 1]) / p - 1) < 1e-4 and float(w[T:].abs().max()) == 0
    assert abs(float(w.sum()) - 1) < 1e-4
    ctx.close()


def test_a_step_in_a_graph():
    """Append, attend, weigh and choose recorded once and replayed: every replay as the eager run, with eager work and
    waits in between."""
    rng = np.random.default_rng(7)
    B, H, dh, T = 2, 4, 64, 90
    ctx, cache, _ = build(rng, B, H, H, dh, 1, (T, T - 20), cap=160)
    names = ("k", "v", "k_scale", "v_scale", "pos", "weight")
    start = {n: getattr(cache, n).clone() for n in names}
    q, k, v = (bf16(rng, B, 1, H, dh).cuda() for _ in range(3))
    ln, pos, u = ints(T, T - 20), torch.full((B, 1), 500, dtype=torch.int32, device="cuda"), torch.rand(B, device="cuda")
    head = torch.randn(H * dh, 300, device="cuda")

    def step():
        ln.add_(1)
        ctx.cache_append(cache, k, v, pos, ln)
        out = ctx.cache_attention(cache, q, ln, accumulate=True)
        kept, n = ctx.cache_evict(cache, cache, ln, 88)
        ln.copy_(n)
        return out, ctx.sample(out.view(B, -1).float() @ head, u)

    def reset():
        for n in names:
            getattr(cache, n).copy_(start[n])
        ln.copy_(ints(T, T - 20))

    want = []
    for _ in range(3):
        out, (token, prob) = step()
        want.append((out.clone(), token.clone(), prob.clone(), cache.weight.clone(), ln.clone()))
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.set_stream(side)
        step()                                 # (what a first call sets up is not recorded)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.set_stream(torch.cuda.current_stream())
        out, (token, prob) = step()
    ctx.set_stream(torch.cuda.current_stream())
    reset()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w[0]) and torch.equal(token, w[1]) and torch.equal(prob, w[2])
        assert torch.equal(cache.weight.nan_to_num(-1.0), w[3].nan_to_num(-1.0)) and torch.equal(ln, w[4])
        torch.randn(4096, device="cuda").sort()
    ctx.close()


def test_refusals():
    lib, ctx = mv.load(), mv.Context.for_cache(1, 2, 2, 1, 32, 64)
    cache = garbage_cache(1, 2, 64, 32)
    q = torch.ones(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 3.0)
    ln = ints(4)

    def call(c=cache._c, q_=mv._rows(q), H=4, n_q=1, length=ln.data_ptr(), most=32, scale=0.1, o=mv._rows(out),
             h=ctx.handle):
        ref = lambda s: mv.C.byref(s) if s is not None else None  # noqa: E731
        return lib.mvla_cache_attention(h, ref(c), ref(q_), H, n_q, None, length, most, scale, 1, ref(o))

    def rows(t, **kw):
        r = mv._rows(t)
        for a, b in kw.items():
            setattr(r, a, b)
        return r

    for bad in (dict(c=None), dict(q_=None), dict(o=None), dict(q_=mv.Rows(None, 8, 8, 8, 1)), dict(H=0), dict(H=3),
                dict(n_q=0), dict(length=None), dict(most=0), dict(most=33), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(q_=rows(q, channel=2)), dict(q_=rows(q, token=9)),
                dict(q_=rows(q, data=q.data_ptr() + 2)), dict(o=rows(out, head=68)), dict(h=None)):
        assert call(**bad) == EINVAL, bad
    assert call(n_q=1 << 23) == EUNSUPPORTED
    assert call(n_q=4096) == ENOMEM            # (more queries than the workspace was asked for)
    assert lib.mvla_cache_workspace_bytes(1, 3, 2, 64, 1, 32) == 0
    assert lib.mvla_cache_workspace_bytes(1, 2, 2, 80, 1, 32) == 0
    torch.cuda.synchronize()
    assert (out == 3).all()
    ctx.close()

"""Log probabilities, entropies and most likely tokens against fp64.

Bars.  A thread adds its share of a row's logits one behind the other (at most 130, fewer of a short row), then they go
over lanes, waves and slices in at most 30 additions more; an exponential is off by 2^-22 and by three roundings of its
argument, whose mean size is at most the entropy's: S, without the tokens that reach the maximum and are counted, is off
by a share of (chain + 30) 2^-24 + 2^-22 + 3 2^-24 (H + 1).  y takes that (times the share of S that is not counted) and
the rounding of its own terms.  An entropy takes it three times.  Tokens are equal, whatever their logits."""
import numpy as np
import pytest
import torch

from oracle import many_prompts as M
from pages_helpers import f64, ints
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EINVAL, EUNSUPPORTED = -1, -4


@pytest.fixture(scope="module")
def ctx():
    return mv.Context.for_pages(1, 1, 1, 1, 1, 1, 64)


def check(ctx, x, tokens, T=None, top=0, rows=None):
    """x [B, V] on the GPU, tokens [B, m] (numpy)."""
    B, V = x.shape
    temp = None if T is None else torch.tensor(T, dtype=torch.float32, device="cuda")
    tok = torch.from_numpy(np.ascontiguousarray(tokens.astype(np.int32))).cuda()
    lp, ent, tt, tl = ctx.logprobs(x, tok, temp, top=top)
    again = ctx.logprobs(x, tok, temp, top=top)
    for a, b in zip((lp, ent, tt, tl), again):
        assert a is None or torch.equal(a, b)
    xs = f64(x)
    for b in range(B) if rows is None else rows:
        t = 1.0 if T is None else float(np.float32(T[b]))
        y, H, order = M.logprobs(xs[b], t)
        rest = 0.0 if not t > 0 or order.size == 0 else 1.0 - np.exp(y[order])[xs[b][order] == xs[b][order[0]]].sum()
        tol = (min(130, -(-V // 256) + 2) + 30) * 2.0 ** -24 + 2.0 ** -22 + 3 * 2.0 ** -24 * (H + 1)
        with np.errstate(invalid="ignore"):
            off = tol * rest + 2.0 ** -22 * np.abs(np.where(np.isfinite(y), y, 0.0))
        def near(got, i):
            want = y[i] if abs(y[i]) < 2.0 ** 128 - 2.0 ** 103 else np.copysign(np.inf, y[i])     # (fp32 holds no more)
            assert (got == want) if not np.isfinite(want) else abs(got - want) <= off[i] + 2.0 ** -126, (b, i, got, want, off[i])
        for j, i in enumerate(tokens[b]):
            if 0 <= i < V:
                near(float(lp[b, j]), int(i))
            else:
                assert float(lp[b, j]) == -np.inf
        assert abs(float(ent[b]) - H) <= 3 * tol * (H + rest) + 2.0 ** -22 * H + 2.0 ** -126, (b, float(ent[b]), H)
        if top:
            n = min(top, order.size)
            assert tt[b].tolist() == order[:n].tolist() + [-1] * (top - n), b
            for r in range(n):
                near(float(tl[b, r]), int(order[r]))
            assert torch.all(tl[b, n:] == -float("inf"))


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("B,V,m,top", [(1, 1, 1, 1), (2, 2, 2, 5), (3, 7, 1, 32), (5, 257, 3, 20), (2, 1000, 1, 0), (9, 4099, 2, 32),
                                       (300, 513, 1, 5), (2, 32768, 1, 5), (3, 50021, 4, 32), (1, 262145, 1, 20), (1, 2100007, 2, 32)])
def test_rows(ctx, half, B, V, m, top):
    rng = np.random.default_rng(V)
    x = torch.from_numpy(rng.standard_normal((B, V + 3)) * 3).to(torch.bfloat16 if half else torch.float32).cuda()
    tokens = rng.integers(0, V, (B, m))
    tokens[0, 0] = V - 1
    if B > 1:
        tokens[1, 0] = -1
    rows = sorted(set([0, 1, 2, B - 1])) if B > 9 else None
    rows = [r for r in rows if r < B] if rows else None
    check(ctx, x[:, :V], tokens, None, top, rows)
    check(ctx, x[:, 3:], tokens, list(0.5 + rng.random(B)), top, rows)          # rows at odd addresses


@pytest.mark.parametrize("half", [True, False])
def test_rows_that_are_special(ctx, half):
    """Masked tokens, all of them, NaN, infinities, ties, zeros of both signs, one token far above all others, temperatures."""
    inf, nan = float("inf"), float("nan")
    V = 5000
    rng = np.random.default_rng(1)
    base = rng.standard_normal(V) * 2
    rows = [base.copy() for _ in range(14)]
    rows[1][rng.random(V) < 0.999] = -inf                       # a handful of tokens left
    rows[2][:] = -inf
    rows[3][:] = nan
    rows[4][::3] = nan
    rows[5][[7, 4000]] = inf
    rows[6][:] = 1.25                                            # all equal: more ties than the list holds
    rows[7][:] = np.where(np.arange(V) % 2, 0.0, -0.0)
    rows[8][1234] = 30.0                                         # nearly all of the mass
    rows[9] = np.sort(base)[::-1].copy()
    rows[10] = np.sort(base)
    rows[11][:] = -inf
    rows[11][4999] = -3.0
    rows[12] *= 1e37
    rows[13][:2500] = 3.0                                        # (half of the row ties at the top)
    x = torch.from_numpy(np.stack(rows)).to(torch.bfloat16 if half else torch.float32).cuda()
    tokens = np.stack([rng.integers(0, V, 14), np.full(14, 1234), np.full(14, 4999), np.full(14, 7), np.full(14, V), np.full(14, -5)], 1)
    check(ctx, x, tokens, None, 32)
    check(ctx, x, tokens, [0.7] * 14, 5)
    for T in (0.0, -1.0, nan):
        check(ctx, x, tokens, [T] * 14, 3)
        check(ctx, x, tokens, [T] * 14, 0)
    lp, ent, _, _ = ctx.logprobs(x, torch.from_numpy(tokens.astype(np.int32)).cuda(), torch.full((14,), inf, device="cuda"))
    assert abs(float(ent[0]) - np.log(V)) < 1e-5 and abs(float(lp[0, 0]) + np.log(V)) < 1e-5     # all alike
    lp, ent, _, _ = ctx.logprobs(x, torch.from_numpy(tokens.astype(np.int32)).cuda(), torch.full((14,), 1e-40, device="cuda"))
    assert float(lp[8, 1]) == 0.0 and float(lp[0, 1]) in (0.0, -inf) and float(ent[8]) == 0.0
    assert abs(float(lp[13, 3]) + np.log(2500)) < 1e-5 or x[13].max() > 3


def test_logits_of_any_size(ctx):
    """fp32 logits whose products with 1 / (T log 2) leave the range, at T far from 1."""
    x = torch.tensor([[-3e38, -2.9e38, -3.3e38, -3e38], [3e38, 2.9e38, 3.3e38, -3e38], [1e30, 1e30, 9e29, 0.0], [1e-40, 0.0, -1e-40, 2e-40]],
                     device="cuda")
    tokens = np.tile(np.arange(4), (4, 1))
    for T in (1.0, 1e-3, 1e37):
        check(ctx, x, tokens, [T] * 4, 4)
    y = (torch.randn(2, 3000, device="cuda", generator=torch.Generator("cuda").manual_seed(3)) * 2 + torch.tensor([[3e7], [-4e9]], device="cuda"))
    check(ctx, y, np.arange(8).reshape(2, 4), [1.0, 300.0], 5)     # (far from zero: steps of 2 and of 256)
    lp, ent, _, _ = ctx.logprobs(x[3:], ints([[0, 1, 2, 3]]))
    assert torch.all((lp + np.log(4)).abs() < 1e-6)


def test_many_rows_and_outputs(ctx):
    """More rows than one pass of the scratch holds; tokens of one dimension, none, outputs handed in."""
    rng = np.random.default_rng(2)
    B, V = 70000, 300
    x = torch.from_numpy(rng.standard_normal((B, V))).to(torch.float32).cuda()
    tok = torch.from_numpy(rng.integers(0, V, B).astype(np.int32)).cuda()
    lp, ent, tt, tl = ctx.logprobs(x, tok, top=2)
    want = torch.log_softmax(x.double(), 1)
    assert (lp.double() - want.gather(1, tok[:, None].long())[:, 0]).abs().max() < 1e-5 and lp.shape == (B,)
    assert torch.equal(tt[:, 0].long(), x.argmax(1)) and (ent.double() + (want.exp() * want).sum(1)).abs().max() < 1e-5
    none, ent2, _, _ = ctx.logprobs(x, None)
    assert none is None and torch.equal(ent2, ent)
    out = (torch.empty_like(lp), None, torch.empty_like(tt), torch.empty_like(tl))
    ctx.logprobs(x, tok, top=2, out=out)
    assert torch.equal(out[0], lp) and torch.equal(out[2], tt) and torch.equal(out[3], tl)
    flat = torch.zeros(3, device="cuda").expand(5, 3)            # one row five times
    lp, ent, _, _ = ctx.logprobs(flat, ints([[0]] * 5))
    assert torch.all((lp + np.log(3)).abs() < 1e-6)


def test_long_rows_of_many(ctx):
    """Slices whose scratch is more than the context's: rows in turns."""
    B, V = 2500, 66000
    x = torch.randn(B, V, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(torch.bfloat16)
    tok = torch.randint(0, V, (B, 1), device="cuda", dtype=torch.int32)
    lp, ent, tt, _ = ctx.logprobs(x, tok, top=32)
    want = torch.log_softmax(x[-300:].double(), 1)
    assert (lp[-300:].double() - want.gather(1, tok[-300:].long())).abs().max() < 2e-5
    order = torch.sort(x[-300:].float(), dim=1, descending=True, stable=True).indices[:, :32]
    assert torch.equal(tt[-300:].long(), order)


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("vectors", [256, 1024, 2048, 4096])
def test_rows_at_the_ends_of_a_workgroup(ctx, half, vectors):
    """One logit more or less than a thread's vectors hold, at every address; few rows and many."""
    rng = np.random.default_rng(vectors)
    whole = vectors * (8 if half else 4)
    for B, V, shift in ((2, whole - 1, 0), (2, whole, 1), (3, whole + 1, 3), (2, whole + 9, 0), (300, whole + 1, 1)):
        x = torch.from_numpy(rng.standard_normal((B, V + 3)) * 3).to(torch.bfloat16 if half else torch.float32).cuda()
        tokens = rng.integers(0, V, (B, 2))
        tokens[:, 1] = V - 1
        check(ctx, x[:, shift:shift + V], tokens, None, 20, [0, B - 1])


def test_slices_joined_in_replays(ctx):
    """Slices joined by the last one to end: replays over other logits, calls of other sizes in between, the same bits."""
    g = torch.Generator("cuda").manual_seed(3)
    cases = [(1, 262145, torch.bfloat16), (40, 50021, torch.float32), (3, 40000, torch.float32)]
    logits = [torch.randn(B, V, device="cuda", generator=g).to(t) for B, V, t in cases]
    tokens = [torch.randint(0, V, (B, 1), device="cuda", dtype=torch.int32) for B, V, _ in cases]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        own = mv.Context.for_pages(1, 1, 1, 1, 1, 1, 64)
        own.logprobs(logits[0], tokens[0], top=32)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = [own.logprobs(x, t, top=32) for x, t in zip(logits, tokens)]
        for turn in range(4):
            for x in logits:
                x.copy_(torch.randn(x.shape, device="cuda", generator=g) * (turn + 1))
            graph.replay()
            stream.synchronize()
            for x, t, outs in zip(logits, tokens, got):
                want = own.logprobs(x, t, top=32)
                stream.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(outs, want))
                order = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :32]
                assert torch.equal(outs[2].long(), order)
    torch.cuda.current_stream().wait_stream(stream)


def test_refusals(ctx):
    x, tok = torch.zeros(2, 10, device="cuda"), ints([1, 2])
    for kw, code in ((dict(top=33), EUNSUPPORTED), (dict(top=-1), EINVAL)):
        with pytest.raises((mv.MvlaError, RuntimeError)) as e:
            ctx.logprobs(x, tok, out=(torch.empty(2, device="cuda"), None, torch.empty(2, max(kw["top"], 0), dtype=torch.int32, device="cuda"),
                                      torch.empty(2, max(kw["top"], 0), device="cuda")) if kw["top"] > 0 else None, **kw)
        if kw["top"] > 0:
            assert e.value.code == code
    lib = mv.load()
    args = lambda **k: [k.get("x", x.data_ptr()), 0, 10, k.get("B", 2), k.get("V", 10), None, k.get("tok", tok.data_ptr()), k.get("m", 1),
                        k.get("lp", x.data_ptr()), None, 0, None, None]
    for k, code in ((dict(x=None), EINVAL), (dict(x=x.data_ptr() + 2), EINVAL), (dict(B=0), EINVAL), (dict(V=0), EINVAL), (dict(m=-1), EINVAL),
                    (dict(tok=None), EINVAL), (dict(lp=None), EINVAL), (dict(V=2 ** 22 + 1), EUNSUPPORTED)):
        assert lib.mvla_logprobs(ctx.handle, *args(**k)) == code, k
    for bad in (x.half(), x.cpu(), x.t()):
        with pytest.raises(AssertionError):
            ctx.logprobs(bad, tok)
    with pytest.raises(AssertionError):
        ctx.logprobs(x, tok.long())

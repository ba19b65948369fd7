"""Token choice against its definition in fp64.

Uniform numbers are put into the middle of the chosen token's share of the row's mass, shares of at least 1e-4 of it: a
running sum in another arithmetic (2^-40 of the largest weight a term, 2^-22 relative a weight) cannot cross into the next
token's.  A probability is a quotient of such sums: 1e-5."""
import numpy as np
import pytest
import torch

from answer_helpers import context
from oracle import answering as A
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EINVAL, EUNSUPPORTED = -1, -4


def logits_of(rng, B, V, kind):
    x = 2.0 * rng.standard_normal((B, V))
    x[:, rng.integers(0, V, max(1, V // 50))] += 5.0
    if kind == "masked":
        x[rng.random((B, V)) < 0.9] = -np.inf
        x[:, V // 2] = 0.5
    if kind == "ties":
        x = np.round(x)
    if kind == "signs":
        x = x - 40.0
        x[:, ::3] = 0.0
        x[:, 1::3] = -0.0
    return x


def settle(rows, u, *settings):
    """u moved to the middle of the share that it falls on; tokens of small shares are passed over."""
    out = []
    for b, x in enumerate(rows):
        tokens, p = A.sample_set(x, *(float(s[b]) if i != 1 else int(s[b]) for i, s in enumerate(settings)))
        c = np.cumsum(p)
        at = int(np.sum(c <= u[b]))
        good = np.flatnonzero(p > 1e-4)
        at = int(good[np.argmin(np.abs(good - at))]) if len(good) else int(np.argmax(p))
        out.append(np.float32(c[at] - 0.5 * p[at]))
    return np.array(out, np.float32)


def run_and_check(ctx, t, rows, u, temperature, top_k, top_p, min_p):
    dev = lambda a, dt=torch.float32: torch.tensor(np.asarray(a), dtype=dt, device="cuda")  # noqa: E731
    token, prob = ctx.sample(t, dev(u), dev(temperature), dev(top_k, torch.int32), dev(top_p), dev(min_p))
    for b, x in enumerate(rows):
        want, p = A.sample(x, float(u[b]), float(temperature[b]), int(top_k[b]), float(top_p[b]), float(min_p[b]))
        assert int(token[b]) == want, (b, int(token[b]), want)
        assert abs(float(prob[b]) - p) <= 1e-5 * p, (b, float(prob[b]), p)


@pytest.mark.parametrize("kind", ["plain", "masked", "ties", "signs"])
@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 1024, 4099, 32771])
@pytest.mark.parametrize("half", [True, False])
def test_settings_by_row(V, kind, half):
    rng = np.random.default_rng(V)
    B = 24
    t = torch.from_numpy(logits_of(rng, B, V, kind)).to(torch.bfloat16 if half else torch.float32)
    rows = t.double().numpy()
    f32 = np.float32
    temperature = rng.choice([0.0, 0.3, 0.8, 1.0, 2.5], B).astype(f32)
    top_k = rng.choice([0, 1, 2, 7, 50, V, V + 5, -1], B)
    top_p = rng.choice([0.0, 0.1, 0.55, 0.9, 0.997, 1.0, 1.5], B).astype(f32)
    min_p = rng.choice([0.0, 0.013, 0.11, 0.7, 1.0, 3.0, -1.0], B).astype(f32)
    u = settle(rows, rng.random(B), temperature, top_k, top_p, min_p)
    ctx = context(1, 1)
    run_and_check(ctx, t.cuda(), rows, u, temperature, top_k, top_p, min_p)
    ctx.close()


@pytest.mark.parametrize("half,pad,offset", [(True, 1, 1), (True, 7, 3), (False, 1, 1), (False, 3, 2), (True, 8, 8)])
def test_rows_that_start_anywhere(half, pad, offset):
    rng = np.random.default_rng(pad)
    B, V = 9, 5003
    dt = torch.bfloat16 if half else torch.float32
    wide = torch.full((B, V + pad + offset), 99.0, dtype=dt, device="cuda")    # (what lies beside a row is larger)
    wide[:, offset:offset + V] = torch.from_numpy(logits_of(rng, B, V, "plain")).to(dt).cuda()
    t = wide[:, offset:offset + V]
    rows = t.double().cpu().numpy()
    ones, none = np.ones(B), np.zeros(B)
    u = settle(rows, rng.random(B), ones, none, 0.9 * ones, none)
    ctx = context(1, 1)
    run_and_check(ctx, t, rows, u, ones, none.astype(int), np.float32(0.9) * ones, none)
    ctx.close()


def test_long_rows():
    rng = np.random.default_rng(11)
    B, V = 3, 262147
    t = torch.from_numpy(logits_of(rng, B, V, "plain")).to(torch.float32)
    rows = t.double().numpy()
    temperature, top_k = np.array([0.7, 1.0, 0.5], np.float32), np.array([0, 5000, 0])
    top_p, min_p = np.array([0.95, 1.0, 0.5], np.float32), np.array([0.0, 0.0, 0.002], np.float32)
    u = settle(rows, rng.random(B), temperature, top_k, top_p, min_p)
    ctx = context(1, 1)
    run_and_check(ctx, t.cuda(), rows, u, temperature, top_k, top_p, min_p)
    ctx.close()


def test_defaults_and_ends():
    x = torch.tensor([[0.0, 2.0, 1.0, 2.0]], device="cuda").repeat(6, 1)
    ctx = context(1, 1)
    u = torch.tensor([0.0, 0.9999999, 1.0, 7.0, -1.0, float("nan")], device="cuda")
    token, prob = ctx.sample(x, u)
    p = np.exp([0, 2, 1, 2]) / np.exp([0, 2, 1, 2]).sum()
    assert token.tolist() == [0, 3, 3, 3, 0, 0]
    assert np.allclose(prob.cpu().numpy(), p[token.cpu().numpy()], rtol=1e-6)
    # settings that are no numbers leave their filter out; a temperature that is none is greedy
    nan = torch.full((6,), float("nan"), device="cuda")
    assert ctx.sample(x, u, None, None, nan, nan)[0].tolist() == [0, 3, 3, 3, 0, 0]
    token, prob = ctx.sample(x, u, nan)
    assert token.tolist() == [1] * 6 and prob.tolist() == [1.0] * 6
    ctx.close()


def test_rows_of_infinities_and_no_numbers():
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[-inf, -inf, -inf], [nan, -inf, nan], [nan, 1.0, nan], [1.0, inf, inf], [-inf, 5.0, -inf],
                      [nan, inf, 3.0]], device="cuda")
    ctx = context(1, 1)
    u = torch.tensor([0.5, 0.5, 0.5, 0.7, 0.99, 0.3], device="cuda")
    k = torch.full((6,), 2, dtype=torch.int32, device="cuda")
    p = torch.full((6,), 0.9, device="cuda")
    for args in ((), (None, k), (None, None, p), (None, k, p, 1 - p)):
        token, prob = ctx.sample(x, u, *args)
        assert token.tolist() == [-1, -1, 1, 2, 1, 1], args
        assert prob.tolist() == [0.0, 0.0, 1.0, 0.5, 1.0, 1.0]
    ctx.close()


def test_the_same_choice_every_time():
    rng = np.random.default_rng(13)
    t = torch.from_numpy(logits_of(rng, 8, 50021, "ties")).to(torch.bfloat16).cuda()
    ctx, u = context(1, 1), torch.rand(8, device="cuda")
    p = torch.full((8,), 0.97, device="cuda")
    first = [x.clone() for x in ctx.sample(t, u, None, None, p)]
    for _ in range(5):
        again = ctx.sample(t, u, None, None, p)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    ctx.close()


def test_frequencies_follow_the_probabilities():
    """4096 draws of one row: counts within five standard deviations."""
    x = torch.tensor(np.log([0.5, 0.25, 0.125, 0.0625, 0.0625]), dtype=torch.float32, device="cuda").repeat(4096, 1)
    u = (torch.arange(4096, device="cuda") + 0.5) / 4096
    token, _ = context(1, 1).sample(x, u.float())
    counts = torch.bincount(token, minlength=5).cpu().numpy()
    assert np.all(np.abs(counts - 4096 * np.array([0.5, 0.25, 0.125, 0.0625, 0.0625])) <= 1)


def test_refusals():
    lib, ctx = mv.load(), context(1, 1)
    x, u = torch.zeros(2, 8, device="cuda"), torch.zeros(2, device="cuda")
    token = torch.full((2,), -7, dtype=torch.int32, device="cuda")

    def call(logits=x.data_ptr(), half=0, B=2, V=8, u_=u.data_ptr(), t=token.data_ptr(), h=ctx.handle):
        return lib.mvla_sample(h, logits, half, 8, B, V, None, None, None, None, u_, t, None)

    for bad in (dict(logits=None), dict(B=0), dict(V=0), dict(u_=None), dict(t=None), dict(h=None),
                dict(logits=x.data_ptr() + 2), dict(logits=x.data_ptr() + 1, half=1)):
        assert call(**bad) == EINVAL, bad
    assert call(V=(1 << 22) + 1) == EUNSUPPORTED
    torch.cuda.synchronize()
    assert token.tolist() == [-7, -7]
    assert call() == 0
    with pytest.raises(AssertionError):
        ctx.sample(x.half(), u)
    ctx.close()

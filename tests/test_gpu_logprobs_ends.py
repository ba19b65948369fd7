"""Log probabilities at the ends of their arguments' ranges (bars: test_gpu_logprobs)."""
import numpy as np
import pytest
import torch

from pages_helpers import ints
from paper_2604_09244_amd import binding as mv
from test_gpu_logprobs import check, ctx                            # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("half", [True, False])
def test_infinite_temperature(ctx, half):                           # noqa: F811
    """All logits above -infinity count alike; where some are +infinity, these alone."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((4, 3001)) * 3
    x[1, [5, 2000]] = INF
    x[2, ::2] = -INF
    x[3, :2990] = -INF
    x[3, 2995] = INF
    x = torch.from_numpy(x).to(torch.bfloat16 if half else torch.float32).cuda()
    tokens = np.tile([0, 5, 2000, 2995, 3000], (4, 1))
    check(ctx, x, tokens, [INF] * 4, 0)
    check(ctx, x, tokens, [INF] * 4, 7)


@pytest.mark.parametrize("half", [True, False])
def test_ties_at_a_temperature_without_inverse(ctx, half):          # noqa: F811
    """1 / T is beyond fp32: the tokens at the maximum share everything, one alone has it."""
    rng = np.random.default_rng(3)
    x = np.clip(rng.standard_normal((3, 5000)) * 2, -7.5, 7.5)
    x[0, 1234] = 9.0
    x[1, :2500] = 9.0
    x[2, [7, 4999]] = 9.0
    x = torch.from_numpy(x).to(torch.bfloat16 if half else torch.float32).cuda()
    tokens = np.tile([1234, 7, 4999, 3000], (3, 1))
    check(ctx, x, tokens, [1e-40] * 3, 5)
    lp, ent, _, _ = ctx.logprobs(x, torch.from_numpy(tokens.astype(np.int32)).cuda(), torch.full((3,), 1e-40, device="cuda"))
    log = lambda n: -float(np.float32(np.log(n)))
    want = [[0.0, -INF, -INF, -INF], [log(2500), log(2500), -INF, -INF], [-INF, log(2), log(2), -INF]]
    for got, row in zip(lp.tolist(), want):
        assert all(g == w or abs(g - w) <= 2.0 ** -22 * abs(w) for g, w in zip(got, row)), (got, row)
    assert float(ent[0]) == 0.0


def test_rows_in_turns(ctx):                                        # noqa: F811
    """Slices of more rows than the scratch holds (one row of logits, read by 2000 with temperatures and tokens of their own:
    256 slices with 32 best each are 69632 bytes, 1927 rows a turn where 256 compute units have 128 MiB)."""
    B, V, top = 2000, 1 << 22, 32
    rng = np.random.default_rng(4)
    logits = torch.from_numpy(rng.standard_normal(V) * 3).to(torch.float32).cuda()
    T = (0.5 + torch.from_numpy(rng.random(B))).float().cuda()
    tokens = torch.from_numpy(rng.integers(0, V, (B, 2)).astype(np.int32)).cuda()
    slices, scratch = 256, 2 * 256 * 256 * torch.cuda.get_device_properties(0).multi_processor_count * 4
    turn = (scratch - 256) // (slices * (16 + 8 * top))
    assert turn < B
    lp, ent, tt, tl = ctx.logprobs(logits.expand(B, V), tokens, T, top=top)
    order = torch.sort(logits, descending=True, stable=True).indices[:top]
    assert torch.all(tt == order.int())
    tol = 160 * 2.0 ** -24 + 2.0 ** -22
    for row in (0, 1, turn // 2, turn - 1, turn, turn + 1, B - 1):
        y = torch.log_softmax(logits.double() / T[row].double(), 0)
        H = float(-(y.exp() * y).sum())
        off = tol + 3 * 2.0 ** -24 * (H + 1)
        assert torch.all((lp[row].double() - y[tokens[row].long()]).abs() <= off + 2.0 ** -22 * y[tokens[row].long()].abs()), row
        assert torch.all((tl[row].double() - y[order]).abs() <= off + 2.0 ** -22 * y[order].abs()), row
        assert abs(float(ent[row]) - H) <= 3 * off * (H + 1) + 2.0 ** -22 * H, row


def test_no_rows(ctx):                                              # noqa: F811
    """A step with nothing to score: empty results, as of the other calls without rows."""
    x = torch.zeros(0, 100, device="cuda")
    lp, ent, tt, tl = ctx.logprobs(x, ints([]).view(0, 3), torch.zeros(0, device="cuda"), top=4)
    assert lp.shape == (0, 3) and ent.shape == (0,) and tt.shape == tl.shape == (0, 4)
    assert lp.dtype == ent.dtype == tl.dtype == torch.float32 and tt.dtype == torch.int32
    lp, ent, tt, tl = ctx.logprobs(x.bfloat16(), None)
    assert lp is None and ent.shape == (0,) and tt is None and tl is None
    with pytest.raises(AssertionError):
        ctx.logprobs(x, ints([1]))
    for logits, top in ((torch.zeros(2, 0, device="cuda"), 0), (x, 33)):      # (of no tokens; more than there are)
        with pytest.raises(mv.MvlaError):
            ctx.logprobs(logits, None, top=top)

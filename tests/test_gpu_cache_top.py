"""The top of the range: what append makes of the largest finite values, and queries that do not see such rows."""
import numpy as np
import pytest
import torch

from answer_helpers import bf16, context, fill, garbage_cache, held, ints
from oracle import answering as A
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
LARGEST = float(torch.finfo(torch.bfloat16).max)


@pytest.mark.parametrize("columns", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
def test_finite_values_stay_finite(dh, columns):
    """Every positive and negative value from 2^126 on, with and without smaller neighbours in its block."""
    bits = torch.arange(0x7e80, 0x7f80, dtype=torch.int32)
    top = torch.cat([bits, bits + 0x8000]).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros(1, len(top), 1, dh, dtype=torch.bfloat16)
    x[0, :, 0, 3] = top
    x[0, :, 0, 32:] = top[:, None]
    x[0, ::2, 0, 5] = 1.0e38
    n = len(top)
    dev = x.cuda()
    if columns:
        dev = dev.permute(0, 2, 3, 1).contiguous().permute(0, 3, 1, 2)
    ctx, cache = context(1, 1, dh=dh), garbage_cache(1, 1, dh, n)
    ctx.cache_append(cache, dev, dev, torch.arange(n, dtype=torch.int32, device="cuda")[None], ints(n))
    want_c, want_p = A.fp4_encode(x[0, :, 0].double().numpy())
    assert want_p.max() == 252
    for codes, powers in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        assert np.array_equal(powers[0, 0].cpu().numpy(), want_p)
        got = A.fp4_unpack(codes[0, 0].cpu().numpy())
        assert np.array_equal(np.where(want_c % 8 > 0, got, 0), np.where(want_c % 8 > 0, want_c, 0))
    k, v = ctx.cache_read(cache, None, n)
    assert torch.isfinite(k).all() and torch.equal(k, v)
    assert np.array_equal(k[0, 0].double().cpu().numpy(), A.fp4_decode(want_c, want_p))
    ctx.close()


@pytest.mark.parametrize("power", [None, 253, 254])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n_q,H,H_kv", [(4, 2, 2), (3, 4, 1), (40, 2, 2), (130, 1, 1)])
def test_a_large_new_row_does_not_reach_the_queries_before_it(n_q, H, H_kv, dh, power):
    """The last new row holds the largest finite values (as append writes them), or powers that append never writes:
    rows before it see nothing of that."""
    rng = np.random.default_rng(n_q)
    T = 150
    cap = 160
    k, v = bf16(rng, 1, T, H_kv, dh), bf16(rng, 1, T, H_kv, dh)
    v[0, T - 1] = LARGEST
    v[0, T - 1, :, ::2] = -LARGEST
    ctx, cache = context(1, H, H_kv, n_q, cap, dh), garbage_cache(1, H_kv, dh, cap)
    fill(ctx, cache, k, v, (T,))
    if power:
        cache.v_scale[0, :, T - 1] = power
    cache.weight[:, :, :T] = 0.5
    q = bf16(rng, 1, n_q, H, dh).cuda()
    out = ctx.cache_attention(cache, q, ints(T), accumulate=True)[0]
    kk, vv = held(cache, 0, T)
    vv = vv.copy()
    vv[:, T - 1] = 0                            # (nobody but the last query sees it)
    ref, p = A.cache_attention(q[0].double().cpu().numpy(), kk, vv, n_q, dh ** -0.5)
    reach = np.einsum("iht,htd->ihd", p, np.abs(np.repeat(vv, H // H_kv, 0)))
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - ref)[:-1] <= (2.0 ** -8 * np.abs(ref) + 2.0 ** -7.9 * reach)[:-1])
    assert torch.isfinite(cache.weight[0, :, :T]).all()
    if not power:                               # what the last query sees is a share of the largest level
        share = np.repeat(held(cache, 0, T)[1][:, T - 1], H // H_kv, 0) * p[-1, :, T - 1:T]
        assert np.all(np.abs(got[-1] - share) <= 2.0 ** -6.9 * np.abs(share))
    ctx.close()

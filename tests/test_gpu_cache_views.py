"""Caches and rows that lie anywhere: weights and positions at every 4 bytes."""
import numpy as np
import pytest
import torch

from answer_helpers import bf16, context, fill, ints
from paper_2604_09244_amd import binding as mv
from test_gpu_cache_attention import check

pytestmark = pytest.mark.gpu


def shifted_cache(B, H_kv, dh, cap, shift):
    """A cache whose weights and positions start `shift` values behind an aligned address, and the whole arrays."""
    n = B * H_kv * cap
    weight, pos = torch.full((n + 8,), 3.0, device="cuda"), torch.full((n + 8,), -7, dtype=torch.int32, device="cuda")
    u8 = lambda k: torch.zeros(B, H_kv, cap, k, dtype=torch.uint8, device="cuda")  # noqa: E731
    view = lambda t: t[shift:shift + n].view(B, H_kv, cap)  # noqa: E731
    return mv.Cache4(u8(dh // 2), u8(dh // 2), u8(dh // 32), u8(dh // 32), view(pos), view(weight)), weight, pos


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("B,H,H_kv,dh,n_q,T", [(1, 2, 2, 64, 1, 40), (1, 1, 1, 128, 1, 5003), (1, 4, 2, 64, 3, 4098),
                                               (2, 2, 2, 128, 40, 333), (1, 1, 1, 64, 130, 301)])
def test_weights_at_any_four_bytes(B, H, H_kv, dh, n_q, T, shift):
    rng = np.random.default_rng(T)
    cap = (T + 31) // 32 * 32
    cache, weight, pos = shifted_cache(B, H_kv, dh, cap, shift)
    ctx = context(B, H, H_kv, n_q, cap, dh)
    fill(ctx, cache, bf16(rng, B, T, H_kv, dh), bf16(rng, B, T, H_kv, dh), (T,) * B)
    cache.weight[:, :, :T] = torch.rand(B, H_kv, T, device="cuda")
    q, before = bf16(rng, B, n_q, H, dh).cuda(), cache.weight.clone()
    print("case", B, H, H_kv, dh, n_q, T, shift, flush=True)
    out = ctx.cache_attention(cache, q, ints(*(T,) * B), max_length=T, accumulate=True)
    check(cache, q, out, before, (T,) * B, (n_q,) * B, dh ** -0.5)
    assert torch.equal(cache.weight[:, :, T:], before[:, :, T:])
    assert (weight[:shift] == 3).all() and (weight[shift + before.numel():] == 3).all()
    kept, new = ctx.cache_evict(cache, cache, ints(*(T,) * B), max(1, T // 2))
    assert (new == max(1, T // 2)).all() and (pos[:shift] == -7).all() and (pos[shift + before.numel():] == -7).all()
    ctx.close()


def backwards(t, dims):
    """The rows description of t [B, n, H, dh] with the axes `dims` walked from their ends."""
    flipped = t.flip(dims).contiguous()
    at, stride = flipped.data_ptr(), list(flipped.stride())
    for d in dims:
        at += 2 * (t.shape[d] - 1) * stride[d]
        stride[d] = -stride[d]
    return mv.Rows(at, *stride), flipped


@pytest.mark.parametrize("dims", [(0,), (1,), (2,), (0, 1, 2)])
@pytest.mark.parametrize("n_q,H,H_kv,dh", [(1, 4, 2, 128), (9, 2, 2, 64), (40, 2, 1, 128), (130, 2, 2, 64)])
def test_rows_that_are_walked_backwards(n_q, H, H_kv, dh, dims):
    rng = np.random.default_rng(n_q)
    lib, B, T = mv.load(), 2, 200
    ctx = context(B, H, H_kv, n_q, 224, dh)
    k, v, q = bf16(rng, B, T, H_kv, dh), bf16(rng, B, T, H_kv, dh), bf16(rng, B, n_q, H, dh).cuda()
    pos = torch.arange(T, dtype=torch.int32).repeat(B, 1).cuda()
    length = ints(T, T - 30)
    caches = [mv.Cache4.empty(B, H_kv, dh, 224) for _ in range(3)]
    for c in caches:
        for t in (c.k, c.v, c.k_scale, c.v_scale, c.weight):
            t.zero_()
    ctx.cache_append(caches[0], k.cuda(), v.cuda(), pos, ints(T, T))
    for c, channels in ((caches[1], ()), (caches[2], (3,))):       # (channels backwards: the form that takes any)
        (kr, k_held), (vr, v_held) = backwards(k.cuda(), dims + channels), backwards(v.cuda(), dims)
        assert lib.mvla_cache_append(ctx.handle, c._ref, mv.C.byref(kr), mv.C.byref(vr), pos.data_ptr(), T, None,
                                     ints(T, T).data_ptr()) == 0
        torch.cuda.synchronize()
        for name in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(getattr(c, name), getattr(caches[0], name)), (name, channels)
    want = ctx.cache_attention(caches[0], q, length, max_length=T, accumulate=True)
    qr, q_held = backwards(q, dims)
    out_r, out = backwards(torch.zeros_like(want), dims)
    assert lib.mvla_cache_attention(ctx.handle, caches[1]._ref, mv.C.byref(qr), H, n_q, None, length.data_ptr(), T, dh ** -0.5, 1,
                                    mv.C.byref(out_r)) == 0
    torch.cuda.synchronize()
    assert torch.equal(out.flip(dims), want) and torch.equal(caches[1].weight, caches[0].weight)
    ctx.close()

"""Shared plumbing of the tests of the 4-bit cache (no arithmetic of the HIP path)."""
import numpy as np
import torch

from oracle import answering as A
from paper_2604_09244_amd import binding as mv


def bf16(rng, *shape, scale=1.0):
    """Normal values that bf16 holds, as a CPU tensor."""
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(torch.bfloat16)


def garbage_cache(B, H_kv, dh, capacity):
    """A cache whose every byte is 0xff: codes -6, powers that are no numbers, weights and positions that are none."""
    c = mv.Cache4.empty(B, H_kv, dh, capacity)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        t.fill_(255)
    c.pos.fill_(-77)
    c.weight.fill_(float("nan"))
    return c


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def fill(ctx, cache, k, v, lengths, pos=None):
    """Rows k, v [B, T, H_kv, dh] (CPU) as a cache's first ones; lengths [B] of them count."""
    B, T = k.shape[:2]
    pos = torch.arange(T, dtype=torch.int32).repeat(B, 1) if pos is None else pos
    ctx.cache_append(cache, k.cuda(), v.cuda(), pos.cuda(), ints(*lengths), ints(*lengths))


def held(cache, b, T):
    """What the cache's bytes stand for: k, v [H_kv, T, dh] in fp64."""
    out = []
    for codes, powers in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        c = A.fp4_unpack(codes[b, :, :T].cpu().numpy())
        out.append(A.fp4_decode(c, powers[b, :, :T].cpu().numpy().astype(np.int64)))
    return out


def context(B=8, H=32, H_kv=None, n_q=64, length=4096, dh=128):
    return mv.Context.for_cache(B, H, H_kv or H, n_q, length, dh)

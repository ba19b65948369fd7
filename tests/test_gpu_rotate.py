"""Rotation against complex multiplication in fp64.

Bar: a product's two terms are each off by their own rounding, the table's and the sum's, 2^-22 of |x1| + |x2| together,
times the gain; the result by half a step of bf16, 2^-8 of itself."""
import copy
import pickle

import numpy as np
import pytest
import torch

from oracle import many_prompts as M
from pages_helpers import bf16, f64, ints
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EINVAL, EUNSUPPORTED = -1, -4


@pytest.fixture(scope="module")
def ctx():
    return mv.Context.for_pages(1, 1, 1, 1, 1, 1, 64)


def near(got, want, x, gain=1.0):
    x = np.abs(f64(x))
    reach = (x + np.max(x, -1, keepdims=True)) * gain
    assert np.all(np.abs(f64(got) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * reach)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dh,rot", [(128, 128), (128, 64), (64, 64), (64, 48), (64, 16), (128, 112), (72, 32), (256, 256),
                                    (64, 50), (2, 2), (10, 6), (66, 64), (128, 2)])
def test_rotation(ctx, dh, rot, inter):
    rng = np.random.default_rng(dh + rot)
    for n, H, H_kv in ((1, 1, 1), (5, 3, 1), (70, 32, 8), (3, 70, 0)):
        q, k = bf16(rng, n, H, dh).cuda(), bf16(rng, n, H_kv, dh).cuda() if H_kv else None
        pos = rng.integers(0, 3000, n)
        rope = ctx.rotary_table(rot, 3000)
        f = M.frequencies(rot)
        for inverse in (False, True):
            qo, ko = ctx.rotate(q, k, ints(pos.tolist()), rope, interleaved=inter, inverse=inverse)
            near(qo, M.rotate(f64(q), pos, f, inter, inverse), q)
            if H_kv:
                near(ko, M.rotate(f64(k), pos, f, inter, inverse), k)
            assert torch.equal(qo[..., rot:], q[..., rot:])
        # in place
        q2, k2 = q.clone(), None if k is None else k.clone()
        ctx.rotate(q2, k2, ints(pos.tolist()), rope, interleaved=inter, inverse=True, out=(q2, k2))
        assert torch.equal(q2, qo) and (k is None or torch.equal(k2, ko))


@pytest.mark.parametrize("factor,gain", [(1.0, 1.0), (8.0, 1.0), (32.0, 1.35), (2.5, 0.5)])
def test_tables_of_far_positions(ctx, factor, gain):
    """Angles of positions up to 131071, scaled and not: within half a step of fp32 and of the angle's own rounding in fp64
    (position * frequency is off by 2^-53 of itself, up to 131072 radians: 2^-36)."""
    how = dict(factor=factor, low_turns=1.0, high_turns=4.0, trained=8192.0)
    c, s = ctx.rotary_table(128, 131072, base=500000.0, gain=gain, **how)
    f = M.frequencies(128, 500000.0, **how)
    at = np.array([0, 1, 2, 1000, 65535, 131071])
    ang = at[:, None] * f
    for got, want in ((c, np.cos(ang)), (s, np.sin(ang))):
        assert np.all(np.abs(f64(got[torch.from_numpy(at).cuda()]) - gain * want) <= gain * (2.0 ** -24 + 2.0 ** -35))
    rng = np.random.default_rng(0)
    q = bf16(rng, 6, 4, 128).cuda()
    qo, _ = ctx.rotate(q, None, ints(at.tolist()), (c, s), interleaved=True)
    near(qo, M.rotate(f64(q), at, f, True, gain=gain), q, gain)


def test_plain_table_is_the_layers_table(ctx):
    c, s = ctx.rotary_table(128, 500)
    rc, rs = torch.empty_like(c), torch.empty_like(s)
    mv._check(mv.load().mvla_rope_table(ctx.handle, 10000.0, 500, 128, rc.data_ptr(), rs.data_ptr()), "table")
    assert torch.equal(c, rc) and torch.equal(s, rs)


def test_strides_batches_and_positions(ctx):
    """Rows inside a projection's output, samples, transposed outputs, odd addresses; positions outside the table count as its ends."""
    rng = np.random.default_rng(3)
    B, n, H, Hk, dh = 3, 11, 4, 2, 64
    qkv = bf16(rng, B, n, H + 2 * Hk, dh).cuda()
    q, k = qkv[:, :, :H], qkv[:, :, H:H + Hk]
    pos = torch.from_numpy(rng.integers(-50, 400, (B, n)).astype(np.int32)).cuda()
    rope = ctx.rotary_table(64, 300)
    at, f = np.clip(pos.cpu().numpy(), 0, 299), M.frequencies(64)
    for inter in (False, True):
        qo, ko = ctx.rotate(q, k, pos, rope, interleaved=inter)
        near(qo, M.rotate(f64(q), at, f, inter), q)
        near(ko, M.rotate(f64(k), at, f, inter), k)
        back = torch.zeros(B, H, n, dh, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        flat = torch.zeros(B * n * Hk * dh + 1, dtype=torch.bfloat16, device="cuda")[1:].view(B, n, Hk, dh)
        ctx.rotate(q, k, pos, rope, interleaved=inter, out=(back, flat))
        assert torch.equal(back, qo) and torch.equal(flat, ko)
        wide = torch.zeros(B, n, H, dh, 2, dtype=torch.bfloat16, device="cuda")
        wide[..., 1] = q
        ctx.rotate(wide[..., 1], k, pos, rope, interleaved=inter, out=(wide[..., 1], flat))
        assert torch.equal(wide[..., 1], qo) and not wide[..., 0].any()
        whole = qkv.clone()
        ctx.rotate(whole[:, :, :H], whole[:, :, H:H + Hk], pos, rope, interleaved=inter, out=(whole[:, :, :H], whole[:, :, H:H + Hk]))
        assert torch.equal(whole[:, :, :H], qo) and torch.equal(whole[:, :, H:H + Hk], ko) and torch.equal(whole[:, :, H + Hk:], qkv[:, :, H + Hk:])


def test_rotation_is_its_transposes_inverse(ctx):
    """<R x, y> = <x, R^T y> with R^T the inverse: what a gradient of a rotation needs (bar: bf16 steps of both sides)."""
    rng = np.random.default_rng(4)
    x, y = bf16(rng, 40, 2, 64).cuda(), bf16(rng, 40, 2, 64).cuda()
    pos, rope = torch.arange(40, dtype=torch.int32, device="cuda") * 37, ctx.rotary_table(48, 2000)
    for inter in (False, True):
        a = (f64(ctx.rotate(x, None, pos, rope, interleaved=inter)[0]) * f64(y)).sum()
        b = (f64(x) * f64(ctx.rotate(y, None, pos, rope, interleaved=inter, inverse=True)[0])).sum()
        assert abs(a - b) <= 2 * 2.0 ** -8 * np.abs(f64(x)).sum() * np.abs(f64(y)).max()


def test_empty_calls_and_refusals(ctx):
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos, rope = torch.zeros(4, dtype=torch.int32, device="cuda"), ctx.rotary_table(64, 10)
    a, b = ctx.rotate(q[:0], q[:0], pos[:0], rope)
    assert a.shape == b.shape == (0, 2, 64)
    for kw, code in ((dict(rotated=0), EINVAL), (dict(rotated=3), EINVAL), (dict(rotated=258), EUNSUPPORTED), (dict(rope_len=0), EINVAL),
                     (dict(base=0.0), EINVAL), (dict(base=float("nan")), EINVAL), (dict(factor=0.5), EINVAL), (dict(gain=0.0), EINVAL),
                     (dict(factor=2.0, low_turns=4.0, high_turns=4.0), EINVAL), (dict(factor=2.0, trained=0.0), EINVAL),
                     (dict(factor=float("inf")), EINVAL)):
        args = dict(dict(rotated=64, rope_len=10), **kw)
        how = mv.Rotation(args.get("base", 1e4), args.get("factor", 1.0), args.get("low_turns", 1.0), args.get("high_turns", 4.0),
                          args.get("trained", 8192.0), args.get("gain", 1.0), args["rotated"])
        assert mv.load().mvla_rotation_table(ctx.handle, mv.C.byref(how), args["rope_len"], rope[0].data_ptr(), rope[1].data_ptr()) == code, kw
    big = ctx.rotary_table(128, 10)
    with pytest.raises(mv.MvlaError) as e:                     # more than a head has
        ctx.rotate(q, None, pos, big)
    assert e.value.code == EINVAL
    with pytest.raises(mv.MvlaError) as e:                     # the same address, other strides
        ctx.rotate(q, None, pos, rope, out=(q.view(2, 4, 64).transpose(0, 1), None))
    assert e.value.code == EINVAL
    wide = torch.zeros(4, 2, 320, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(mv.MvlaError) as e:
        ctx.rotate(wide, None, pos, rope)
    assert e.value.code == EUNSUPPORTED
    for bad in (q.float(), q.cpu()):
        with pytest.raises(AssertionError):
            ctx.rotate(bad, None, pos, rope)
    with pytest.raises(AssertionError):
        ctx.rotate(q, q[:3], pos, rope)
    with pytest.raises(AssertionError):
        ctx.rotate(q, None, pos.long(), rope)


def test_a_pair_of_tables_serves_like_a_rotary_table(ctx):
    g = torch.Generator(device="cuda").manual_seed(9)
    q = torch.randn(5, 2, 64, generator=g, device="cuda").bfloat16()
    pos, rope = torch.arange(5, dtype=torch.int32, device="cuda"), ctx.rotary_table(64, 10)
    cos, sin = rope
    assert type(rope) is mv.RotaryTable and rope.rope_len == 10 and rope.rotated == 64 and cos is rope[0] and sin is rope[1]
    want = ctx.rotate(q, None, pos, rope)[0]
    assert torch.equal(ctx.rotate(q, None, pos, (cos, sin))[0], want)
    for bad in [(cos.t().contiguous().t(), sin), (cos, sin[:9]), (cos.half(), sin), (cos, sin.cpu())]:
        with pytest.raises(AssertionError):
            ctx.rotate(q, None, pos, bad)


def test_a_copied_rotary_table_is_its_own(ctx):
    rope = ctx.rotary_table(64, 10)
    for twin in (copy.deepcopy(rope), pickle.loads(pickle.dumps(rope))):
        assert type(twin) is mv.RotaryTable and twin._cos == twin[0].data_ptr() != rope._cos and torch.equal(twin[1], rope[1])


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dh,rot", [(64, 32), (64, 30), (128, 74), (72, 2), (50, 20)])
def test_values_behind_the_rotated_ones_keep_their_bits(ctx, dh, rot, inter):
    rng = np.random.default_rng(rot)
    q = torch.from_numpy(rng.integers(-32768, 32768, (70, 5, dh)).astype(np.int16)).cuda()      # NaN of every kind among them
    pos, rope = torch.arange(70, dtype=torch.int32, device="cuda"), ctx.rotary_table(rot, 70)
    got = ctx.rotate(q.view(torch.bfloat16), None, pos, rope, interleaved=inter)[0].view(torch.int16)
    assert torch.equal(got[..., rot:], q[..., rot:])

"""Rows into pages and out of them: exact, against the format's definition in fp64."""
import numpy as np
import pytest
import torch

from oracle import many_prompts as M
from pages_helpers import Case, bf16, deal, f64, garbage_pool, ints
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EINVAL, EUNSUPPORTED = -1, -4


def all_bytes(cache):
    return [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_rows_come_back(dh, bits, page):
    rng = np.random.default_rng(dh + bits + page)
    lengths, new = [0, 1, 15, 16, 17, 130, 300], [0, 1, 15, 3, 17, 0, 77]
    H = 3
    n_pages, table = deal(rng, lengths, page, entries=21)
    cache = garbage_pool(n_pages, H, dh, page, bits)
    before = all_bytes(cache)
    at = np.concatenate([[2], 2 + np.cumsum(new)])         # (two rows before the first sequence and three behind the last are nobody's)
    n = int(at[-1]) + 3
    spread = torch.from_numpy(np.exp(4 * rng.standard_normal((n, H, 1))))
    k, v = ((bf16(rng, n, H, dh).double() * spread).to(torch.bfloat16) for _ in range(2))
    batch = mv.PageBatch(ints(at.tolist()), ints(lengths), torch.from_numpy(table).cuda())
    ctx = mv.Context.for_pages(len(lengths), H, H, n, n, 512, dh)
    ctx.pages_append(cache, batch, k.cuda(), v.cuda())
    first = [t - c for t, c in zip(lengths, new)]
    kr, vr = ctx.pages_read(cache, batch, ints(first), 80)
    for x, got in ((k, kr), (v, vr)):
        for b, c in enumerate(new):
            rows = x[at[b]:at[b + 1]].double().numpy().transpose(1, 0, 2)
            want = rows if bits == 16 else M.fp8_decode(*M.fp8_encode(rows))
            assert np.array_equal(f64(got[b, :, :c]), want), b
            # behind the table's last page: zeros
            slots = -(-lengths[b] // page) * page - first[b]
            assert not got[b, :, max(slots, 0):].view(torch.int16).any()
    # every other byte of the pool is as it was
    touched = np.zeros((n_pages, page), bool)
    for b, (t, c) in enumerate(zip(lengths, new)):
        for s in range(t - c, t):
            touched[table[b, s // page], s % page] = True
    touched = torch.from_numpy(touched).cuda()[:, None, :, None]
    for x, y in zip(before, all_bytes(cache)):
        assert torch.equal(torch.where(touched, 0, x.view(torch.uint8)), torch.where(touched, 0, y.view(torch.uint8)))


@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("dh,bits", [(128, 8), (64, 8), (128, 16)])
def test_many_rows_come_back(dh, bits, wide):
    """So many rows that a lane takes several: of sequences that begin and end anywhere, with bad pages among them."""
    rng = np.random.default_rng(dh + bits + wide)
    lengths, new = [700, 1, 0, 1203, 33, 900], [511, 1, 0, 1203, 2, 17]
    H, page = 11, 32
    n_pages, table = deal(rng, lengths, page, entries=40)
    table[3, 7], table[0, 20] = -5, n_pages                   # (no pages: not written, zeros)
    cache = garbage_pool(n_pages, H, dh, page, bits)
    before = all_bytes(cache)
    at = np.concatenate([[3], 3 + np.cumsum(new)])
    n = int(at[-1]) + 5
    k, v = (bf16(rng, n, H, dh, scale=3.0) for _ in range(2))
    kc, vc = ((x.cuda() if wide else torch.stack([x, x], -1).cuda()[..., 1]) for x in (k, v))
    batch = mv.PageBatch(ints(at.tolist()), ints(lengths), torch.from_numpy(table).cuda())
    ctx = mv.Context.for_pages(len(lengths), H, H, n, n, 40 * page, dh)
    ctx.pages_append(cache, batch, kc, vc)
    first = [t - c for t, c in zip(lengths, new)]
    kr, vr = ctx.pages_read(cache, batch, ints(first), 1204)
    touched = np.zeros((n_pages, page), bool)
    for x, got in ((k, kr), (v, vr)):
        for b, c in enumerate(new):
            rows = x[at[b]:at[b + 1]].double().numpy().transpose(1, 0, 2)
            want = rows if bits == 16 or c == 0 else M.fp8_decode(*M.fp8_encode(rows))
            want = want.copy()
            for s in range(c):
                p = table[b, (first[b] + s) // page]
                if 0 <= p < n_pages:
                    touched[p, (first[b] + s) % page] = True
                else:
                    want[:, s] = 0.0
            assert np.array_equal(f64(got[b, :, :c]), want), b
    touched = torch.from_numpy(touched).cuda()[:, None, :, None]
    for x, y in zip(before, all_bytes(cache)):
        assert torch.equal(torch.where(touched, 0, x.view(torch.uint8)), torch.where(touched, 0, y.view(torch.uint8)))


@pytest.mark.parametrize("dh", [64, 128])
def test_codes_and_powers(dh):
    """Every exponent, ties, the ends of the range, blocks with no number: codes and powers as the definition has them."""
    rng = np.random.default_rng(dh)
    n, H, page = 512, 2, 32
    x = np.exp2(rng.integers(-133, 128, (n, H, 1)).astype(float)) * rng.standard_normal((n, H, dh))
    x[:40] = np.round(x[:40] / np.abs(x[:40]).max(-1, keepdims=True) * 448) * 0.5     # (multiples of a half of steps: ties)
    x[40] = 0.0
    x[41, 0, 5], x[42, 0, 40], x[43, 1, 0] = np.inf, np.nan, -np.inf
    x[44] = float(torch.finfo(torch.bfloat16).max)
    x[45, :, ::2] = -x[44, :, ::2] if dh else 0
    x[46, 0, :3] = 463.0, 464.0, -464.0
    x = torch.from_numpy(x).to(torch.bfloat16)
    cache = garbage_pool(16, H, dh, page, 8)
    batch = mv.PageBatch(ints([0, n]), ints([n]), torch.arange(16, dtype=torch.int32, device="cuda")[None])
    ctx = mv.Context.for_pages(1, H, H, n, n, n, dh)
    ctx.pages_append(cache, batch, x.cuda(), x.flip(0).cuda())
    for src, got, power in ((x, cache.k, cache.k_scale), (x.flip(0), cache.v, cache.v_scale)):
        codes, powers = M.fp8_encode(src.double().numpy().transpose(1, 0, 2))
        assert np.array_equal(power.transpose(0, 1).flatten(1, 2).cpu().numpy(), powers)
        fine = np.repeat(powers != 255, 32, -1)
        assert np.array_equal(np.where(fine, got.transpose(0, 1).flatten(1, 2).cpu().numpy(), 0), np.where(fine, codes, 0))
    kr, _ = ctx.pages_read(cache, batch, None, n)
    assert np.array_equal(f64(kr[0]), M.fp8_decode(*M.fp8_encode(x.double().numpy().transpose(1, 0, 2))), equal_nan=True)


@pytest.mark.parametrize("bits", [16, 8])
def test_strides(bits):
    """Rows inside a larger tensor, backwards, at any two bytes, channels that do not lie side by side."""
    rng = np.random.default_rng(3)
    n, H, dh = 37, 3, 64
    src = bf16(rng, 3 * n * 2 * H * dh + 64).cuda()
    views = [src[:n * 2 * H * dh].view(n, 2 * H, dh)[:, H:], src[1:1 + n * H * dh].view(n, H, dh),
             src[:n * H * dh].view(H, n, dh).transpose(0, 1), src[:n * H * dh].view(dh, H, n).permute(2, 1, 0),
             src[:2 * n * H * dh].view(n, H, dh, 2)[..., 1], src[:H * dh].view(1, H, dh).expand(n, H, dh)]
    batch = mv.PageBatch(ints([0, 20, n]), ints([20, 17]), ints([[0, 1, -1], [3, 2, -1]]))
    ctx = mv.Context.for_pages(2, H, H, n, n, 64, dh)
    for k in views:
        for v in (views[0], k):
            cache = garbage_pool(4, H, dh, 16, bits)
            ctx.pages_append(cache, batch, k, v)
            kr, vr = ctx.pages_read(cache, batch, None, 20)
            for x, got in ((k, kr), (v, vr)):
                for b, (a, e) in enumerate(((0, 20), (20, n))):
                    rows = f64(x[a:e]).transpose(1, 0, 2)
                    want = rows if bits == 16 else M.fp8_decode(*M.fp8_encode(rows))
                    assert np.array_equal(f64(got[b, :, :e - a]), want)


def test_no_pages_and_no_rows():
    """Numbers that are no page, slots before the first and behind the table, starts and lengths out of range: nothing is
    written, and reads give zeros."""
    rng = np.random.default_rng(4)
    n, H, dh, page = 40, 2, 64, 16
    x = bf16(rng, n, H, dh).cuda()
    ctx = mv.Context.for_pages(3, H, H, n, n, 64, dh)
    for start, length, table in (([0, 20, 40, 40], [20, 20, 0], [[-1, 9], [2 ** 31 - 1, -2 ** 31], [0, 1]]),
                                 ([0, 40, 40, 40], [0, 5, 7], [[0, 1], [0, 1], [0, 1]]),      # no slots: all before the first
                                 ([50, 60, 70, 80], [32, 32, 32], [[0, 1], [0, 1], [0, 1]]),  # starts beyond the rows
                                 ([-9, -5, -1, 0], [32, 32, 32], [[0, 1], [0, 1], [0, 1]]),
                                 ([40, 30, 20, 10], [32, 32, 32], [[0, 1], [0, 1], [0, 1]])):  # descending
        cache = garbage_pool(9, H, dh, page, 8)
        before = all_bytes(cache)
        batch = mv.PageBatch(ints(start), ints(length), ints(table))
        ctx.pages_append(cache, batch, x, x)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(before, all_bytes(cache))), start
    batch = mv.PageBatch(ints([0, 0, 0, 0]), ints([0, 0, 0]), ints([[-1, 9], [4, 70], [2 ** 31 - 1, -2 ** 31]]))
    cache = garbage_pool(9, H, dh, page, 8)
    for first in ([0, 16, 0], [-20, 32, 2 ** 31 - 1], [-2 ** 31, 31, -1]):
        k, v = ctx.pages_read(cache, batch, ints(first), 16)
        for got in (k, v):
            for b, f in enumerate(first):
                for i in range(16):
                    s = f + i
                    real = b == 1 and 0 <= s < 16
                    assert bool(got[b, :, i].isnan().all()) == real and (real or not got[b, :, i].view(torch.int16).any())
    # a length behind the table's end counts as the table's
    cache = garbage_pool(9, H, dh, page, 16)
    ctx.pages_append(cache, mv.PageBatch(ints([0, n]), ints([1000]), ints([[5, 3]])), x, x)
    k, _ = ctx.pages_read(cache, mv.PageBatch(ints([0, n]), ints([0]), ints([[5, 3]])), None, 32)
    assert torch.equal(k[0].transpose(0, 1), x[n - 32:])


def test_empty_calls_and_refusals():
    ctx = mv.Context.for_pages(1, 2, 2, 8, 8, 32, 64)
    cache = garbage_pool(2, 2, 64, 16, 8)
    batch = mv.PageBatch(ints([0, 8]), ints([8]), ints([[0, 1]]))
    x = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    ctx.pages_append(cache, batch, x[:0], x[:0])
    k, v = ctx.pages_read(cache, batch, None, 0)
    assert k.shape == (1, 2, 0, 64)
    for field, value, code in (("bits", 4, EUNSUPPORTED), ("dh", 96, EUNSUPPORTED), ("page", 24, EUNSUPPORTED), ("page", 512, EUNSUPPORTED),
                               ("page", 8, EUNSUPPORTED), ("n_pages", 0, EINVAL), ("H_kv", 0, EINVAL), ("k", 0, EINVAL),
                               ("k_scale", 0, EINVAL), ("v", cache.v.data_ptr() + 8, EINVAL)):
        bad = garbage_pool(2, 2, 64, 16, 8)
        setattr(bad._c, field, value)
        with pytest.raises(mv.MvlaError) as e:
            mv._check(mv.load().mvla_pages_append(ctx.handle, bad._ref, batch._ref, mv._rows_of(x),
                                                  mv._rows_of(x), 8), "append")
        assert e.value.code == code, field
        with pytest.raises(mv.MvlaError) as e:
            mv._check(mv.load().mvla_pages_read(ctx.handle, bad._ref, batch._ref, None, 8, k.data_ptr(), v.data_ptr()), "read")
        assert e.value.code == code, field
    for field, value, code in (("B", 0, EINVAL), ("start", 0, EINVAL), ("length", 0, EINVAL), ("table", 0, EINVAL),
                               ("table_pitch", 0, EINVAL), ("table_pitch", 2 ** 27, EUNSUPPORTED), ("B", 70000, EUNSUPPORTED)):
        bad = mv.PageBatch(ints([0, 8]), ints([8]), ints([[0, 1]]))
        setattr(bad._c, field, value)
        with pytest.raises(mv.MvlaError) as e:
            ctx.pages_append(cache, bad, x, x)
        assert e.value.code == code, field
    for bad in (x.float(), x.cpu(), x[:, :1], x[..., :32]):
        with pytest.raises(AssertionError):
            ctx.pages_append(cache, batch, bad, bad)

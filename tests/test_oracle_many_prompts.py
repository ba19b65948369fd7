"""The oracle of the calls for many prompts against independent forms."""
import numpy as np
import torch

from oracle import many_prompts as M


def test_fp8_codes_are_torchs():
    """Under the power of each block the codes are those of torch's own 8-bit type; edges by hand."""
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.standard_normal((40, 64)) * np.exp(3 * rng.standard_normal((40, 1)))).to(torch.bfloat16)
    codes, powers = M.fp8_encode(x.double().numpy())
    y = x.double().numpy() / np.repeat(2.0 ** (powers - 127.0), 32, -1)
    t = torch.from_numpy(y).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)
    assert np.array_equal(codes, t.numpy())
    assert np.all(np.max(np.abs(y.reshape(40, 2, 32)), -1) < 464) and np.all(np.max(np.abs(y.reshape(40, 2, 32)), -1) >= 231)
    all_codes = np.arange(256).repeat(32).reshape(256, 32)
    v = M.fp8_decode(all_codes, np.full((256, 1), 127))[:, 0]
    w = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, w, equal_nan=True)
    big = np.zeros((3, 32))
    big[0, 0], big[1, 0], big[2, 0] = 463.9, 464.0, float(torch.finfo(torch.bfloat16).max)
    codes, powers = M.fp8_encode(big)
    assert powers[:, 0].tolist() == [127, 128, 247] and codes[:, 0].tolist() == [126, 118, 119]
    assert np.all(np.isfinite(M.fp8_decode(codes, powers).astype(np.float32)))


def test_rotation_keeps_lengths_and_turns_back():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 3, 48)), rng.integers(0, 100000, 5)
    for f in (M.frequencies(32), M.frequencies(48, factor=8.0)):
        for inter in (False, True):
            y = M.rotate(x, pos, f, inter)
            assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
            assert np.allclose(M.rotate(y, pos, f, inter, inverse=True), x)
            assert np.array_equal(y[..., 2 * f.size:], x[..., 2 * f.size:])
    f = M.frequencies(64, factor=4.0)
    g = M.frequencies(64)
    assert f[0] == g[0] and np.isclose(f[-1], g[-1] / 4) and np.all(np.diff(f) < 0)


def test_attention_is_torchs():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((4, 6, 64)), rng.standard_normal((2, 9, 64)), rng.standard_normal((2, 9, 64))
    out, lse, p = M.attention(q, k, v, 9, 0.2)
    kk, vv = (torch.from_numpy(t).repeat_interleave(3, 0) for t in (k, v))
    mask = torch.ones(4, 9).tril(5).bool()
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(0, 1), kk, vv, attn_mask=mask, scale=0.2)
    assert np.allclose(out, want.transpose(0, 1).numpy()) and np.allclose(p.sum(-1), 1)
    x = np.einsum("ihd,htd->iht", q, kk.numpy()) * 0.2
    assert np.allclose(np.exp(np.where(mask.numpy()[:, None], x, -np.inf) - lse[..., None]), p)
    out, lse, p = M.attention(q, k, v, 2, 0.2)      # more new rows than rows: the first see nothing
    assert not out[:2].any() and np.all(lse[:2] == -np.inf) and np.all(lse[2:] > -np.inf)


def test_logprobs_are_torchs():
    rng = np.random.default_rng(3)
    x = rng.standard_normal(50) * 4
    y, H, order = M.logprobs(x, 0.7)
    want = torch.log_softmax(torch.from_numpy(x) / 0.7, 0).numpy()
    assert np.allclose(y, want) and np.isclose(H, -(np.exp(want) * want).sum()) and x[order[0]] == x.max()
    x[3], x[7] = np.inf, np.inf
    y, H, _ = M.logprobs(x)
    assert np.isclose(y[3], -np.log(2)) and np.isclose(H, np.log(2)) and y[0] == -np.inf
    y, H, order = M.logprobs(np.full(4, -np.inf))
    assert np.all(y == -np.inf) and H == 0 and order.size == 0

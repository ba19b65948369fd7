"""Rotation by position, the key/value cache in pages, attention over it and log probabilities in numpy fp64, written from
their definitions (include/mvla.h); test infrastructure only."""
import numpy as np


# ---- rotation --------------------------------------------------------------------------------------------------
def frequencies(rotated, base=10000.0, factor=1.0, low_turns=1.0, high_turns=4.0, trained=8192.0):
    f = base ** (-2.0 * np.arange(rotated // 2) / rotated)
    if factor > 1:
        for i in range(f.size):
            turns = trained * f[i] / (2 * np.pi)
            stays = min(max((turns - low_turns) / (high_turns - low_turns), 0.0), 1.0)
            f[i] = stays * f[i] + (1 - stays) * f[i] / factor
    return f


def rotate(x, pos, f, interleaved, inverse=False, gain=1.0):
    """x [..., heads, dh], pos [...]: pairs turned by pos * f, as complex numbers."""
    x = np.asarray(x, np.float64)
    n = 2 * f.size
    turn = gain * np.exp((-1j if inverse else 1j) * np.asarray(pos, np.float64)[..., None] * f)[..., None, :]
    y = x.copy()
    a, b = (x[..., 0:n:2], x[..., 1:n:2]) if interleaved else (x[..., :n // 2], x[..., n // 2:n])
    z = (a + 1j * b) * turn
    if interleaved:
        y[..., 0:n:2], y[..., 1:n:2] = z.real, z.imag
    else:
        y[..., :n // 2], y[..., n // 2:n] = z.real, z.imag
    return y


# ---- rows in 8 bits ---------------------------------------------------------------------------------------------
def _levels():
    mags = [m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)]
    return np.array(mags[:127])


LEVELS = _levels()          # magnitudes of codes 0 .. 126, ascending; 127 is NaN


def fp8_encode(x):
    """Rows [..., dh] -> (codes [..., dh], powers [..., dh/32] as biased exponents)."""
    x = np.asarray(x, np.float64)
    codes = np.zeros(x.shape, np.int64)
    powers = np.zeros(x.shape[:-1] + (x.shape[-1] // 32,), np.int64)
    for at in np.ndindex(*powers.shape):
        sl = at[:-1] + (slice(32 * at[-1], 32 * at[-1] + 32),)
        if not np.all(np.isfinite(x[sl])):
            powers[at] = 255
            continue
        y = np.clip(x[sl], -247 * 2.0 ** 120, 247 * 2.0 ** 120)
        e = 0
        while np.max(np.abs(y)) >= 464.0 * 2.0 ** (e - 127):
            e += 1
        powers[at] = e
        a = np.abs(y) / 2.0 ** (e - 127)
        up = np.clip(np.searchsorted(LEVELS, a), 1, 126)          # the levels around each value
        down = up - 1
        du, dd = LEVELS[up] - a, a - LEVELS[down]
        best = np.where((du < dd) | ((du == dd) & (up % 2 == 0)), up, down)
        codes[sl] = best + 128 * np.signbit(x[sl])
    return codes, powers


def fp8_decode(codes, powers):
    codes, powers = np.asarray(codes, np.int64), np.asarray(powers, np.int64)
    v = np.where(codes % 128 == 127, np.nan, LEVELS[np.minimum(codes % 128, 126)]) * np.where(codes >= 128, -1.0, 1.0)
    p = np.where(powers == 255, np.nan, 2.0 ** (powers.astype(np.float64) - 127))
    return v * np.repeat(p, 32, axis=-1)


# ---- attention ---------------------------------------------------------------------------------------------------
def attention(q, k, v, length, scale, there=None):
    """One sequence: q [c, H, dh], k, v [H_kv, slots, dh] (rows of slots from `length` on do not matter), there: slots
    that have a page.  Returns (out, lse [c, H], p [c, H, slots])."""
    c, H, dh = q.shape
    H_kv, slots, _ = k.shape
    out, lse, prob = np.zeros(q.shape), np.full((c, H), -np.inf), np.zeros((c, H, slots))
    for i in range(c):
        sees = np.arange(slots) < min(max(length - c + i + 1, 0), length)
        if there is not None:
            sees &= there
        at = np.flatnonzero(sees)
        if at.size == 0:
            continue
        for h in range(H):
            kk, vv = k[h // (H // H_kv), at], v[h // (H // H_kv), at]
            x = kk @ q[i, h] * scale
            m = np.max(x)
            e = np.exp(x - m)
            lse[i, h] = m + np.log(e.sum())
            prob[i, h, at] = e / e.sum()
            out[i, h] = prob[i, h, at] @ vv
    return out, lse, prob


# ---- log probabilities ---------------------------------------------------------------------------------------------
def logprobs(x, T=1.0):
    """One row: (y [V], entropy, order): log probabilities, and tokens above -infinity in descending order."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    y = np.full(x.shape, -np.inf)
    if order.size == 0:
        return y, 0.0, order
    if not T > 0:
        y[order[0]] = 0.0
        return y, 0.0, order
    m = x.max()
    if m == np.inf:
        y[x == m] = -np.log((x == m).sum())
    else:
        with np.errstate(invalid="ignore"):
            d = (x - m) / T
        d = np.where(x == -np.inf, -np.inf, d)
        rest = np.exp(d[x < m]).sum()
        count = (x == m).sum()
        y = d - (np.log1p(rest) if count == 1 else np.log(count + rest))
    w = np.exp(y)
    return y, float(-(w[w > 0] * y[w > 0]).sum()), order

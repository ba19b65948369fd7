"""The 4-bit key/value cache, attention over it, eviction and token choice in numpy fp64, written from their
definitions (include/mvla.h); test infrastructure only."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def fp4_encode(x):
    """Rows [..., dh] -> (codes [..., dh] of 0 .. 15, powers [..., dh/32] as biased exponents)."""
    x = np.asarray(x, np.float64)
    codes = np.zeros(x.shape, np.int64)
    powers = np.zeros(x.shape[:-1] + (x.shape[-1] // 32,), np.int64)
    for at in np.ndindex(*powers.shape):
        sl = at[:-1] + (slice(32 * at[-1], 32 * at[-1] + 32),)
        y = x[sl]
        if not np.all(np.isfinite(y)):
            powers[at] = 255
            continue
        e = 0
        while e < 252 and np.max(np.abs(y)) >= 7.0 * 2.0 ** (e - 127):    # (a level of 252 is below 2^128)
            e += 1
        powers[at] = e
        a = np.abs(y) / 2.0 ** (e - 127)
        d = np.abs(a[:, None] - LEVELS)
        # nearest level; of two equally near ones the even code
        best = np.array([min(range(8), key=lambda c: (row[c], c % 2)) for row in d])
        codes[sl] = best + 8 * np.signbit(y)
    return codes, powers


def fp4_decode(codes, powers):
    v = np.where(codes >= 8, -1.0, 1.0) * LEVELS[codes % 8]
    p = np.where(powers == 255, np.nan, 2.0 ** (powers.astype(np.float64) - 127))
    return v * np.repeat(p, 32, axis=-1)


def fp4_unpack(packed):
    """Bytes [..., dh/2] -> codes [..., dh] (the even value in the low half)."""
    packed = np.asarray(packed).astype(np.int64)
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (2 * packed.shape[-1],))


def cache_attention(q, k, v, n_new, scale):
    """One sample: q [n_q, H, dh], k, v [H_kv, length, dh].  Returns (out [n_q, H, dh], p [n_q, H, length])."""
    n_q, H, dh = q.shape
    H_kv, length, _ = k.shape
    out, prob = np.zeros(q.shape), np.zeros((n_q, H, length))
    for i in range(min(n_new, n_q)):
        sees = min(length, length - n_new + i + 1)
        if sees <= 0:
            continue
        for h in range(H):
            kk, vv = k[h // (H // H_kv), :sees], v[h // (H // H_kv), :sees]
            x = kk @ q[i, h] * scale
            e = np.exp(x - np.max(x))
            prob[i, h, :sees] = e / e.sum()
            out[i, h] = prob[i, h, :sees] @ vv
    return out, prob


def cache_evict(weight, pos, budget, first_pos, recent_from):
    """One sample and key head, rows in use only.  Slot of the old rows that each new slot holds."""
    n = len(weight)
    if n <= budget:
        return list(range(n))
    w = [float(x) if x > 0 else 0.0 for x in weight]
    stays = [bool(p < first_pos or (recent_from is not None and p >= recent_from)) for p in pos]
    order = sorted(range(n), key=lambda t: (not stays[t], -w[t], t))
    kept = set(order[:budget])
    late = iter(t for t in range(budget, n) if t in kept)
    return [t if t in kept else next(late) for t in range(budget)]


def sample_set(logits, temperature, top_k, top_p, min_p):
    """Tokens that may be chosen, ascending, and their probabilities."""
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if top == -np.inf:
        return np.array([], np.int64), np.array([])
    if not temperature > 0:
        return order[:1], np.ones(1)
    with np.errstate(invalid="ignore"):
        w = np.where(x[order] == top, 1.0, np.exp((x[order] - top) / temperature))
    if 0 < top_k < len(order):
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        stay = before < max(top_p, 0.0) * w.sum()
        stay[0] = True
        order, w = order[stay], w[stay]
    if min_p > 0:
        stay = w >= min(min_p, 1.0)
        order, w = order[stay], w[stay]
    up = np.argsort(order)
    return order[up], w[up] / w.sum()


def sample(logits, u, temperature, top_k, top_p, min_p):
    """(token, probability) of one row."""
    tokens, p = sample_set(logits, temperature, top_k, top_p, min_p)
    if len(tokens) == 0:
        return -1, 0.0
    at = min(int(np.sum(np.cumsum(p) <= u)), len(p) - 1)
    while p[at] == 0:
        at -= 1
    return int(tokens[at]), float(p[at])

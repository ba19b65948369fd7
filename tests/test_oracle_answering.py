"""Pins of the answering oracle: against hand-worked values and independently written forms (CPU)."""
import numpy as np
import pytest
import torch

from oracle import answering as A


def test_levels_ties_and_powers_by_hand():
    row = np.zeros(32)
    row[:8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.99]       # power 1: every tie goes to the even code
    c, e = A.fp4_encode(row)
    assert e.tolist() == [127]
    assert A.LEVELS[c[:8]].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0]
    row[7] = 7.0                                                    # from 7 on the next power
    c, e = A.fp4_encode(row)
    assert e.tolist() == [128] and A.fp4_decode(c, e)[7] == 8.0
    assert A.fp4_encode(np.zeros(32))[1].tolist() == [0]
    for bad in (np.inf, -np.inf, np.nan):
        row[3] = bad
        c, e = A.fp4_encode(row)
        assert e.tolist() == [255] and np.all(np.isnan(A.fp4_decode(c, e)))


def test_every_level_is_its_own_code_at_every_power():
    signed = np.concatenate([A.LEVELS, -A.LEVELS])
    for e in (0, 1, 100, 127, 250):
        row = np.concatenate([signed, signed]) * 2.0 ** (e - 127)
        c, p = A.fp4_encode(row)
        assert np.array_equal(A.fp4_decode(c, p), row)
    packed = np.array([[0x21, 0x0f]])
    assert A.fp4_unpack(packed).tolist() == [[1, 2, 15, 0]]


@pytest.mark.parametrize("n_new", [3, 2])
def test_attention_equals_the_library_one(n_new):
    rng = np.random.default_rng(1)
    n_q, H, H_kv, T, dh = 3, 4, 2, 9, 64
    q, k, v = rng.standard_normal((n_q, H, dh)), rng.standard_normal((H_kv, T, dh)), rng.standard_normal((H_kv, T, dh))
    out, p = A.cache_attention(q, k, v, n_new, 0.2)
    see = torch.arange(T)[None] < torch.arange(T - n_new + 1, T + 1)[:, None]
    ref = torch.nn.functional.scaled_dot_product_attention(
        torch.tensor(q[:n_new]).transpose(0, 1), torch.tensor(k).repeat_interleave(2, 0),
        torch.tensor(v).repeat_interleave(2, 0), attn_mask=see, scale=0.2).transpose(0, 1).numpy()
    assert np.allclose(out[:n_new], ref, atol=1e-12) and not out[n_new:].any()
    assert np.allclose(p[:n_new].sum(-1), 1) and not p[n_new:].any()


def test_eviction_by_hand():
    w, pos = [5, 0, 3, 3, 0, 9, 3], [0, 2, 4, 6, 8, 10, 12]
    assert A.cache_evict(w, pos, 4, 0, None) == [0, 5, 2, 3]          # slots 0, 2, 3, 5 stay; 5 fills slot 1
    assert A.cache_evict(w, pos, 4, 3, None) == [0, 1, 2, 5]          # positions 0 and 2 stay whatever their weight
    assert A.cache_evict(w, pos, 4, 0, 8) == [0, 4, 5, 6]             # the last three positions stay
    assert A.cache_evict(w, pos, 7, 0, None) == list(range(7))
    assert A.cache_evict([1, float("nan"), -2, 0], [0, 1, 2, 3], 2, 0, None) == [0, 1]   # these count as 0


def test_sampling_sets_by_hand():
    x = np.log([0.4, 0.1, 0.3, 0.15, 0.05])
    keep = lambda *a: A.sample_set(x, *a)[0].tolist()  # noqa: E731
    assert keep(1.0, 0, 1.0, 0.0) == [0, 1, 2, 3, 4]
    assert keep(1.0, 2, 1.0, 0.0) == [0, 2]
    assert keep(1.0, 0, 0.69, 0.0) == [0, 2] and keep(1.0, 0, 0.71, 0.0) == [0, 2, 3]
    assert keep(1.0, 0, 0.0, 0.0) == [0]
    assert keep(1.0, 0, 1.0, 0.3) == [0, 2, 3]
    assert keep(0.0, 0, 1.0, 0.0) == [0]
    assert [A.sample(x, u, 1.0, 0, 1.0, 0.0)[0] for u in (0.0, 0.39, 0.41, 0.51, 0.81, 0.96)] == [0, 0, 1, 2, 3, 4]
    assert A.sample(np.full(4, -np.inf), 0.5, 1.0, 0, 1.0, 0.0) == (-1, 0.0)
    assert A.sample_set(np.array([0.0, np.inf, 1.0, np.inf]), 1.0, 0, 1.0, 0.0)[1].tolist() == [0.0, 0.5, 0.0, 0.5]
    ties = np.array([1.0, 2.0, 2.0, 2.0])
    assert A.sample_set(ties, 1.0, 2, 1.0, 0.0)[0].tolist() == [1, 2]

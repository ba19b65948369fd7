"""What a context of the cache's calls is sized for (host arithmetic, no GPU): every call of up to n_q queries and
max_length slots, not the largest one alone."""
import ctypes
import random

import pytest

from paper_2604_09244_amd import binding as mv


def need(*args):
    """Bytes of scratch that one call takes (B, H, H_kv, dh, n_q, max_length, accumulate)."""
    f = getattr(mv.load(), "_ZN4mvla21cache_attention_bytesEiiiiiib")
    f.argtypes, f.restype = [ctypes.c_int] * 6 + [ctypes.c_bool], ctypes.c_size_t
    return f(*args)


def reserved(B, H, H_kv, dh, n_q, max_length):
    """Bytes of scratch of a context for such calls: what is asked for less what every context holds."""
    lib = mv.load()
    fixed = lib.mvla_cache_workspace_bytes(1, 1, 1, 64, 1, 32) - 512      # (256 bytes of scratch, 256 to align it)
    return lib.mvla_cache_workspace_bytes(B, H, H_kv, dh, n_q, max_length) - fixed - 256


def smaller_calls(n_q, group):
    """Numbers of queries up to n_q: all of the few, then those around a change of path or of the rows' blocks."""
    marks = {n + d for r in (16, 32, 48, 64, 96, 128, 256, 384, 512, 1024) for n in (r // group,) for d in (0, 1)}
    return sorted({n for n in set(range(1, 18)) | marks | {n_q} if 1 <= n <= n_q})


@pytest.mark.parametrize("B,H,H_kv,dh,n_q,max_length", [
    (64, 32, 8, 128, 48, 16384), (64, 32, 8, 128, 512, 16384), (16, 32, 8, 128, 128, 2624), (1, 32, 32, 128, 49, 2624),
    (8, 32, 32, 128, 48, 1840), (1, 1, 1, 64, 1000, 40000), (2, 8, 1, 64, 100, 5000), (3, 256, 1, 128, 7, 3000)])
def test_a_context_holds_every_smaller_call(B, H, H_kv, dh, n_q, max_length):
    have = reserved(B, H, H_kv, dh, n_q, max_length)
    for n in smaller_calls(n_q, H // H_kv):
        for length in {1, 32, 1000, max_length // 2, max_length - 31, max_length}:
            for accumulate in (False, True):
                if 0 < length <= max_length:
                    assert need(B, H, H_kv, dh, n, length, accumulate) <= have, (n, length, accumulate)


def test_sizes_at_random():
    rng = random.Random(3)
    for _ in range(400):
        H_kv, group, dh = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 3, 4, 8, 17]), rng.choice([64, 128])
        B, n_q = int(2 ** rng.uniform(0, 7)), int(2 ** rng.uniform(0, 11))
        length = int(2 ** rng.uniform(0, 15))
        have = reserved(B, H_kv * group, H_kv, dh, n_q, length)
        for n in smaller_calls(n_q, group):
            for l in {length, rng.randint(1, length)}:
                assert need(B, H_kv * group, H_kv, dh, n, l, True) <= have, (B, H_kv, group, dh, n_q, length, n, l)


def test_a_context_of_layers_holds_steps_of_fewer_tokens():
    """mvla_decode_step takes its layer's buffers and the attention's behind them."""
    lib = mv.load()
    for B, n, D, H, F, length in ((64, 48, 1024, 8, 2816, 16384), (2, 130, 256, 4, 1024, 4000), (1, 49, 4096, 32, 11008, 2624)):
        have = lib.mvla_decode_workspace_bytes(B, n, D, H, F, length)
        for fewer in smaller_calls(n, 1):
            assert lib.mvla_decode_workspace_bytes(B, fewer, D, H, F, length) <= have, (B, n, fewer)


def test_sizes_that_no_call_takes():
    size, layers = mv.load().mvla_cache_workspace_bytes, mv.load().mvla_decode_workspace_bytes
    assert size(1, 1, 1, 64, 1, 1 << 30) > 0 and layers(1, 1, 64, 1, 64, 1 << 30) > 0
    for bad in ((1, 1, 1, 64, 1, (1 << 30) + 32), (1, 1, 1, 64, 1, 2 ** 31 - 1), (1, 1, 1, 64, 128 * 65535 + 1, 64),
                (1, 64, 1, 64, 2 ** 31 - 1, 64), (65536, 1, 1, 64, 1, 64), (1, 40000, 40000, 64, 1, 64)):
        assert size(*bad) == 0, bad
    for bad in ((1, 1, 64, 1, 64, 2 ** 31 - 1), (65536, 1, 64, 1, 64, 64), (1, 128 * 65535 + 1, 64, 1, 64, 64)):
        assert layers(*bad) == 0, bad

"""The first sizes beyond those that the header allows for the many-prompts calls (no GPU needed: each is refused before
anything is launched, and no pointer is followed)."""
import ctypes as C

import pytest

from paper_2604_09244_amd import binding as mv

EINVAL, EUNSUPPORTED = -1, -4
_memory = C.create_string_buffer(8192)
AT = (C.addressof(_memory) + 255) // 256 * 256        # an aligned address, for the context too
ROWS = mv._pack_rows(AT, 0, 64, 64, 1)


def pages(H_kv=2, dh=64, page=16, n_pages=4):
    return C.byref(mv.PagesC(n_pages, H_kv, dh, page, 16, AT, AT, None, None))


def batch(B=1, pitch=4):
    return C.byref(mv.PageBatchC(B, AT, AT, AT, pitch))


def append(p, b, n):
    return mv.load().mvla_pages_append(AT, p, b, ROWS, ROWS, n)


def read(p, b, n):
    return mv.load().mvla_pages_read(AT, p, b, None, n, AT, AT)


def attention(p, b, n, H=2, scale=1.0):
    return mv.load().mvla_pages_attention(AT, p, b, ROWS, H, n, 1, 64, scale, ROWS, None)


@pytest.mark.parametrize("p,b,n", [(dict(H_kv=1 << 15), {}, 1), (dict(n_pages=(1 << 30) + 1), {}, 1), ({}, dict(B=1 << 16), 1),
                                   (dict(H_kv=1025), dict(B=1 << 12), 1), ({}, dict(pitch=(1 << 26) + 1), 1),
                                   (dict(H_kv=1 << 10, dh=128), {}, 1 << 17), (dict(H_kv=1 << 14), {}, 1 << 14)])
def test_pages(p, b, n):
    assert append(pages(**p), batch(**b), n) == EUNSUPPORTED
    assert read(pages(**p), batch(**b), n) == EUNSUPPORTED
    if n == 1:
        assert attention(pages(**p), batch(**b), n, H=p.get("H_kv", 2)) == EUNSUPPORTED


def test_attention():
    assert attention(pages(), batch(), 1 << 27) == EUNSUPPORTED
    assert attention(pages(H_kv=1), batch(), 1, H=1 << 28) == EUNSUPPORTED
    for scale in (0.0, -1.0, 2.36e38, 3.4e38, float("inf"), float("nan")):
        assert attention(pages(), batch(), 1, scale=scale) == EINVAL, scale


@pytest.mark.parametrize("H,H_kv,B,n,dh", [(1 << 15, 0, 1, 1, 64), ((1 << 14) + 1, 1 << 14, 1, 1, 64), (1, 0, 1 << 15, 1 << 15, 2),
                                           (16, 16, 1 << 9, 1 << 9, 256), (32, 0, 1, 1 << 20, 64), (1, 0, 1, 1, 258)])
def test_rotate(H, H_kv, B, n, dh):
    k = ROWS if H_kv else None
    assert mv.load().mvla_rotate(AT, ROWS, H, ROWS, k, H_kv, k, AT, B, n, dh, 2, 0, 0, AT, AT, 4) == EUNSUPPORTED


def test_logprobs():
    call = lambda B, V, m, top: mv.load().mvla_logprobs(AT, AT, 0, V, B, V, None, AT, m, AT, AT, top, AT, AT)
    assert call(0, 8, 1, 0) == EINVAL and call(1, 0, 1, 0) == EINVAL
    assert call(1, (1 << 22) + 1, 1, 0) == EUNSUPPORTED and call(1, 8, 1, 33) == EUNSUPPORTED
    assert call(1 << 16, 8, 1 << 15, 0) == EUNSUPPORTED

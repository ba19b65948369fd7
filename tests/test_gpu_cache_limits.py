"""Caches of more slots than the kernels count: refused on the host, before anything is launched."""
import pytest
import torch

from answer_helpers import context, garbage_cache, ints
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu
EUNSUPPORTED = -4


def test_capacities_beyond_the_largest():
    lib, ctx, cache = mv.load(), context(1, 2, dh=64), garbage_cache(1, 2, 64, 32)
    x = torch.ones(1, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    out, ln, pos = torch.full((1, 2, 4, 64), 9.0, dtype=torch.bfloat16, device="cuda"), ints(4), ints(0, 1, 2, 3)
    kept, rows = torch.full((1, 2, 1), -5, dtype=torch.int32, device="cuda"), mv._rows(x)
    ref = mv.C.byref
    for capacity in ((1 << 30) + 32, 2 ** 31 - 32):
        c = mv.Cache4C.from_buffer_copy(cache._c)
        c.capacity = capacity
        assert lib.mvla_cache_append(ctx.handle, ref(c), ref(rows), ref(rows), pos.data_ptr(), 4, None, ln.data_ptr()) == EUNSUPPORTED
        assert lib.mvla_cache_read(ctx.handle, ref(c), None, 4, out.data_ptr(), out.data_ptr()) == EUNSUPPORTED
        assert lib.mvla_cache_attention(ctx.handle, ref(c), ref(rows), 2, 4, None, ln.data_ptr(), 4, 0.1, 0,
                                        ref(mv._rows(torch.empty_like(x)))) == EUNSUPPORTED
        assert lib.mvla_cache_evict(ctx.handle, ref(c), ref(cache._c), ln.data_ptr(), 4, 1, 0, None, ints(0).data_ptr(),
                                    kept.data_ptr()) == EUNSUPPORTED
    torch.cuda.synchronize()
    assert (cache.k == 255).all() and (out == 9).all() and (kept == -5).all()
    ctx.close()

"""The calls for many prompts from several threads at once, each with a context and a stream of its own: what they give alone."""
import threading

import numpy as np
import pytest
import torch

from pages_helpers import Case, bf16
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu


def test_threads():
    cases = []
    for i, (lengths, counts, bits) in enumerate((((700, 90), (60, 1), 16), ((3000, 40), (1, 1), 8), ((64, 130, 257), (20, 130, 1), 8))):
        rng = np.random.default_rng(i)
        c = Case(rng, 4, 2, 64, 16, bits, lengths, counts)
        logits = bf16(rng, 5, 40000, scale=3.0).cuda()
        tokens = torch.from_numpy(rng.integers(0, 40000, (5, 1)).astype(np.int32)).cuda()
        cases.append((c, logits, tokens))

    def call(ctx, c, logits, tokens):
        out, lse = ctx.pages_attention(c.cache, c.batch, c.q, max_q=max(c.counts), max_length=max(c.lengths), with_lse=True)
        rope = ctx.rotary_table(64, 4096)
        turned, _ = ctx.rotate(c.q, None, torch.arange(c.n, dtype=torch.int32, device="cuda"), rope)
        return [out, lse, turned, *ctx.pages_read(c.cache, c.batch, None, 33), *ctx.logprobs(logits, tokens, top=5)]

    want = [call(c.ctx, c, x, t) for c, x, t in cases]
    torch.cuda.synchronize()
    wrong = [None] * len(cases)
    begin = threading.Barrier(len(cases))

    def work(i):
        try:
            c, x, t = cases[i]
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                ctx = mv.Context.for_pages(len(c.lengths), c.H, c.H_kv, c.n, max(c.counts), max(c.lengths), c.dh)
                begin.wait(60)
                for turn in range(20):
                    got = call(ctx, c, x, t)
                    stream.synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                        raise AssertionError(turn)
        except BaseException as e:
            wrong[i] = e

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == [None] * len(cases), wrong

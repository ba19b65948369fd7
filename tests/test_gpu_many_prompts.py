"""The calls for many prompts together, as a serving loop makes them: rotation, rows into pages, attention, log probabilities;
eagerly, in a captured graph, on another stream; two contexts; a device that is not the current one."""
import numpy as np
import pytest
import torch

from oracle import many_prompts as M
from pages_helpers import bf16, deal, f64, garbage_pool, ints
from paper_2604_09244_amd import binding as mv

pytestmark = pytest.mark.gpu

H, H_KV, DH, PAGE, V = 4, 2, 64, 16, 900


class Loop:
    """A layer's part of a serving step over a batch whose sequences grow: queries, keys, values and head are random."""

    def __init__(self, seed, bits, lengths, room):
        rng = np.random.default_rng(seed)
        self.rng, self.bits, self.B = rng, bits, len(lengths)
        most = max(lengths) + room
        n_pages, table = deal(rng, [t + room for t in lengths], PAGE)
        self.cache = garbage_pool(n_pages, H_KV, DH, PAGE, bits)
        self.table = torch.from_numpy(table).cuda()
        self.length = ints([0] * self.B)
        self.ctx = mv.Context.for_pages(self.B, H, H_KV, sum(lengths), max(lengths), most, DH)
        self.rope = self.ctx.rotary_table(48, most)
        self.freq = M.frequencies(48)
        self.head = (torch.randn(H * DH, V, generator=torch.Generator().manual_seed(seed)) * 0.2).to(torch.bfloat16).cuda()
        self.most = most
        self.k = [np.zeros((0, H_KV, DH)) for _ in lengths]
        self.v = [np.zeros((0, H_KV, DH)) for _ in lengths]

    def inputs(self, counts):
        n = sum(counts)
        starts = np.concatenate([[0], np.cumsum(counts)]).tolist()
        qkv = bf16(self.rng, n, H + 2 * H_KV, DH).cuda()
        return ints(starts), qkv

    def step(self, start, qkv, pos, tokens, max_q):
        """What a program runs: everything on the device, nothing waits."""
        ctx = self.ctx
        batch = mv.PageBatch(start, self.length, self.table)
        q, k = ctx.rotate(qkv[:, :H], qkv[:, H:H + H_KV], pos, self.rope, interleaved=True)
        ctx.pages_append(self.cache, batch, k, qkv[:, H + H_KV:])
        out, lse = ctx.pages_attention(self.cache, batch, q, max_q=max_q, max_length=self.most, with_lse=True)
        logits = out.flatten(1) @ self.head
        return out, lse, logits, ctx.logprobs(logits, tokens, top=4)

    def check(self, counts, qkv, out, lse, logits, probs, tokens):
        """Against the oracle on the rounded rotations (bars: pages_helpers, test_gpu_logprobs)."""
        at = 0
        for b, c in enumerate(counts):
            x = f64(qkv[at:at + c])
            pos = len(self.k[b]) + np.arange(c)
            turn = lambda y: torch.from_numpy(M.rotate(y, pos, self.freq, True)).to(torch.bfloat16).double().numpy()
            rows = lambda y: y if self.bits == 16 else M.fp8_decode(*M.fp8_encode(y))
            q = turn(x[:, :H])
            self.k[b] = np.concatenate([self.k[b], rows(turn(x[:, H:H + H_KV]))])
            self.v[b] = np.concatenate([self.v[b], rows(x[:, H + H_KV:])])
            k, v = self.k[b].transpose(1, 0, 2), self.v[b].transpose(1, 0, 2)
            want, want_lse, p = M.attention(q, k, v, k.shape[1], DH ** -0.5)
            reach = np.einsum("iht,htd->ihd", p, np.abs(np.repeat(v, H // H_KV, 0)))
            # (a rotated value may round to the other neighbour than fp64's: two steps of queries and keys, 2^-7 of a logit's terms)
            kk = np.repeat(k, H // H_KV, 0)
            size = DH ** -0.5 * np.max(np.einsum("ihd,htd->iht", np.abs(q), np.abs(kk)), initial=0.0)
            flips = 2.0 ** -7 if self.bits == 16 else 2.0 ** -4
            assert np.all(np.abs(f64(out[at:at + c]) - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + flips * size) * reach)
            assert np.all(np.abs(f64(lse[at:at + c]) - want_lse) <= flips * size)
            at += c
        x = f64(logits)
        lp, ent, tt, tl = probs
        for r in range(x.shape[0]):
            y, ent_want, order = M.logprobs(x[r])
            assert abs(float(lp[r]) - y[int(tokens[r])]) < 1e-5 and abs(float(ent[r]) - ent_want) < 1e-5
            assert tt[r].tolist() == order[:4].tolist() and np.allclose(f64(tl[r]), y[order[:4]], atol=1e-5)


def run(loop, counts, max_q):
    start, qkv = loop.inputs(counts)
    n = sum(counts)
    pos = torch.cat([torch.arange(len(loop.k[b]), len(loop.k[b]) + c, dtype=torch.int32) for b, c in enumerate(counts)]).cuda()
    tokens = torch.randint(0, V, (n,), dtype=torch.int32, device="cuda")
    loop.length += ints(counts)
    res = loop.step(start, qkv, pos, tokens, max_q)
    torch.cuda.synchronize()
    loop.check(counts, qkv, *res, tokens)


@pytest.mark.parametrize("bits", [16, 8])
def test_prompts_then_answers(bits):
    """Prompts of different lengths at once, then next tokens, a late prompt's second chunk beside them, a sequence that rests."""
    loop = Loop(bits, bits, [50, 9, 130], 40)
    run(loop, [50, 9, 70], 70)
    run(loop, [1, 1, 60], 60)
    for counts in ([1, 1, 1], [1, 0, 1], [0, 3, 1], [1, 1, 1]):
        run(loop, counts, 3)


@pytest.mark.parametrize("bits", [16, 8])
def test_a_step_in_a_graph(bits):
    """One next token of every sequence, captured and replayed with other rows, lengths and pages; eager calls in between on
    the same context; each replay is the eager result bit for bit."""
    loop = Loop(1, bits, [300, 45, 20], 30)
    run(loop, [300, 45, 20], 300)
    start, qkv = loop.inputs([1, 1, 1])
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    tokens = torch.zeros(3, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loop.ctx.set_stream(side)
    with torch.cuda.stream(side):
        loop.length += 1
        loop.step(start, qkv, pos, tokens, 1)                   # (what is set up once is set up here)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            res = loop.step(start, qkv, pos, tokens, 1)
        for turn in range(4):
            loop.length += 1
            qkv.copy_(bf16(loop.rng, 3, H + 2 * H_KV, DH))
            pos.copy_(loop.length - 1)
            tokens.copy_(torch.randint(0, V, (3,), dtype=torch.int32))
            graph.replay()
            side.synchronize()
            got = [t.clone() for t in (*res[:3], *res[3])]
            eager = loop.step(start, qkv, pos, tokens, 1)
            side.synchronize()
            for a, b in zip(got, (*eager[:3], *eager[3])):
                assert torch.equal(a, b), turn
    loop.ctx.set_stream(torch.cuda.current_stream())


def test_a_chunk_in_a_graph():
    """A chunk beside next tokens (parts and their join included), replayed with lengths that differ from the captured ones."""
    rng = np.random.default_rng(9)
    lengths, counts = [2000, 700, 300], [60, 1, 20]
    loop = Loop(2, 16, lengths, 10)
    run(loop, lengths, 2000)
    q = bf16(rng, sum(counts), H, DH).cuda()
    start = ints(np.concatenate([[0], np.cumsum(counts)]).tolist())
    batch = mv.PageBatch(start, loop.length, loop.table)
    call = lambda: loop.ctx.pages_attention(loop.cache, batch, q, max_q=60, max_length=2000, with_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loop.ctx.set_stream(side)
    with torch.cuda.stream(side):
        call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out, lse = call()
        for lens, cnt in ((lengths, counts), ([100, 600, 0], [60, 1, 20]), ([2000, 64, 63], [1, 60, 20]), ([1999, 1, 300], [20, 1, 60])):
            loop.length.copy_(ints(lens))
            start.copy_(ints(np.concatenate([[0], np.cumsum(cnt)]).tolist()))
            q.copy_(bf16(rng, sum(counts), H, DH))
            graph.replay()
            side.synchronize()
            a, b = out.clone(), lse.clone()
            eager, eager_lse = call()
            side.synchronize()
            assert torch.equal(a, eager) and torch.equal(b, eager_lse), lens


def test_another_stream_is_current():
    """Calls run on the context's stream and allocate there, whatever stream is current; results are there when that stream
    has been waited for."""
    loop = Loop(3, 16, [64, 100], 4)
    start, qkv = loop.inputs([64, 100])
    pos = torch.cat([torch.arange(64), torch.arange(100)]).to(torch.int32).cuda()
    tokens = torch.zeros(164, dtype=torch.int32, device="cuda")
    loop.length += ints([64, 100])
    batch = mv.PageBatch(start, loop.length, loop.table)
    q, k = loop.ctx.rotate(qkv[:, :H], qkv[:, H:H + H_KV], pos, loop.rope)
    loop.ctx.pages_append(loop.cache, batch, k, qkv[:, H + H_KV:])
    want = loop.ctx.pages_attention(loop.cache, batch, q)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        q2, k2 = loop.ctx.rotate(qkv[:, :H], qkv[:, H:H + H_KV], pos, loop.rope)
        loop.ctx.pages_append(loop.cache, batch, k2, qkv[:, H + H_KV:])
        got = loop.ctx.pages_attention(loop.cache, batch, q2)
    loop.ctx.stream.synchronize()
    assert torch.equal(got, want) and torch.equal(q2, q)
    # a context of its own on the other stream
    with torch.cuda.stream(other):
        ctx = mv.Context.for_pages(2, H, H_KV, 164, 100, 128, DH)
        assert torch.equal(ctx.pages_attention(loop.cache, batch, q), want)
        lp = ctx.logprobs(q[:, 0].contiguous(), tokens)[0]
        other.synchronize()
    assert torch.equal(lp, loop.ctx.logprobs(q[:, 0].contiguous(), tokens)[0])


def test_kernel_times_are_recorded():
    """The calls have names in the per-kernel timing."""
    loop = Loop(4, 8, [40, 40], 4)
    loop.ctx.profile_enable(None, 64)
    run(loop, [40, 40], 40)
    names = [n for n, _, _ in loop.ctx.profile_read()]
    assert names == ["rotate", "pages_append", "pages_attention", "logprobs"]
    loop.ctx.profile_enable([], 0)

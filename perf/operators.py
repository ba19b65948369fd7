"""The operators that answer from a pruned prefill, as cases that can be timed and compared: a key/value cache
held in 4 bits, the attention that reads it, the eviction of rows that little attention went to, and the choice of
the next token.

A cache holds, per sample and key head, rows of head-dim values in blocks of 32: a code of 4 bits a value (sign and
one of 0, 1/2, 1, 3/2, 2, 3, 4, 6) and one power of two a block, 2^(e - 127) with e a byte; e = 255 makes the whole
block NaN.  The power is the smallest under which the block's largest magnitude stays below 7; values round to the
nearest code, ties to the even one.  With the rows go their position ids and the attention weight that has
accumulated on them.

Kinds:
  fill    Context.cache_append, and cache_read of the rows that were appended
  attend  Context.cache_attention: softmax(q k^T * scale) v over the rows that a query sees; `weigh`: the weights,
          summed over the queries and the query heads that share a key head, are added to the rows' own
  evict   Context.cache_evict into a cache of the budget's size, and cache_read of it: the rows of highest weight
          stay, first and recent positions before all others; a kept row keeps its slot where that lies within the
          budget, the others fill the free slots in ascending order
  sample  Context.sample: temperature, top-k, top-p and min-p, and one uniform number a row

Heads and head sizes are those of this package's models (32 of 128, 8 of 128, 4 of 64), with key heads of their own
or shared by a few query heads.  Token counts are those of its workloads (237 to 2624 tokens, 16 to 64 language
tokens, 1 to 16 samples) and beyond, up to 16384.
"""
import math
import random

import torch

own = False
DEV = "cuda"
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- the cases ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one robot after its pruned call: a decoded token's key and value rows, all 32 heads of a layer
        dict(name="fill_1x1_at_237", kind="fill", B=1, heads=32, dh=128, n=1, T=237, ragged=False),
        # the benchmark's batch: every kept token of a layer goes to the cache at once, lengths that differ
        dict(name="fill_16x1344", kind="fill", B=16, heads=32, dh=128, n=1344, T=1344, ragged=True),
        # the next token of that one robot: the smallest call of the decoding loop, latency is all of it
        dict(name="attend_1x237", kind="attend", B=1, heads=32, group=1, dh=128, nq=1, T=237, ragged=False,
             empty=False, weigh=True),
        # small heads, lengths of any kind and one sample that has no token yet
        dict(name="attend_7x611_dh64", kind="attend", B=7, heads=4, group=1, dh=64, nq=1, T=611, ragged=True,
             empty=True, weigh=True),
        # a decoding step of the benchmark's batch on all its tokens
        dict(name="attend_16x2624", kind="attend", B=16, heads=32, group=1, dh=128, nq=1, T=2624, ragged=False,
             empty=False, weigh=True),
        # the longest caches, key heads shared by four query heads: memory
        dict(name="attend_64x16384_g4", kind="attend", B=64, heads=8, group=4, dh=128, nq=1, T=16384, ragged=True,
             empty=False, weigh=True),
        # the language tokens of a new instruction against the cached scene: they weigh its rows
        dict(name="attend_8x48_of_1840", kind="attend", B=8, heads=32, group=1, dh=128, nq=48, T=1840, ragged=True,
             empty=False, weigh=True),
        # a new view of 512 tokens against what is cached: products
        dict(name="attend_4x512_of_2624", kind="attend", B=4, heads=32, group=1, dh=128, nq=512, T=2624,
             ragged=False, empty=False, weigh=False),
        # a robot's cache cut to what a pruned call keeps
        dict(name="evict_1x544_to_237", kind="evict", B=1, heads=32, dh=128, T=544, budget=237, ragged=False),
        # the benchmark's batch at half its tokens, samples that end anywhere
        dict(name="evict_16x2624_to_1344", kind="evict", B=16, heads=32, dh=128, T=2624, budget=1344, ragged=True),
        # one answer's next token: one row, all of the latency
        dict(name="sample_1x32768", kind="sample", B=1, V=32768, half=False, pad=0, masked=False),
        # many answers, a large vocabulary, settings that differ by row, rows with most tokens forbidden
        dict(name="sample_96x131073", kind="sample", B=96, V=131073, half=True, pad=7, masked=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["attend"] * 5 + ["fill", "fill", "evict", "evict", "sample", "sample"])
    heads, dh = rng.choice([(32, 128), (32, 128), (8, 128), (8, 64), (4, 64)])
    B = _log_int(rng, 1, 64)
    ragged = rng.random() < 0.6
    if kind == "sample":
        V = _log_int(rng, 256, 131072)
        return dict(kind=kind, B=_log_int(rng, 1, 96), V=V, half=rng.random() < 0.6, pad=rng.choice([0, 0, 1, 8]),
                    masked=rng.random() < 0.4)
    if kind == "fill":
        n = _log_int(rng, 1, min(8192, max(1, 688000 // (B * heads) * (128 // dh))))
        return dict(kind=kind, B=B, heads=heads, dh=dh, n=n, T=n + rng.choice([0, rng.randint(1, 300)]),
                    ragged=ragged)
    if kind == "evict":
        T = _log_int(rng, 40, min(16384, 1340000 // (B * heads) * (128 // dh)))
        return dict(kind=kind, B=B, heads=heads, dh=dh, T=T, budget=max(16, int(T * rng.uniform(0.1, 0.95))),
                    ragged=ragged)
    group = rng.choice([1, 1, 2, 4, 8])
    T = _log_int(rng, 1, min(16384, 8000000 // (B * heads)))
    nq = 1
    if rng.random() < 0.45:   # more than one query: what a chunk of tokens takes, within the largest listed one
        nq = _log_int(rng, 2, max(2, min(512, T, 170000000 // (B * heads * group * T))))
    return dict(kind=kind, B=B, heads=heads, group=group, dh=dh, nq=nq, T=T, ragged=ragged,
                empty=ragged and rng.random() < 0.3, weigh=rng.random() < 0.7)


# ---- inputs -----------------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens in each sample's cache: the first has them all."""
    B, T = case["B"], case["T"]
    rng = random.Random(1000 * B + T)
    ln = [T if b == 0 or not case["ragged"] else rng.randint(max(1, T // 4), T) for b in range(B)]
    if case.get("empty") and B > 1:
        ln[B - 1] = 0
    return ln


def _new_counts(case):
    """How many of the nq (or n) new rows each sample has."""
    n = case["nq"] if case["kind"] == "attend" else case["n"]
    rng = random.Random(77 * case["B"] + n)
    return [min(t, n if b == 0 or not case["ragged"] else rng.randint(max(1, n // 2), n))
            for b, t in enumerate(_lengths(case))]


def _capacity(rows):
    return (rows + 31) // 32 * 32


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _empty_cache(B, heads, dh, capacity):
    u8 = dict(dtype=torch.uint8, device=DEV)
    return dict(k=torch.zeros(B, heads, capacity, dh // 2, **u8), v=torch.zeros(B, heads, capacity, dh // 2, **u8),
                k_scale=torch.zeros(B, heads, capacity, dh // 32, **u8),
                v_scale=torch.zeros(B, heads, capacity, dh // 32, **u8),
                pos=torch.zeros(B, heads, capacity, dtype=torch.int32, device=DEV),
                weight=torch.zeros(B, heads, capacity, dtype=torch.float32, device=DEV))


def _key_spread(heads, dh, g):
    """Keys have a few channels that are several times larger than the rest, the same for every token."""
    s = torch.exp(0.4 * torch.randn(heads, 1, dh, generator=g, device=DEV))
    return torch.where(torch.rand(heads, 1, dh, generator=g, device=DEV) < 0.03, 4.0 * s, s)


def _filled_cache(case, g):
    B, heads, dh, T = case["B"], case["heads"], case["dh"], case["T"]
    c = _empty_cache(B, heads, dh, _capacity(T))
    spread = _key_spread(heads, dh, g)
    for b in range(B):
        for name, s in (("k", spread), ("v", 1.0)):
            x = (torch.randn(heads, T, dh, generator=g, device=DEV) * s).to(torch.bfloat16)
            c[name][b, :, :T], c[name + "_scale"][b, :, :T] = _codes(x)
    # pruned tokens keep the position ids that they had: gaps
    gaps = torch.randint(1, 4, (B, 1, T), generator=g, device=DEV, dtype=torch.int32)
    c["pos"][:, :, :T] = torch.cumsum(gaps, -1).to(torch.int32) - gaps[:, :, :1]
    # heavy-tailed, with ties: many rows that no query has looked at
    w = torch.exp(2.0 * torch.randn(B, heads, T, generator=g, device=DEV) - 6.0)
    c["weight"][:, :, :T] = torch.where(torch.rand(B, heads, T, generator=g, device=DEV) < 0.2, 0.0, w)
    return c, spread


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]
    s = dict(case=case, kind=kind)
    bf = torch.bfloat16
    if kind == "sample":
        return {**s, **_sampling_inputs(case, g)}
    B, heads, dh = case["B"], case["heads"], case["dh"]
    ln = _lengths(case)
    s["length"] = _ints(ln)
    if kind == "fill":
        n = case["n"]
        s["cache"] = _empty_cache(B, heads, dh, _capacity(case["T"] + n))
        s["cache"]["weight"].fill_(0.25)   # (of rows that were here before: new ones start at none)
        # key and value rows as a layer's projection leaves them: the heads of a token side by side
        s["k_new"] = (torch.randn(B, n, heads, dh, generator=g, device=DEV)
                      * _key_spread(heads, dh, g).view(1, 1, heads, dh)).to(bf)
        s["v_new"] = torch.randn(B, n, heads, dh, generator=g, device=DEV).to(bf)
        new = _new_counts(case)
        s["n_new"] = _ints(new)
        s["first"] = _ints([t - m for t, m in zip(ln, new)])
        s["pos_new"] = (s["first"][:, None] + torch.arange(n, dtype=torch.int32, device=DEV)).contiguous()
        return s
    s["cache"], spread = _filled_cache(case, g)
    if kind == "evict":
        s["smaller"] = _empty_cache(B, heads, dh, _capacity(case["budget"]))
        # the eight first positions and what was added last stay whatever their weight
        s["recent_from"] = torch.stack([s["cache"]["pos"][b, 0, max(0, ln[b] - max(4, case["budget"] // 8))]
                                        for b in range(B)])
        return s
    H = heads * case["group"]
    q = torch.randn(B, case["nq"], H, dh, generator=g, device=DEV) * 1.5
    # (queries look away from the large channels)
    s["q"] = (q / spread.view(1, 1, heads, 1, dh).expand(-1, -1, -1, case["group"], -1).reshape(1, 1, H, dh)).to(bf)
    s["n_new"] = _ints(_new_counts(case))
    return s


def _sampling_inputs(case, g):
    B, V = case["B"], case["V"]
    x = 2.5 * torch.randn(B, V + case["pad"], generator=g, device=DEV)
    x[:, ::max(1, V // 61)] += 6.0
    if case["masked"]:   # a grammar that allows a small part of the vocabulary, in every second row
        x[1::2][torch.rand(x[1::2].shape, generator=g, device=DEV) < 0.97] = -math.inf
        x[:, 5] = 0.0
    x = x.to(torch.bfloat16 if case["half"] else torch.float32)
    r = torch.rand(4, B, generator=g, device=DEV)
    row = torch.arange(B, device=DEV)
    s = dict(logits=x[:, :V],
             temperature=torch.where(row % 7 == 6, 0.0, 0.6 + 0.8 * r[0]),
             top_k=torch.where(row % 3 == 2, 0, (4 + 200 * r[1]).int()).to(torch.int32),
             top_p=torch.where(row % 4 == 3, 1.0, 0.7 + 0.29 * r[2]),
             min_p=torch.where(row % 2 == 1, 0.0, 0.05 * r[3]))
    s["u"] = _settled(s, torch.rand(48, B, generator=g, device=DEV))
    return s


def _settled(s, tries):
    """Uniform numbers whose token is not a matter of rounding: of each row's tries the first that falls on a
    token with some share of the row's mass, moved to the middle of that share.  (At the very border of two
    tokens either is right to the last bit, and no two orders of summation agree.)"""
    x = s["logits"].double()
    xs, order = torch.sort(x, descending=True, stable=True)
    w = torch.exp((xs - xs[:, :1]) / torch.where(s["temperature"] > 0, s["temperature"], 1.0).double()[:, None])
    w = w * _prefix(w, s).double()
    c = torch.cumsum(torch.zeros_like(w).scatter_(1, order, w), 1)
    c = c / c[:, -1:]
    at = torch.searchsorted(c, tries.double().T.contiguous(), right=True).clamp_(max=x.shape[1] - 1)
    hi = c.gather(1, at)
    lo = torch.where(at > 0, c.gather(1, (at - 1).clamp_(min=0)), 0.0)
    width = hi - lo
    fine = width > 1e-4
    pick = torch.where(fine.any(1), fine.int().argmax(1), width.argmax(1))[:, None]
    return (0.5 * (lo + hi)).gather(1, pick)[:, 0].float()


# ---- plain forms ------------------------------------------------------------------------------------------------
def _codes(x):
    """Codes [..., dh/2] (two a byte, the even value low) and scale bytes [..., dh/32] of rows [..., dh]."""
    y = x.float().view(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = y.abs().amax(-1)
    m, ex = torch.frexp(top)               # top = m * 2^ex with m in [1/2, 1): below 7 * 2^(ex - 3) or 7 * 2^(ex - 2)
    e = torch.where(top > 0, ex - 3 + (m >= 0.875).int() + 127, 0).clamp(min=0)
    bad = ~torch.isfinite(top)
    y = torch.ldexp(y, (127 - e)[..., None])
    a = y.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
         + 8 * (y < 0))
    c = torch.where(bad[..., None], 0, c).to(torch.uint8).view(*x.shape[:-1], x.shape[-1] // 2, 2)
    return c[..., 0] | (c[..., 1] << 4), torch.where(bad, 255, e).to(torch.uint8)


def _values(codes, scale):
    """Rows [..., dh] in 32 bits that the codes stand for."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float32, device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).view(*codes.shape[:-1], scale.shape[-1], 32)
    e = scale.int()
    power = torch.where(e == 0, 0x00400000, torch.where(e == 255, 0x7FC00000, e << 23)).view(torch.float32)
    return (table[c.int()] * power[..., None]).view(*codes.shape[:-1], codes.shape[-1] * 2)


def _read(c, first, n):
    """The n rows of each sample from slot first[b] on, as bf16."""
    b = torch.arange(first.numel(), device=DEV)[:, None]
    at = first.long()[:, None] + torch.arange(n, device=DEV)
    rows = lambda x: x.transpose(1, 2)[b, at].transpose(1, 2)  # noqa: E731
    return tuple(_values(rows(c[x]), rows(c[x + "_scale"])).to(torch.bfloat16) for x in ("k", "v"))


def _plain_fill(s):
    c, n = s["cache"], s["case"]["n"]
    b = torch.arange(s["case"]["B"], device=DEV)[:, None]
    at = s["first"].long()[:, None] + torch.arange(n, device=DEV)
    real = torch.arange(n, device=DEV) < s["n_new"][:, None]

    def put(name, new):
        old = c[name].transpose(1, 2)
        shape = real.shape + (1,) * (old.dim() - 2)
        old[b, at] = torch.where(real.view(shape), new, old[b, at])

    k, ke = _codes(s["k_new"])
    v, ve = _codes(s["v_new"])
    put("k", k), put("k_scale", ke), put("v", v), put("v_scale", ve)
    put("pos", s["pos_new"][..., None])
    put("weight", torch.zeros((), device=DEV))
    k, v = _read(c, s["first"], n)
    return dict(k=k, v=v, pos=c["pos"], weight=c["weight"])


def _plain_attend(s):
    case, c = s["case"], s["cache"]
    B, heads, group, dh, nq, T = (case[x] for x in ("B", "heads", "group", "dh", "nq", "T"))
    k, v = (_values(c[x][:, :, :T], c[x + "_scale"][:, :, :T]) for x in ("k", "v"))
    # query rows of a key head: (query, head of the group)
    q = s["q"].float().view(B, nq, heads, group, dh).permute(0, 2, 1, 3, 4).reshape(B, heads, nq * group, dh)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(dh))
    i = torch.arange(nq * group, device=DEV) // group
    sees = (s["length"] - s["n_new"])[:, None] + i + 1
    sees = torch.where(i < s["n_new"][:, None], sees, 0).clamp_(min=0)[:, None, :, None]
    seen = torch.arange(T, device=DEV) < sees
    x = torch.where(seen, x, -math.inf)
    p = torch.where(seen, torch.exp(x - x.amax(-1, keepdim=True)), 0.0)
    p = p / torch.where(sees > 0, p.sum(-1, keepdim=True), 1.0)
    o = torch.matmul(p, v).view(B, heads, nq, group, dh).permute(0, 2, 1, 3, 4).reshape(B, nq, heads * group, dh)
    if not case["weigh"]:
        return dict(out=o.to(torch.bfloat16))
    c["weight"][:, :, :T] += p.sum(2)
    return dict(out=o.to(torch.bfloat16), weight=c["weight"])


def _plain_evict(s):
    case, c, d = s["case"], s["cache"], s["smaller"]
    T, budget = case["T"], case["budget"]
    slot = torch.arange(T, device=DEV)
    there = (slot < s["length"][:, None])[:, None]
    pos, weight = c["pos"][:, :, :T], c["weight"][:, :, :T]
    stays = (pos < 8) | (pos >= s["recent_from"][:, None, None])
    key = weight.contiguous().view(torch.int32).long() + (stays.long() << 31)
    order = torch.sort(torch.where(there, key, -1), dim=-1, descending=True, stable=True).indices
    n = torch.minimum(s["length"], torch.tensor(budget, device=DEV)).to(torch.int32)
    keep = torch.zeros_like(there.expand_as(key)).scatter(-1, order, (slot < n[:, None])[:, None].expand_as(order))
    inside = (slot < n[:, None])[:, None]
    hole, mover = inside & ~keep, ~inside & keep
    # movers by their rank (the others to a place behind), then each hole takes the mover of its rank
    rank = torch.where(mover, torch.cumsum(mover, -1) - 1, T)
    movers = torch.zeros(*key.shape[:-1], T + 1, dtype=torch.long, device=DEV)
    movers.scatter_(-1, rank, slot.expand_as(rank))
    kept = torch.where(hole, movers.gather(-1, (torch.cumsum(hole, -1) - 1).clamp_(min=0)), slot)
    kept = torch.where(inside, kept, -1)[..., :budget]
    row = kept.clamp(min=0)
    for x in ("k", "v", "k_scale", "v_scale"):
        rows = c[x].gather(2, row[..., None].expand(-1, -1, -1, c[x].shape[-1]))
        d[x][:, :, :budget] = torch.where((kept >= 0)[..., None], rows, d[x][:, :, :budget])
    for x in ("pos", "weight"):
        d[x][:, :, :budget] = torch.where(kept >= 0, c[x].gather(2, row), d[x][:, :, :budget])
    k, v = _read(d, torch.zeros_like(n), budget)
    return dict(kept=kept.to(torch.int32), length=n, pos=d["pos"], weight=d["weight"], k=k, v=v)


def _prefix(w, s):
    """Which of a row's tokens, in descending order with weights w (the largest is 1), may be chosen."""
    rank = torch.arange(w.shape[1], device=w.device)
    k = s["top_k"][:, None]
    in_k = (rank < k) | (k <= 0)
    w = torch.where(in_k, w, 0.0)
    p = s["top_p"][:, None]
    before = torch.cumsum(w, 1) - w
    in_p = (before < p * w.sum(1, keepdim=True)) | (p >= 1.0) | (rank == 0)
    return in_k & in_p & (w >= s["min_p"][:, None]) & ((s["temperature"][:, None] > 0) | (rank == 0))


def _plain_sample(s):
    x, order = torch.sort(s["logits"].float(), descending=True, stable=True)
    t = torch.where(s["temperature"] > 0, s["temperature"], 1.0)
    w = torch.exp((x - x[:, :1]) / t[:, None])
    w = torch.where(_prefix(w, s), w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)
    c = torch.cumsum(w, 1)
    total = c[:, -1:]
    token = (c <= s["u"][:, None] * total).sum(1, keepdim=True)
    return dict(token=token[:, 0].to(torch.int32), prob=(w.gather(1, token) / total)[:, 0])


# ---- one pass -----------------------------------------------------------------------------------------------------
_contexts = {}


def _context(s):
    """The context that a program keeps for calls of this size."""
    from paper_2604_09244_amd import binding as mv
    c = s["case"]
    key = tuple(c.get(x, 0) for x in ("B", "heads", "group", "nq", "T", "dh"))
    if key not in _contexts:
        _contexts[key] = mv.Context.for_cache(c["B"], c.get("heads", 1) * c.get("group", 1), c.get("heads", 1),
                                              c.get("nq", 1), c.get("T", 1), c.get("dh", 128))
    return mv, _contexts[key]


def run(state):
    s, kind = state, state["kind"]
    if not own:
        return dict(fill=_plain_fill, attend=_plain_attend, evict=_plain_evict, sample=_plain_sample)[kind](s)
    if "handle" not in s:   # what a program keeps beside its tensors
        mv, ctx = _context(s)
        s["handle"] = ctx, *(mv.Cache4(**s[x]) for x in ("cache", "smaller") if x in s)
    ctx, *caches = s["handle"]
    if kind == "sample":
        token, prob = ctx.sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return dict(token=token, prob=prob)
    case, cache = s["case"], caches[0]
    if kind == "fill":
        ctx.cache_append(cache, s["k_new"], s["v_new"], s["pos_new"], s["length"], s["n_new"])
        k, v = ctx.cache_read(cache, s["first"], case["n"])
        return dict(k=k, v=v, pos=cache.pos, weight=cache.weight)
    if kind == "attend":
        out = ctx.cache_attention(cache, s["q"], s["length"], s["n_new"], max_length=case["T"],
                                  accumulate=case["weigh"])
        return dict(out=out, weight=cache.weight) if case["weigh"] else dict(out=out)
    kept, n = ctx.cache_evict(cache, caches[1], s["length"], case["budget"], first_pos=8,
                              recent_from=s["recent_from"], max_length=case["T"])
    k, v = ctx.cache_read(caches[1], None, case["budget"])
    return dict(kept=kept, length=n, pos=caches[1].pos, weight=caches[1].weight, k=k, v=v)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "sample":
        n = case["B"] * case["V"]
        return {"bytes": (2.0 if case["half"] else 4.0) * n + 28.0 * case["B"], "flops": 4.0 * n}
    B, heads, dh = case["B"], case["heads"], case["dh"]
    row = 2.0 * (dh // 2 + dh // 32)          # a key and a value row as the cache holds them
    if kind == "fill":
        new = heads * float(sum(_new_counts(case)))
        read = float(B * heads * case["n"])
        return {"bytes": new * (4.0 * dh + row + 8) + read * (row + 4.0 * dh), "flops": 6.0 * dh * new}
    ln = _lengths(case)
    rows = heads * float(sum(ln))
    if kind == "evict":
        kept = heads * float(sum(min(t, case["budget"]) for t in ln))
        back = float(B * heads * case["budget"])
        return {"bytes": 8 * rows + kept * (2 * row + 20) + back * (row + 4.0 * dh), "flops": rows}
    group, nq = case["group"], case["nq"]
    seen = heads * group * float(sum(m * (t - m) + m * (m + 1) // 2 for t, m in zip(ln, _new_counts(case))))
    return {"bytes": rows * (row + (8 if case["weigh"] else 0)) + 4.0 * B * nq * heads * group * dh,
            "flops": 4.0 * dh * seen}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------
def _decode64(codes, scale):
    """Values of codes by the format's definition: sign, two exponent bits, one mantissa bit; subnormal 1/2."""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2).double()
    sign = torch.where(c >= 8, -1.0, 1.0).double()
    c = c % 8
    ex, man = torch.floor(c / 2), c % 2
    mag = torch.where(ex == 0, 0.5 * man, (1 + 0.5 * man) * torch.pow(2.0, ex - 1))
    e = scale.double().repeat_interleave(32, -1)
    return sign * mag * torch.where(e == 255, math.nan, torch.pow(2.0, e - 127))


def _nearest64(x):
    """Rows as the cache holds them: each block's smallest power under which all stays below 7, each value the
    nearest level (of two equally near ones that with the even code)."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.ceil(torch.log2(top / 7.0)), -127.0)
    e = torch.where(top < 7.0 * torch.pow(2.0, e), e, e + 1).clamp(min=-127.0)
    a = (y * torch.pow(2.0, -e)).abs()
    best, value = torch.full_like(a, math.inf), torch.zeros_like(a)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):
        d = (a - LEVELS[code]).abs()
        value = torch.where(d < best, LEVELS[code], value)
        best = torch.minimum(d, best)
    return (torch.sign(y) * value * torch.pow(2.0, e)).flatten(-2)


def _exact_attend(case, s):
    c, nq, group = s["cache"], case["nq"], case["group"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    weight = c["weight"].double()
    ln, new = _lengths(case), _new_counts(case)
    for b in range(case["B"]):
        for h in range(case["heads"]):
            if ln[b] == 0:
                continue
            k = _decode64(c["k"][b, h, :ln[b]], c["k_scale"][b, h, :ln[b]])
            v = _decode64(c["v"][b, h, :ln[b]], c["v_scale"][b, h, :ln[b]])
            q = s["q"][b, :new[b], h * group:(h + 1) * group].double()
            x = torch.tensordot(q, k, dims=([2], [1])) / math.sqrt(case["dh"])
            last = ln[b] - new[b] + torch.arange(new[b], device=DEV)
            x.masked_fill_(torch.arange(ln[b], device=DEV) > last[:, None, None], -math.inf)
            p = torch.softmax(x, -1)
            out[b, :new[b], h * group:(h + 1) * group] = torch.tensordot(p, v, dims=([2], [0]))
            weight[b, h, :ln[b]] += p.sum((0, 1))
    return dict(out=out, weight=weight) if case["weigh"] else dict(out=out)


def _exact_evict(case, s):
    c, budget = s["cache"], case["budget"]
    cap = s["smaller"]["k"].shape[2]
    shape = (case["B"], case["heads"])
    weight = torch.zeros(*shape, cap, dtype=torch.float64, device=DEV)
    k, v = (torch.zeros(*shape, budget, case["dh"], dtype=torch.float64, device=DEV) for _ in range(2))
    recent = s["recent_from"].tolist()
    for b, t in enumerate(_lengths(case)):
        w, pos = c["weight"][b, :, :t].double(), c["pos"][b, :, :t]
        n = min(t, budget)
        best = torch.argsort(-w, dim=-1, stable=True)                       # by weight, then those that stay first
        other = ~((pos < 8) | (pos >= recent[b])).gather(-1, best)
        best = best.gather(-1, torch.argsort(other.to(torch.uint8), dim=-1, stable=True))[:, :n]
        for h in range(case["heads"]):
            kept = set(best[h].tolist())
            late = iter(sorted(x for x in kept if x >= n))
            at = torch.tensor([x if x in kept else next(late) for x in range(n)], device=DEV, dtype=torch.long)
            weight[b, h, :n] = c["weight"][b, h, at].double()
            k[b, h, :n] = _decode64(c["k"][b, h, at], c["k_scale"][b, h, at])
            v[b, h, :n] = _decode64(c["v"][b, h, at], c["v_scale"][b, h, at])
    return dict(kept=None, length=None, pos=None, weight=weight, k=k, v=v)


def _exact_sample(s):
    prob = []
    for b in range(s["logits"].shape[0]):
        x, t = s["logits"][b].double(), float(s["temperature"][b])
        if not t > 0:
            prob.append(1.0)
            continue
        down = torch.argsort(-x, stable=True)
        p = torch.softmax(x / t, 0)[down]
        k = int(s["top_k"][b])
        p = p[:k] if 0 < k < p.numel() else p
        p = p / p.sum()
        n = p.numel()
        if float(s["top_p"][b]) < 1:
            n = max(1, int((torch.cat([p.new_zeros(1), torch.cumsum(p, 0)[:-1]]) < float(s["top_p"][b])).sum()))
        p = p[:n]
        n = int((p >= float(s["min_p"][b]) * p[0]).sum())
        index, p = down[:n], p[:n] / p[:n].sum()
        by_index = torch.argsort(index)
        at = int((torch.cumsum(p[by_index], 0) <= float(s["u"][b])).sum())
        prob.append(float(p[by_index][min(at, n - 1)]))
    return dict(token=None, prob=torch.tensor(prob, dtype=torch.float64))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(s)
    if case["kind"] == "attend":
        return _exact_attend(case, s)
    if case["kind"] == "evict":
        return _exact_evict(case, s)
    rows = torch.arange(case["n"], device=DEV)[:, None] < s["n_new"][:, None, None, None]   # [B, 1, n, 1]
    k, v = (torch.stack([_nearest64(x.transpose(0, 1)) for x in s[name]]) for name in ("k_new", "v_new"))
    weight = s["cache"]["weight"].double()
    for b, (t, m) in enumerate(zip(_lengths(case), _new_counts(case))):
        weight[b, :, t - m:t] = 0.0
    return dict(k=torch.where(rows, k, 0.0), v=torch.where(rows, v, 0.0), pos=None, weight=weight)

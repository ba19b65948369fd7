"""Operators for serving answers from many prompts at once, as cases that can be timed and compared: the rotation of
queries and keys by position, a key/value cache in pages that sequences of any length share, the attention of new
tokens over it, and the log probabilities of tokens.

Tokens of several sequences lie packed one sequence behind the other: `start` [B + 1] says where each one's begin.
A sequence's cached slots are its page table's pages in order, `page` slots each; `length` counts the new tokens.
A page holds, per key head, rows of head-dim values, as they are (16 bits) or as codes of 8 bits (sign, four exponent
bits, three mantissa bits; at most 448) in blocks of 32 with one power of two a block, 2^(e - 127) with e a byte:
the smallest under which the block's largest magnitude stays below 464; values round to the nearest code, ties to
the even one (finite ones beyond 247 * 2^120 as that, so that all codes stay finite).

Kinds:
  rotate    Context.rotate: pairs of a head's first `rot` values, side by side or half of `rot` apart, turned by
            position times frequency; frequencies as they are, or those of long waves lowered for long contexts
  store     Context.pages_append of new tokens' keys and values, and pages_read of what was written
  attend    Context.pages_attention: softmax(q k^T * scale) v over the slots that a query sees, and the logarithm
            of each row's sum of exponentials
  logprobs  Context.logprobs: of given tokens, with each row's entropy and its most likely tokens

Heads and head sizes are those of this package's models (32 of 128, 8 of 128, 4 of 64), with key heads of their own
or shared by a few query heads.  Token counts are those of its workloads (237 to 2624 tokens, 16 to 64 language
tokens, 1 to 16 samples) and beyond, up to 16384 cached and 131072 in position.
"""
import math
import random

import torch

own = False
DEV = "cuda"
LARGEST = 247 * 2.0 ** 120   # what bf16 holds beyond would round to 2^128


# ---- the cases ------------------------------------------------------------------------------------------------
def listed():
    return [
        # one robot's next token, all heads of a layer: latency
        dict(name="rotate_1_token", kind="rotate", n=1, heads=32, group=1, dh=128, rot=128, pairs="halves", far=2624,
             scaled=False),
        # a benchmark batch's tokens (16 x 2624) in one call, key heads shared by four, half of each head turned in pairs
        # side by side, positions far behind the trained ones
        dict(name="rotate_41984_tokens", kind="rotate", n=41984, heads=8, group=4, dh=128, rot=64, pairs="sides",
             far=131072, scaled=True),
        # a decoding step of 64 sequences of any length: one row each into pages of 16, in 8 bits
        dict(name="store_64x1_8bit", kind="store", B=64, heads=8, dh=128, n=1, T=2624, page=16, bits=8, ragged=True),
        # every kept token of a layer goes to the cache at once, in 8 bits
        dict(name="store_16x1344_8bit", kind="store", B=16, heads=32, dh=128, n=1344, T=1344, page=64, bits=8,
             ragged=True),
        # the next token of one robot: the smallest call of an answer's loop
        dict(name="attend_1x237", kind="attend", B=1, heads=32, group=1, dh=128, nq=1, T=237, page=16, bits=16,
             ragged=False, mixed=False),
        # a decoding step of the benchmark's batch on all its tokens, values as they are: memory
        dict(name="attend_16x2624", kind="attend", B=16, heads=32, group=1, dh=128, nq=1, T=2624, page=32, bits=16,
             ragged=False, mixed=False),
        # many long sequences in 8 bits, key heads shared by four query heads: memory
        dict(name="attend_64x16384_g4_8bit", kind="attend", B=64, heads=8, group=4, dh=128, nq=1, T=16384, page=64,
             bits=8, ragged=True, mixed=False),
        # one prompt's chunk of 512 tokens beside 31 answers' next tokens
        dict(name="attend_512_beside_31x1", kind="attend", B=32, heads=8, group=4, dh=128, nq=512, T=2624, page=16,
             bits=16, ragged=True, mixed=True),
        # a chunk of 2048 tokens of a long prompt: products
        dict(name="attend_1x2048_of_16384", kind="attend", B=1, heads=32, group=1, dh=128, nq=2048, T=16384, page=64,
             bits=16, ragged=False, mixed=False),
        # chunks of a few prompts in 8 bits, small heads, counts that end anywhere
        dict(name="attend_7x611_of_1840_dh64_8bit", kind="attend", B=7, heads=4, group=2, dh=64, nq=611, T=1840, page=32,
             bits=8, ragged=True, mixed=False),
        # one answer's next token with the five most likely ones: latency
        dict(name="logprobs_1x32768", kind="logprobs", B=1, V=32768, half=False, pad=0, given=1, top=5, masked=False),
        # a prompt's tokens judged against a large vocabulary, rows of odd length, rows with most tokens forbidden
        dict(name="logprobs_2624x131073", kind="logprobs", B=2624, V=131073, half=True, pad=7, given=1, top=20,
             masked=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["attend"] * 5 + ["rotate", "rotate", "store", "store", "logprobs", "logprobs"])
    if kind == "logprobs":
        V = _log_int(rng, 512, 131073)
        return dict(kind=kind, B=_log_int(rng, 1, min(2624, 170000000 // V)), V=V, half=rng.random() < 0.6,
                    pad=rng.choice([0, 0, 1, 8]), given=rng.choice([1, 1, 1, 2, 7]), top=rng.choice([0, 1, 5, 20, 32]),
                    masked=rng.random() < 0.4)
    heads, dh = rng.choice([(32, 128), (32, 128), (8, 128), (8, 64), (4, 64)])
    group = rng.choice([1, 1, 2, 4, 8]) if heads < 32 else 1
    if kind == "rotate":
        n = _log_int(rng, 1, min(41984, 41984 * 40 // (heads * (group + 1))))
        rot = rng.choice([dh, dh, dh // 2, dh - 16, 2 * rng.randint(1, dh // 2)])
        return dict(kind=kind, n=n, heads=heads, group=group, dh=dh, rot=rot, pairs=rng.choice(["halves", "sides"]),
                    far=max(n, _log_int(rng, 512, 131072)), scaled=rng.random() < 0.5)
    B = _log_int(rng, 1, 64)
    page, bits = rng.choice([16, 16, 32, 64, 128, 256]), rng.choice([16, 8])
    ragged = rng.random() < 0.6
    if kind == "store":
        n = _log_int(rng, 1, min(8192, max(1, 688000 // (B * heads) * (128 // dh))))
        return dict(kind=kind, B=B, heads=heads, dh=dh, n=n, T=n + rng.choice([0, rng.randint(1, 300)]), page=page,
                    bits=bits, ragged=ragged)
    T = _log_int(rng, 1, min(16384, 8000000 // (B * heads)))
    mixed = B > 1 and rng.random() < 0.3
    nq = 1
    if mixed or rng.random() < 0.5:   # more than one query: within the largest listed one
        nq = _log_int(rng, 2, max(2, min(2048, T, 1000000000 // ((1 if mixed else B) * heads * group * T))))
    return dict(kind=kind, B=B, heads=heads, group=group, dh=dh, nq=nq, T=T, page=page, bits=bits, ragged=ragged,
                mixed=mixed)


# ---- inputs -----------------------------------------------------------------------------------------------------
def _lengths(case):
    """Tokens of each sequence: the first has them all."""
    B, T = case["B"], case["T"]
    rng = random.Random(1000 * B + T)
    return [T if b == 0 or not case["ragged"] else rng.randint(max(1, T // 4), T) for b in range(B)]


def _new_counts(case):
    """How many of them are new."""
    n = case["nq"] if case["kind"] == "attend" else case["n"]
    rng = random.Random(77 * case["B"] + n)
    few = 1 if case.get("mixed") else n
    return [min(t, n if b == 0 else few if not case["ragged"] else rng.randint(max(1, few // 2), few))
            for b, t in enumerate(_lengths(case))]


def _starts(case):
    at = [0]
    for c in _new_counts(case):
        at.append(at[-1] + c)
    return at


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _page_table(case, g):
    """Pages dealt out in any order; entries behind a sequence's last page are -1.  A few pages are nobody's."""
    per = [-(-t // case["page"]) for t in _lengths(case)]
    n_pages = sum(per) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((case["B"], max(per)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(per):
        table[b, :m] = order[at:at + m]
        at += m
    return n_pages, table


def _empty_pages(case, n_pages):
    shape = (n_pages, case["heads"], case["page"])
    if case["bits"] == 16:
        return {x: torch.zeros(*shape, case["dh"], dtype=torch.bfloat16, device=DEV) for x in ("k", "v")}
    new = lambda n: torch.zeros(*shape, n, dtype=torch.uint8, device=DEV)  # noqa: E731
    return dict(k=new(case["dh"]), v=new(case["dh"]), k_scale=new(case["dh"] // 32), v_scale=new(case["dh"] // 32))


def _key_spread(heads, dh, g):
    """Keys have a few channels that are several times larger than the rest, the same for every token."""
    s = torch.exp(0.4 * torch.randn(heads, 1, dh, generator=g, device=DEV))
    return torch.where(torch.rand(heads, 1, dh, generator=g, device=DEV) < 0.03, 4.0 * s, s)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    kind = case["kind"]
    s = dict(case=case, kind=kind)
    bf = torch.bfloat16
    if kind == "logprobs":
        return {**s, **_logits(case, g)}
    heads, dh = case["heads"], case["dh"]
    if kind == "rotate":
        n, H = case["n"], heads * case["group"]
        # rows as a projection leaves them: a token's queries, keys and values side by side
        qkv = torch.randn(n, H + 2 * heads, dh, generator=g, device=DEV).to(bf)
        s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + heads]
        s["pos"] = torch.randint(0, case["far"], (n,), generator=g, device=DEV, dtype=torch.int32)
        return s
    s["start"], s["length"] = _ints(_starts(case)), _ints(_lengths(case))
    n_pages, s["table"] = _page_table(case, g)
    spread = _key_spread(heads, dh, g)
    N = _starts(case)[-1]
    if kind == "store":
        s["pages"] = _empty_pages(case, n_pages)
        kv = torch.randn(N, 2, heads, dh, generator=g, device=DEV)
        kv[:, 0] *= spread.view(1, heads, dh)
        kv = kv.to(bf)
        s["k_new"], s["v_new"] = kv[:, 0], kv[:, 1]
        s["first"] = s["length"] - (s["start"][1:] - s["start"][:-1])
        return s
    s["pages"] = _empty_pages(case, n_pages)
    step = max(1, (1 << 28) // (heads * case["page"] * dh))
    for name, w in (("k", spread), ("v", 1.0)):
        for at in range(0, n_pages, step):
            part = s["pages"][name][at:at + step]
            x = (torch.randn(part.shape[0], heads, case["page"], dh, generator=g, device=DEV) * w).to(bf)
            if case["bits"] == 16:
                part.copy_(x)
            else:
                part[:], s["pages"][name + "_scale"][at:at + step] = _codes(x)
    group = case["group"]
    q = torch.randn(N, heads, group, dh, generator=g, device=DEV) * 1.5
    # (queries look away from the large channels)
    s["q"] = (q / spread.view(1, heads, 1, dh)).view(N, heads * group, dh).to(bf)
    return s


def _logits(case, g):
    B, V = case["B"], case["V"]
    x = torch.empty(B, V + case["pad"], dtype=torch.bfloat16 if case["half"] else torch.float32, device=DEV)
    token = torch.empty(B, case["given"], dtype=torch.int32, device=DEV)
    step = max(1, (1 << 28) // (V + case["pad"]))
    for at in range(0, B, step):
        part = 2.5 * torch.randn(min(step, B - at), V + case["pad"], generator=g, device=DEV)
        part[:, ::max(1, V // 61)] += 6.0
        if case["masked"]:   # a grammar that allows an eighth of the vocabulary, in every second row
            odd = part[1::2]
            odd.masked_fill_(torch.rand(odd.shape, generator=g, device=DEV) < 0.875, -math.inf)
        x[at:at + step] = part
        noise = -torch.log(torch.empty(part.shape[0], V, device=DEV).exponential_(generator=g))
        token[at:at + step] = torch.topk(part[:, :V] + noise, case["given"], dim=1).indices   # as the model draws them
    row = torch.arange(B, device=DEV)
    r = torch.rand(B, generator=g, device=DEV)
    return dict(logits=x[:, :V], tokens=token, temperature=torch.where(row % 3 == 1, 0.6 + 0.8 * r, 1.0))


# ---- plain forms ------------------------------------------------------------------------------------------------
def _times_power(x, n):
    """x * 2^n in 32 bits for -200 < n < 200, by two powers from their bits (exact where the result is normal)."""
    a = torch.div(n, 2, rounding_mode="floor").to(torch.int32)
    power = lambda m: ((m + 127) << 23).view(torch.float32)  # noqa: E731
    return x * power(a) * power(n.to(torch.int32) - a)


def _codes(x):
    """Codes [..., dh] and scale bytes [..., dh/32] of rows [..., dh] of finite values."""
    y = x.float().clamp(-LARGEST, LARGEST).unflatten(-1, (-1, 32))
    top = y.abs().amax(-1)
    m, ex = torch.frexp(top)          # top = m * 2^ex with m in [1/2, 1): below 464 * 2^(ex - 9), or twice that
    e = torch.where(top > 0, ex - 9 + (m >= 0.90625).int() + 127, 0).clamp(min=0)
    y = _times_power(y, (127 - e)[..., None])
    a = y.abs()
    _, ex = torch.frexp(a)
    ex = (ex - 1).clamp(min=-6)       # exponent of the value, at least that of the smallest normal one
    n = torch.round(_times_power(a, 3 - ex)).int()         # eighths of a power; 16: the next power
    c = torch.where(n >= 8, ((ex + 7) << 3) + n - 8, n) + 128 * (y < 0).int()
    return c.to(torch.uint8).flatten(-2), e.to(torch.uint8)


def _values(codes, scale):
    """Rows [..., dh] in 32 bits that the codes stand for."""
    c = codes.int()
    ex, man = (c >> 3) & 15, (c & 7).float()
    mag = torch.where(ex == 0, man / 512, _times_power(man + 8, ex - 10))
    x = torch.where(c >= 128, -mag, mag).unflatten(-1, (-1, 32))
    return _times_power(x, (scale.int() - 127)[..., None]).flatten(-2)


def _slot_rows(s, b, at):
    """Pages' rows of slots `at` of sequences `b` (both any shape): which page, which row of it; -1: no page."""
    page, table = s["case"]["page"], s["table"]
    entry = torch.div(at, page, rounding_mode="floor")
    ok = (entry >= 0) & (entry < table.shape[1])
    p = torch.where(ok, table[b, entry.clamp(0, table.shape[1] - 1)].long(), -1)
    return p, at - entry * page


def _gather(s, name, b, at):
    """Rows [..., heads, dh] in 32 bits, zeros where there is no page."""
    p, row = _slot_rows(s, b, at)
    x = s["pages"][name][p.clamp(min=0), :, row]
    x = x.float() if s["case"]["bits"] == 16 else _values(x, s["pages"][name + "_scale"][p.clamp(min=0), :, row])
    return torch.where((p >= 0)[..., None, None], x, 0.0)


def _angles(case, pos):
    """Angles [n, rot/2] in 64 bits."""
    f = torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=DEV),
                  -torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
    if case["scaled"]:   # waves that turn less than once within the trained 8192 positions eight times longer, from four on as is
        stays = ((8192 * f / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * (stays + (1.0 - stays) / 8.0)
    return pos.double()[:, None] * f


def _plain_rotate(s):
    case, out = s["case"], []
    a = _angles(case, s["pos"])
    c, n = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]
    rot, half = case["rot"], case["rot"] // 2
    first, second = ((slice(0, half), slice(half, rot)) if case["pairs"] == "halves"
                     else (slice(0, rot, 2), slice(1, rot, 2)))
    for name in ("q", "k"):
        x = s[name].float()
        y = x.clone()
        y[..., first] = x[..., first] * c - x[..., second] * n
        y[..., second] = x[..., second] * c + x[..., first] * n
        out.append(y.to(torch.bfloat16))
    return dict(q=out[0], k=out[1])


def _plain_store(s):
    case, starts = s["case"], s["start"]
    N, n = s["k_new"].shape[0], case["n"]
    row = torch.arange(N, device=DEV)
    b = (row[:, None] >= starts[None, 1:]).sum(1)          # the sequence of each row
    at = s["first"].long()[b] + row - starts.long()[b]
    p, r = _slot_rows(s, b, at)
    for name, new in (("k", s["k_new"]), ("v", s["v_new"])):
        if case["bits"] == 16:
            s["pages"][name][p, :, r] = new
        else:
            s["pages"][name][p, :, r], s["pages"][name + "_scale"][p, :, r] = _codes(new)
    b = torch.arange(case["B"], device=DEV)[:, None]
    at = s["first"].long()[:, None] + torch.arange(n, device=DEV)
    return {x: _gather(s, x, b, at).transpose(1, 2).to(torch.bfloat16).contiguous() for x in ("k", "v")}


def _plain_attend(s):
    case = s["case"]
    heads, group, dh, page = (case[x] for x in ("heads", "group", "dh", "page"))
    ln, starts = s["length"].long(), s["start"].long()
    N, B = s["q"].shape[0], case["B"]
    out = torch.zeros(N, heads * group, dh, device=DEV)
    lse = torch.zeros(N, heads * group, device=DEV)
    # sequences of about one size together: (first sequence, how many, padded queries)
    counts = _new_counts(case)
    runs = [(0, 1, counts[0]), (1, B - 1, max(counts[1:] or [1]))] if case["mixed"] else [(0, B, max(counts))]
    for b0, nb, nq in runs:
        b = torch.arange(b0, b0 + nb, device=DEV)
        slot = torch.arange(case["T"], device=DEV)
        k, v = (_gather(s, x, b[:, None], slot.expand(nb, -1)).transpose(1, 2) for x in ("k", "v"))
        i = torch.arange(nq, device=DEV)
        mine = i < (starts[b + 1] - starts[b])[:, None]                                  # [nb, nq]
        at = (starts[b][:, None] + i).clamp(max=N - 1)
        q = s["q"][at].float().view(nb, nq, heads, group, dh).permute(0, 2, 1, 3, 4).reshape(nb, heads, nq * group, dh)
        x = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(dh))
        sees = (ln[b] - (starts[b + 1] - starts[b]))[:, None] + i + 1
        sees = sees.clamp(max=case["T"]).repeat_interleave(group, 1)[:, None, :, None]
        x = torch.where(slot < sees, x, -math.inf)
        m = x.amax(-1, keepdim=True)
        p = torch.exp(x - m)
        del x
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v.contiguous()) / total
        back = lambda t: t.view(nb, heads, nq, group, -1).permute(0, 2, 1, 3, 4)[mine]  # noqa: E731
        out[at[mine]] = back(o).reshape(-1, heads * group, dh)
        lse[at[mine]] = back(m + torch.log(total)).reshape(-1, heads * group)
    return dict(out=out.to(torch.bfloat16), lse=lse)


def _plain_logprobs(s):
    top = s["case"]["top"]
    x = s["logits"].float()
    m = x.amax(1, keepdim=True)
    d = (x - m) / s["temperature"][:, None]
    w = torch.exp(d)
    total = w.sum(1, keepdim=True)
    y = torch.log(total)
    entropy = y[:, 0] - torch.where(w > 0, w * d, 0.0).sum(1) / total[:, 0]
    out = dict(logprob=d.gather(1, s["tokens"].long()) - y, entropy=entropy)
    if top:
        down, order = torch.sort(x, descending=True, stable=True)
        out["top_token"] = order[:, :top].to(torch.int32)
        out["top_logprob"] = (down[:, :top] - m) / s["temperature"][:, None] - y
    return out


# ---- one pass -----------------------------------------------------------------------------------------------------
_contexts, _tables = {}, {}


def _context(case):
    """The context that a program keeps for calls of this size."""
    from paper_2604_09244_amd import binding as mv
    key = tuple(sorted((k, v) for k, v in case.items() if k != "name"))
    if key not in _contexts:
        N = _starts(case)[-1] if "T" in case else 1
        _contexts[key] = mv.Context.for_pages(case.get("B", 1), case.get("heads", 1) * case.get("group", 1),
                                              case.get("heads", 1), N, case.get("nq", 1), case.get("T", 1),
                                              case.get("dh", 128))
        if case["kind"] == "rotate":
            how = dict(factor=8.0, low_turns=1.0, high_turns=4.0, trained=8192) if case["scaled"] else {}
            _tables[key] = _contexts[key].rotary_table(case["rot"], case["far"], **how)
    return mv, _contexts[key], _tables.get(key)


def run(state):
    s, case, kind = state, state["case"], state["kind"]
    if not own:
        return dict(rotate=_plain_rotate, store=_plain_store, attend=_plain_attend, logprobs=_plain_logprobs)[kind](s)
    if "handle" not in s:   # what a program keeps beside its tensors
        mv, ctx, table = _context(case)
        s["handle"] = (ctx, table) if "pages" not in s else (ctx, mv.PagedCache(**s["pages"]),
                                                             mv.PageBatch(s["start"], s["length"], s["table"]))
    ctx, *held = s["handle"]
    if kind == "rotate":
        q, k = ctx.rotate(s["q"], s["k"], s["pos"], held[0], interleaved=case["pairs"] == "sides")
        return dict(q=q, k=k)
    if kind == "store":
        ctx.pages_append(*held, s["k_new"], s["v_new"])
        k, v = ctx.pages_read(*held, s["first"], case["n"])
        return dict(k=k, v=v)
    if kind == "attend":
        out, lse = ctx.pages_attention(*held, s["q"], max_q=case["nq"], max_length=case["T"], with_lse=True)
        return dict(out=out, lse=lse)
    logprob, entropy, token, top = ctx.logprobs(s["logits"], s["tokens"], s["temperature"], top=case["top"])
    out = dict(logprob=logprob, entropy=entropy)
    return dict(out, top_token=token, top_logprob=top) if case["top"] else out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "logprobs":
        n = case["B"] * case["V"]
        return {"bytes": (2.0 if case["half"] else 4.0) * n + case["B"] * (8.0 + 8.0 * case["given"] + 8.0 * case["top"]),
                "flops": 5.0 * n}
    heads, dh = case["heads"], case["dh"]
    if kind == "rotate":
        rows = float(case["n"] * heads * (case["group"] + 1))
        return {"bytes": 4.0 * rows * dh + 4.0 * case["n"] * (1 + case["rot"]), "flops": 3.0 * rows * case["rot"]}
    row = 2.0 * dh * case["bits"] / 8 + (2.0 * (dh // 32) if case["bits"] == 8 else 0.0)   # a key and a value row
    ln, new = _lengths(case), _new_counts(case)
    if kind == "store":
        read = heads * float(sum(min(case["n"], -(-t // case["page"]) * case["page"] - (t - m)) for t, m in zip(ln, new)))
        return {"bytes": heads * float(sum(new)) * (4.0 * dh + row) + read * row + 4.0 * dh * heads * case["B"] * case["n"],
                "flops": 6.0 * dh * heads * float(sum(new))}
    group = case["group"]
    seen = heads * group * float(sum(m * (t - m) + m * (m + 1) // 2 for t, m in zip(ln, new)))
    return {"bytes": heads * float(sum(ln)) * row + sum(new) * heads * group * (4.0 * dh + 4.0),
            "flops": 4.0 * dh * seen}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------
def _power64(e):
    """2^e by a table of Python's own powers."""
    return torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device=DEV)[e.long() + 300]


def _decode64(codes, scale):
    """Values of codes by the format's definition."""
    c = codes.double()
    sign = torch.where(c >= 128, -1.0, 1.0).double()
    c = c % 128
    ex, man = torch.floor(c / 8), c % 8
    mag = torch.where(ex == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * _power64(ex - 7))
    return sign * mag * _power64(scale.int() - 127).repeat_interleave(32, -1)


def _nearest64(x):
    """Rows as the cache holds them in 8 bits: each block's smallest power under which all stays below 464, each value
    the nearest one of three mantissa bits (of two equally near ones the even)."""
    y = x.double().clamp(-247 * 2.0 ** 120, 247 * 2.0 ** 120).unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.frexp(top / 464.0).exponent             # top / 464 below 2^e, and not below 2^(e - 1)
    e = torch.where(top > 0, e, -127).clamp(min=-127)
    a = (y * _power64(-e)).abs()
    step = _power64(torch.frexp(a.clamp(min=2.0 ** -6)).exponent - 4)
    return (torch.sign(y) * torch.round(a / step) * step * _power64(e)).flatten(-2)


def _held64(s, name, b, t):
    """[heads, t, dh] of sequence b's first t slots."""
    pages = s["table"][b, :-(-t // s["case"]["page"])].long()
    x = s["pages"][name][pages]
    x = x.double() if s["case"]["bits"] == 16 else _decode64(x, s["pages"][name + "_scale"][pages])
    return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :t]


def _exact_attend(case, s):
    group, dh = case["group"], case["dh"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    at = _starts(case)
    for b, (t, m) in enumerate(zip(_lengths(case), _new_counts(case))):
        k, v = _held64(s, "k", b, t), _held64(s, "v", b, t)
        last = t - m + torch.arange(m, device=DEV)
        hidden = torch.arange(t, device=DEV) > last[:, None]
        for h in range(case["heads"] * group):
            q = s["q"][at[b]:at[b + 1], h].double()
            x = torch.mm(q, k[h // group].T.contiguous()) / math.sqrt(dh)
            x.masked_fill_(hidden, -math.inf)
            lse[at[b]:at[b + 1], h] = torch.logsumexp(x, -1)
            out[at[b]:at[b + 1], h] = torch.mm(torch.softmax(x, -1), v[h // group].contiguous())
    return dict(out=out, lse=lse)


def _exact_rotate(case, s):
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
    f = 10000.0 ** (-2.0 * i / case["rot"])
    if case["scaled"]:
        turns = 8192.0 * f / (2.0 * math.pi)
        keep = torch.clamp((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = (1.0 - keep) * f / 8.0 + keep * f
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"].double()[:, None] * f)[:, None]
    out = {}
    for name in ("q", "k"):
        y = s[name].double()
        x = y[..., :case["rot"]]
        if case["pairs"] == "halves":
            z = torch.complex(*(t.contiguous() for t in x.chunk(2, -1))) * turn
            z = torch.cat([z.real, z.imag], -1)
        else:
            z = torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()) * turn).flatten(-2)
        out[name] = torch.cat([z, y[..., case["rot"]:]], -1)
    return out


def _exact_store(case, s):
    at, out = _starts(case), {}
    for name in ("k", "v"):
        out[name] = torch.zeros(case["B"], case["heads"], case["n"], case["dh"], dtype=torch.float64, device=DEV)
        for b, m in enumerate(_new_counts(case)):
            x = s[name + "_new"][at[b]:at[b + 1]].transpose(0, 1)
            out[name][b, :, :m] = x.double() if case["bits"] == 16 else _nearest64(x)
    return out


def _exact_logprobs(case, s):
    parts = []
    for at in range(0, case["B"], 64):
        x = s["logits"][at:at + 64].double() / s["temperature"][at:at + 64, None].double()
        y = torch.log_softmax(x, 1)
        entropy = -torch.where(torch.isfinite(y), torch.exp(y) * y, 0.0).sum(1)
        part = dict(logprob=y.gather(1, s["tokens"][at:at + 64].long()), entropy=entropy)
        if case["top"]:
            part.update(top_logprob=torch.topk(y, case["top"], dim=1).values)
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return dict(logprob=out["logprob"], entropy=out["entropy"], top_token=None, top_logprob=out["top_logprob"]) \
        if case["top"] else out


def exact(case, seed):
    s = prepare(case, seed)
    return dict(attend=_exact_attend, rotate=_exact_rotate, store=_exact_store, logprobs=_exact_logprobs)[case["kind"]](
        case, s)

"""A prompt's pruned prefill, then an answer of some tokens from 4-bit caches.

    python examples/answer.py [--workload single_view] [--tokens 32] [--budget 256] [--layers 8]

Seeded weights and inputs of the named workload; the output head is a random matrix, the
embedding its transpose.  Prints each step's tokens and the time of prefill and steps."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_09244_amd import binding as mv            # noqa: E402
from paper_2604_09244_amd import workloads as W           # noqa: E402
from paper_2604_09244_amd.answer import Answer            # noqa: E402


def answer(wl, layers, tokens, budget, vocabulary, seed=0, temperature=0.8, top_k=50, top_p=0.95, min_p=0.0):
    """Token ids and their probabilities [B, tokens], milliseconds of the prefill and of all steps."""
    ctx = mv.Context(wl.B, wl.S, wl.D, wl.H, wl.F, wl.nt,
                     min_bytes=Answer.workspace_bytes(wl.B, wl.S, wl.D, wl.H, wl.F, tokens))
    plan = mv.PrefillPlan(ctx, mv.LayerCfg(wl.D, wl.H, wl.dh, wl.F, wl.rms_eps), layers, wl.B, wl.n2, wl.n3,
                          wl.nt, wl.k_total, min(wl.p, len(layers)), rope_base=wl.rope_base, rope_len=wl.S + tokens)
    loop = Answer(plan, tokens, budget, first_pos=4, n_recent=min(32, (budget or 64) // 2))
    g = torch.Generator(device="cuda").manual_seed(seed)
    head = torch.randn(vocabulary, wl.D, generator=g, device="cuda").mul_(wl.D ** -0.5).to(torch.bfloat16)
    u = torch.rand(tokens, wl.B, generator=g, device="cuda")
    x, pos = W.hidden_states(wl, device="cuda")
    at = torch.full((wl.B, 1), wl.S, dtype=torch.int32, device="cuda")
    ids = torch.empty(wl.B, tokens, dtype=torch.int32, device="cuda")
    probs = torch.empty(wl.B, tokens, dtype=torch.float32, device="cuda")
    settings = [torch.full((wl.B,), v, dtype=d, device="cuda")
                for v, d in ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32))]
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    marks[0].record()
    last = loop.prefill(x, pos, W.scoring_bias(wl, device="cuda"), on_the_fly=True)[:, -1]
    marks[1].record()
    for t in range(tokens):
        token, prob = ctx.sample(last @ head.T, u[t], *settings)
        ids[:, t], probs[:, t] = token, prob
        if t + 1 < tokens:
            last = loop.step(head[token.long()][:, None], at)[:, 0]
            at += 1
    marks[2].record()
    torch.cuda.synchronize()
    ctx.close()
    return ids, probs, marks[0].elapsed_time(marks[1]), marks[1].elapsed_time(marks[2])


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--workload", default="single_view", choices=sorted(W.WORKLOADS))
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--budget", type=int, default=256, help="rows kept a layer; 0: no eviction")
    ap.add_argument("--layers", type=int, default=0, help="0: the workload's")
    ap.add_argument("--vocabulary", type=int, default=32768)
    a = ap.parse_args()
    wl = W.WORKLOADS[a.workload]
    layers = [mv.pack_layer(W.layer_weights(wl, l, device="cuda")) for l in range(a.layers or wl.L)]
    for _ in range(2):         # (the first run loads the code)
        ids, probs, ms_prefill, ms_steps = answer(wl, layers, a.tokens, a.budget or None, a.vocabulary)
    for b in range(wl.B):
        print(f"sample {b}:", " ".join(str(i) for i in ids[b].tolist()))
    print(f"{a.workload}: {wl.S} tokens in {ms_prefill:.2f} ms, then {a.tokens} tokens a sample in {ms_steps:.2f} ms")


if __name__ == "__main__":
    main()

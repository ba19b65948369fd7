"""Layers with caches: what a prefill leaves in them, layers over them, and the answer's loop."""
import ctypes as C
import dataclasses
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle as O
from oracle import answering as A
from paper_2604_09244_amd import binding as mv
from paper_2604_09244_amd import workloads as W
from paper_2604_09244_amd.answer import Answer
from answer_helpers import garbage_cache, held, ints
from helpers import assert_layer_close, layer_cfg, oracle_weights, to64

pytestmark = pytest.mark.gpu
TINY = dataclasses.replace(W.WORKLOADS["tiny"], B=2)


def _plan(wl, L, p, room=8, spare=0):
    layers_cpu = [W.layer_weights(wl, l) for l in range(L)]
    ctx = mv.Context(wl.B, wl.S, wl.D, wl.H, wl.F, wl.nt,
                     min_bytes=Answer.workspace_bytes(wl.B, wl.S, wl.D, wl.H, wl.F, room) + spare)
    layers = [mv.pack_layer({k: v.cuda() for k, v in w.items()}) for w in layers_cpu]
    return mv.PrefillPlan(ctx, layer_cfg(wl), layers, wl.B, wl.n2, wl.n3, wl.nt, wl.k_total, p,
                          rope_base=wl.rope_base, rope_len=wl.S + room), layers_cpu


def _keys_values(x, pos, w, wl):
    """A layer's rotated keys and its values on one sample, [rows, H, dh] in fp64."""
    q, k, u = O.mvla_oracle._qk(x, pos, w, wl.H, wl.rms_eps, wl.rope_base)
    return q, k, (u @ w["wv"].T).reshape(len(x), wl.H, -1)


def _near_held(got, want, powers, what):
    """Cached values against those of the formula.  A block's power of two s puts its values at most s from their
    level (levels reach 6 and lie 2 apart at most, values stay below 7); the block's own power may be one up where
    the stored bf16 value is at the border, which s of the cache covers.  The values are a projection of
    bf16 operands: 2e-2 of their RMS, the layers' bar."""
    scale = np.repeat(2.0 ** (powers.astype(np.float64) - 127), 32, axis=-1)
    bad = np.abs(got - want) > scale * (1 + 2.0 ** -7) + 2e-2 * np.sqrt(np.mean(want ** 2))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off"
    # and not all of them at the bound's reach: four bits leave a relative RMS error near 0.1
    assert np.sqrt(np.mean((got - want) ** 2)) < 0.2 * np.sqrt(np.mean(want ** 2)), what


def _check_rows(cache, b, x, pos, w, wl, what):
    _, k, v = _keys_values(x, pos, w, wl)
    n = len(x)
    hk, hv = held(cache, b, n)
    _near_held(hk, k.transpose(1, 0, 2), cache.k_scale[b, :, :n].cpu().numpy(), what + " keys")
    _near_held(hv, v.transpose(1, 0, 2), cache.v_scale[b, :, :n].cpu().numpy(), what + " values")
    assert (cache.pos[b, :, :n].cpu().numpy() == pos).all(), what
    assert (cache.weight[b, :, :n] == 0).all(), what


@pytest.mark.parametrize("options", [dict(on_the_fly=True), dict(fused_prune=False),
                                     dict(on_the_fly=True, smooth_step=2)])
def test_a_prefill_leaves_every_layers_rows_and_its_result_unchanged(options):
    wl, L, p = TINY, 2, 1
    plan, w = _plan(wl, L, p)
    x, pos = W.hidden_states(wl, device="cuda")
    kb = W.scoring_bias(wl, device="cuda")
    plan.sal_hat.fill_(0.25)
    want = plan.run(x, pos, kb, **options).clone()
    kept = plan.prune["kept_idx"].clone()
    plan.sal_hat.fill_(0.25)
    caches = [garbage_cache(wl.B, wl.H, wl.dh, n) for n in (wl.S, wl.k_total + wl.nt + 40)]
    got = plan.run(x, pos, kb, caches=(mv.Cache4C * L)(*[c._c for c in caches]), **options)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(plan.prune["kept_idx"], kept)
    for b in range(wl.B):
        _check_rows(caches[0], b, to64(x[b]), pos[b].cpu().numpy(), oracle_weights(w[0]), wl, f"layer 0 sample {b}")
        _check_rows(caches[1], b, to64(plan.h_kept[0][b]), plan.prune["pos"][b].cpu().numpy(), oracle_weights(w[1]),
                    wl, f"layer 1 sample {b}")
    n = wl.k_total + wl.nt
    assert (caches[1].k[:, :, n:] == 255).all() and (caches[1].pos[:, :, n:] == -77).all()   # no row past the last
    plan.ctx.close()


def test_a_cold_start_leaves_all_rows_in_every_cache():
    wl, L = TINY, 3
    plan, w = _plan(wl, L, 1)
    x, pos = W.hidden_states(wl, device="cuda")
    caches = [garbage_cache(wl.B, wl.H, wl.dh, wl.S) for _ in range(L)]
    want = plan.run(x, pos, None, smooth_step=1).clone()
    got = plan.run(x, pos, None, smooth_step=1, caches=(mv.Cache4C * L)(*[c._c for c in caches]))
    assert torch.equal(got, want)
    for b in range(wl.B):
        _check_rows(caches[0], b, to64(x[b]), pos[b].cpu().numpy(), oracle_weights(w[0]), wl, f"sample {b}")
    for c in caches[1:]:
        assert (c.pos[:, :, :wl.S] == pos[:, None]).all() and (c.weight[:, :, :wl.S] == 0).all()
    plan.ctx.close()


def test_pruning_before_any_layer_leaves_kept_rows_everywhere():
    wl, L = TINY, 2
    plan, w = _plan(wl, L, 0)
    x, pos = W.hidden_states(wl, device="cuda")
    want = plan.run(x, pos, None, on_the_fly=True).clone()
    n = wl.k_total + wl.nt
    caches = [garbage_cache(wl.B, wl.H, wl.dh, n + 32) for _ in range(L)]
    got = plan.run(x, pos, None, on_the_fly=True, caches=(mv.Cache4C * L)(*[c._c for c in caches]))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    at, kept = plan.prune["pos"], plan.prune["kept_idx"].cpu()
    for c in caches:
        assert (c.pos[:, :, :n] == at[:, None]).all() and (c.pos[:, :, n:] == -77).all()
    for b in range(wl.B):
        _check_rows(caches[0], b, to64(x[b])[kept[b].numpy()], at[b].cpu().numpy(), oracle_weights(w[0]), wl, f"sample {b}")
    plan.ctx.close()


def _decode(plan, caches, x, pos, length, n_new=None, max_length=None, accumulate=1, h=None):
    B, n, D = x.shape
    h = h or [torch.empty_like(x) for _ in range(2)]
    y = C.c_void_p()
    rc = mv.load().mvla_decode_step(plan.ctx.handle, C.byref(plan.cfg), plan._layer_array,
                                    (mv.Cache4C * len(caches))(*[c._c for c in caches]), len(caches),
                                    x.data_ptr(), pos.data_ptr(), B, n, mv._ptr(n_new), length.data_ptr(),
                                    max_length or max(c.capacity for c in caches), accumulate,
                                    (C.c_void_p * 2)(*[t.data_ptr() for t in h]), C.byref(y))
    return rc, next((t for t in h if t.data_ptr() == y.value), None)


@pytest.mark.parametrize("n,n_new,before", [(1, None, (0, 0)), (1, None, (5, 40)), (4, (4, 2), (33, 0)),
                                            (3, (0, 3), (7, 100)), (20, (20, 11), (90, 64))])
def test_a_layer_over_its_cache(n, n_new, before):
    """The layer's formula in fp64 with the keys and values that the cache holds afterwards."""
    wl, B = TINY, 2
    plan, w = _plan(wl, 1, 1, room=64, spare=16 << 20)
    ow = oracle_weights(w[0])
    g = torch.Generator().manual_seed(n)
    cache = garbage_cache(B, wl.H, wl.dh, 128)
    old = torch.randn(B, max(before) + 1, wl.H, wl.dh, generator=g).to(torch.bfloat16).cuda()
    steps = torch.arange(old.shape[1], dtype=torch.int32).repeat(B, 1).cuda()
    # (the first `before` rows of a sample: appended as the last `before` of a run that starts at slot 0)
    plan.ctx.cache_append(cache, old, old.flip(1).contiguous(), steps, ints(*before), ints(*before))
    x, pos = W.hidden_states(wl, B=B)
    x, pos = x[:, :n].contiguous(), (pos[:, :n] + 3).contiguous()
    count = [n] * B if n_new is None else list(n_new)
    length = ints(*[a + c for a, c in zip(before, count)])
    rc, y = _decode(plan, [cache], x.cuda(), pos.cuda(), length, None if n_new is None else ints(*n_new))
    assert rc == 0
    for b in range(B):
        c, total = count[b], before[b] + count[b]
        if c == 0:
            continue
        x64 = to64(x[b, :c])
        q, k, v = _keys_values(x64, pos[b, :c].numpy(), ow, wl)
        hk, hv = held(cache, b, total)
        _near_held(hk[:, before[b]:], k.transpose(1, 0, 2), cache.k_scale[b, :, before[b]:total].cpu().numpy(), "keys")
        _near_held(hv[:, before[b]:], v.transpose(1, 0, 2), cache.v_scale[b, :, before[b]:total].cpu().numpy(), "values")
        o, prob = A.cache_attention(q, hk, hv, c, wl.dh ** -0.5)
        x1 = x64 + o.reshape(c, -1) @ ow["wo"].T
        t = O.rmsnorm(x1, ow["g_mlp"], wl.rms_eps)
        gate = t @ ow["w_gate"].T
        want = x1 + (gate / (1 + np.exp(-gate)) * (t @ ow["w_up"].T)) @ ow["w_down"].T
        assert_layer_close(y[b, :c], want, f"layer over a cache, sample {b}", wl.D)
        # weights: sums over the queries of probabilities whose logits carry bf16 q (2^-8 of them)
        got = cache.weight[b, :, :total].cpu().numpy()
        assert np.allclose(got.sum(-1), c, rtol=1e-5)
        assert np.allclose(got, prob.sum(0), rtol=6e-2, atol=2e-5 * c)
    plan.ctx.close()


def test_layers_over_their_caches_run_in_order():
    """Three layers in one call against three calls of one layer each: the same bits."""
    wl, B, L = TINY, 2, 3
    plan, _ = _plan(wl, L, 1, room=64, spare=16 << 20)
    x, pos = W.hidden_states(wl, B=B, device="cuda")
    x, pos = x[:, :5].contiguous(), pos[:, :5].contiguous()
    a, b = ([garbage_cache(B, wl.H, wl.dh, 64 if l else 32) for l in range(L)] for _ in range(2))
    length = ints(5, 5).repeat(L, 1)
    rc, y = _decode(plan, a, x, pos, length)
    assert rc == 0
    h, whole = x, plan._layer_array
    for l in range(L):
        plan._layer_array = (mv.LayerWeightsC * 1)(plan.structs[l])
        rc, h = _decode(plan, [b[l]], h, pos, length[l])
        assert rc == 0
    plan._layer_array = whole
    assert torch.equal(y, h)
    for l in range(L):
        assert torch.equal(a[l].k[:, :, :5], b[l].k[:, :, :5]) and torch.equal(a[l].weight[:, :, :5], b[l].weight[:, :, :5])
    plan.ctx.close()


def test_decode_refuses_what_it_cannot_run():
    wl, B = TINY, 2
    plan, _ = _plan(wl, 1, 1, room=32)
    x = torch.zeros(B, 2, wl.D, dtype=torch.bfloat16, device="cuda")
    pos, length = ints(0, 1).repeat(B, 1), ints(2, 2)
    cache = mv.Cache4.empty(B, wl.H, wl.dh, 64)
    spare = torch.empty_like(x)
    assert _decode(plan, [cache], x, pos, length)[0] == 0
    assert _decode(plan, [cache], x, pos, length, max_length=-1)[0] == -1
    assert _decode(plan, [cache], x, pos, length, h=[x, spare])[0] == -1
    assert _decode(plan, [cache], x, pos, length, h=[spare, spare])[0] == -1
    assert _decode(plan, [mv.Cache4.empty(B + 1, wl.H, wl.dh, 64)], x, pos, length)[0] == -1
    assert _decode(plan, [mv.Cache4.empty(B, 2 * wl.H, wl.dh, 64)], x, pos, length)[0] == -1
    big = mv.Cache4.empty(B, wl.H, wl.dh, 1 << 20)
    assert _decode(plan, [big], x, pos, length)[0] == -2      # its weights need more workspace than the context has
    kept = (mv.Cache4C * 1)(mv.Cache4.empty(wl.B, wl.H, wl.dh, 32)._c)
    xs, ps = W.hidden_states(wl, device="cuda")
    with pytest.raises(mv.MvlaError):                         # a cache too short for the prefill's rows
        plan.run(xs, ps, None, caches=kept)
    plan.ctx.close()


def test_an_answer_on_its_own_stream_and_under_a_budget():
    """Steps with eviction: lengths, what stays, the same bits again, the same bits on another stream."""
    wl, L, p, steps, budget = TINY, 3, 2, 6, 24
    x, pos = W.hidden_states(wl, device="cuda")
    torch.cuda.synchronize()
    runs = []
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            plan, _ = _plan(wl, L, p)
            loop = Answer(plan, steps, budget, first_pos=2, n_recent=3)
            with pytest.raises(RuntimeError):
                loop.step(x[:, :1].contiguous(), pos[:, :1].contiguous())
            for _ in range(2):
                last = loop.prefill(x, pos, None, on_the_fly=True)[:, -1:]
                at = torch.full((wl.B, 1), wl.S, dtype=torch.int32, device="cuda")
                outs = []
                for t in range(steps):
                    y = loop.step(last.contiguous(), at)
                    last = y.clone()
                    outs.append(last)
                    at += 1
                runs.append((torch.stack(outs), loop.length.clone(), [c.pos[:, :, :budget].clone() for c in loop.caches]))
            with pytest.raises(RuntimeError):
                loop.step(last, at)
            stream.synchronize()
            plan.ctx.close()
    for outs, length, at in runs:
        assert torch.isfinite(outs).all() and torch.equal(outs, runs[0][0])
        assert (length == budget).all()
        for l in range(L):
            assert torch.equal(at[l], runs[0][2][l])
            for row in at[l].flatten(0, 1).tolist():
                assert len(set(row)) == budget
                assert {wl.S + steps - 1 - i for i in range(3)} <= set(row)
                if l < p:                                      # (behind the pruning step only kept positions exist)
                    assert {0, 1} <= set(row)


def test_steps_replay_from_a_graph():
    """The layers' calls of a step captured once; replays on restored caches give the eager bits."""
    wl, L = TINY, 2
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        plan, _ = _plan(wl, L, 1)
        loop = Answer(plan, 8)
        x, pos = W.hidden_states(wl, device="cuda")
        last = loop.prefill(x, pos, None, on_the_fly=True)[:, -1:].contiguous()
        at = torch.full((wl.B, 1), wl.S, dtype=torch.int32, device="cuda")
        length = loop.length + 1
        state = [[getattr(c, f).clone() for f in ("k", "v", "k_scale", "v_scale", "pos", "weight")] for c in loop.caches]

        def restore():
            for c, old in zip(loop.caches, state):
                for f, t in zip(("k", "v", "k_scale", "v_scale", "pos", "weight"), old):
                    getattr(c, f).copy_(t)

        h = [torch.empty_like(last) for _ in range(2)]
        want = _decode(plan, loop.caches, last, at, length, h=h)[1].clone()
        weights = [c.weight.clone() for c in loop.caches]
        restore()
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            rc, y = _decode(plan, loop.caches, last, at, length, h=h)
        assert rc == 0
        for _ in range(3):
            restore()
            y.zero_()
            g.replay()
            st.synchronize()
            assert torch.equal(y, want)
            for l, c in enumerate(loop.caches):
                n = loop.rows[l] + 1
                assert torch.equal(c.weight[:, :, :n], weights[l][:, :, :n])
        plan.ctx.close()


def test_the_example_gives_tokens():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer.py")
    spec = importlib.util.spec_from_file_location("answer_example", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    layers = [mv.pack_layer(W.layer_weights(TINY, l, device="cuda")) for l in range(TINY.L)]
    runs = [mod.answer(TINY, layers, 5, 16, 1000) for _ in range(2)]
    ids, probs = runs[0][:2]
    assert ((ids >= 0) & (ids < 1000)).all() and ((probs > 0) & (probs <= 1)).all()
    assert torch.equal(ids, runs[1][0]) and torch.equal(probs, runs[1][1])

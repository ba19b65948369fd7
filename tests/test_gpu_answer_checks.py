"""What an answer's loop refuses, and what a refusal leaves."""
import pytest
import torch

from paper_2604_09244_amd import binding as mv
from paper_2604_09244_amd import workloads as W
from paper_2604_09244_amd.answer import Answer
from helpers import layer_cfg
from test_gpu_answer import TINY, _plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rope_len", [None, TINY.S + 7])
def test_a_rotary_table_that_ends_before_the_answer(rope_len):
    """Positions behind the table would all be rotated as its last one."""
    wl = TINY
    ctx = mv.Context(wl.B, wl.S, wl.D, wl.H, wl.F, wl.nt,
                     min_bytes=Answer.workspace_bytes(wl.B, wl.S, wl.D, wl.H, wl.F, 8))
    layers = [mv.pack_layer(W.layer_weights(wl, l, device="cuda")) for l in range(2)]
    plan = mv.PrefillPlan(ctx, layer_cfg(wl), layers, wl.B, wl.n2, wl.n3, wl.nt, wl.k_total, 1, rope_base=wl.rope_base,
                          rope_len=rope_len)
    with pytest.raises(ValueError, match="rope_len"):
        Answer(plan, 8)
    if rope_len:
        Answer(plan, 7)                         # (its positions are there)
    ctx.close()


def test_a_cold_start_is_refused_by_an_error():
    """(not by an assertion, which an optimised interpreter leaves out)"""
    plan, _ = _plan(TINY, 2, 1)
    loop = Answer(plan, 4)
    x, pos = W.hidden_states(TINY, device="cuda")
    with pytest.raises(ValueError, match="cold start"):
        loop.prefill(x, pos, None, smooth_step=1)
    with pytest.raises(RuntimeError):           # nothing was filled
        loop.step(x[:, :1].contiguous(), pos[:, :1].contiguous())
    loop.prefill(x, pos, None, smooth_step=2)
    plan.ctx.close()


def test_a_refused_step_leaves_the_answer_as_it_was():
    """A step that the library refuses (its input lies in the buffer that a step writes) counts for nothing."""
    outs, lengths = [], []
    x, pos = W.hidden_states(TINY, device="cuda")
    for refuse in (False, True):
        plan, _ = _plan(TINY, 2, 1)
        loop = Answer(plan, 3, 40)
        last = loop.prefill(x, pos, None, on_the_fly=True)[:, -1:].contiguous()
        at = torch.full((TINY.B, 1), TINY.S, dtype=torch.int32, device="cuda")
        run = []
        for t in range(3):
            y = loop.step(last, at)
            if refuse:
                before = loop.length.clone()
                with pytest.raises(mv.MvlaError if t < 2 else RuntimeError):
                    loop.step(y, at)
                assert torch.equal(loop.length, before)
            last = y.clone()
            run.append(last)
            at += 1
        outs.append(torch.stack(run)), lengths.append(loop.length.clone())
        plan.ctx.close()
    assert torch.equal(outs[0], outs[1]) and torch.equal(lengths[0], lengths[1])


def test_a_context_without_the_steps_workspace():
    """Refused before an answer starts, not at a step of it."""
    wl = TINY
    ctx = mv.Context(wl.B, wl.S, wl.D, wl.H, wl.F, wl.nt)
    layers = [mv.pack_layer(W.layer_weights(wl, l, device="cuda")) for l in range(2)]
    plan = mv.PrefillPlan(ctx, layer_cfg(wl), layers, wl.B, wl.n2, wl.n3, wl.nt, wl.k_total, 1, rope_base=wl.rope_base,
                          rope_len=wl.S + 60000)
    assert ctx.workspace.numel() < Answer.workspace_bytes(wl.B, wl.S, wl.D, wl.H, wl.F, 60000)
    with pytest.raises(mv.MvlaError, match="workspace"):
        Answer(plan, 60000)
    Answer(plan, 60000, 200)                    # (under a budget the caches stay short)
    ctx.close()


def test_an_answer_whose_context_has_another_stream():
    """Called under one stream, with a context bound to another that is busy: what a step does to its lengths waits for
    the steps before it, as everything else of it does."""
    x, pos = W.hidden_states(TINY, device="cuda")
    tokens = torch.randn(4, TINY.B, 1, TINY.D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    at = [torch.full((TINY.B, 1), TINY.S + t, dtype=torch.int32, device="cuda") for t in range(4)]
    a = torch.randn(8192, 8192, device="cuda")
    runs = []
    for busy in (False, True):
        plan, _ = _plan(TINY, 2, 1)
        loop = Answer(plan, 4, 40, n_recent=2)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        plan.ctx.set_stream(side)
        outs = []
        for turn in range(2):
            if busy:
                with torch.cuda.stream(side):
                    for _ in range(4):
                        b = a @ a               # (milliseconds of work before the prefill)
            loop.prefill(x, pos, None, on_the_fly=True)
            for t in range(4):
                y = loop.step(tokens[t], at[t])
                with torch.cuda.stream(side):
                    outs.append(y.clone())
        torch.cuda.synchronize()
        runs.append((torch.stack(outs), loop.length.clone(), [c.pos[:, :, :40].clone() for c in loop.caches]))
        plan.ctx.close()
    for got, want in zip(runs[1], runs[0]):
        assert all(torch.equal(g, w) for g, w in zip(got, want)) if isinstance(got, list) else torch.equal(got, want)

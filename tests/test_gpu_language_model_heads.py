"""Whole training iterations with the operators around attention and at the vocabulary together: queries and keys normalised and turned
by position, a head that scores tokens, a student that learns from a teacher's lists, a policy's gradient through both; against the
oracle step by step, and captured."""
from dataclasses import replace

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import steps as St
import mp_inputs as I
from oracle import FP64, MIXED
from oracle import layers as L
from oracle import models as Mo
from gpu_util import *
from test_gpu_configs import GRAD_TOL, _f64, _graph_step, _snapshot, teacher_forced
from test_gpu_language_model import ADAMW, BASE, batches as batches_

HEAD = replace(I.C4_SMALL, tokens=200, d_model=192, vocab=1003, opt=ADAMW, scale=I.ScaleCfg(init_scale=2.0 ** 12, growth_interval=3))


def batches(wl, seed=0):
    def at(k):
        out = batches_(wl, seed)(k)
        out["positions"] = wl.positions(out.get("doc_start", np.arange(0, wl.tokens + 1, wl.seq_len))) + 100000 * k
        return out
    return at


def oracle_of(wl):
    return Mo.make_transformer_fwd_bwd(wl.n_layers, wl.n_seq, wl.seq_len, wl.n_heads, wl.causal, wl.rope_base)


def lists(wl, seed=0):
    """Hidden states, targets and lists of other values for each step; every fourth token's list ends early."""
    def at(k):
        r = np.random.default_rng([seed, k])
        ids = np.argsort(r.random((wl.tokens, wl.vocab)), 1)[:, :wl.teacher_top].astype(np.int32)
        ids[::4, r.integers(0, wl.teacher_top):] = -1
        logp = np.log(r.dirichlet(np.ones(wl.teacher_top + 1), wl.tokens)[:, :-1]).astype(np.float32)
        return {"h": r.standard_normal((wl.tokens, wl.d_model)).astype(np.float32), "teacher_ids": ids, "teacher_logp": logp,
                "targets": r.integers(0, wl.vocab, wl.tokens).astype(np.int32)}
    return at


@pytest.mark.parametrize("kw", [dict(rope_axes=1, causal=True, qk_norm=True), dict(rope_axes=3, n_docs=5, qk_norm=True, vocab=301),
                                dict(rope_axes=2), dict(rope_axes=1, rope_base=500.0, qk_norm=True, d_model=128, n_heads=1),
                                dict(rope_axes=1, qk_norm=True, seq_len=1, n_seq=61), dict(rope_axes=4, causal=True, d_model=256, n_heads=8)])
@pytest.mark.parametrize("opts", [dict(), dict(prechecked=True, flat_update=True, two_streams=True)])
def test_iterations_with_turned_heads(kw, opts):
    wl = replace(BASE, **kw)
    teacher_forced(St.TransformerStep(wl, **opts), wl, oracle_of(wl), None, 3, batch_fn=batches(wl), grad_mode="vs_fp64")


def test_norms_of_heads_learn():
    wl = replace(BASE, rope_axes=1, causal=True, qk_norm=True)
    step = St.TransformerStep(wl, prechecked=True, flat_update=True)
    step.set_batch(batches(wl)(0))
    step.step()
    for n in ("l0.qn_g", "l0.kn_g", "l1.qn_g", "l1.kn_g"):
        assert n in step.P.names and not torch.equal(step.P.w32[n], torch.ones_like(step.P.w32[n])) and step.P.g16[n].shape == (64,)


def test_captured_iterations_take_every_batch():
    wl = replace(BASE, rope_axes=2, causal=True, n_docs=7, vocab=301, qk_norm=True, scale=I.ScaleCfg(init_scale=2.0 ** 24, growth_interval=3))
    eager, graphed = (St.TransformerStep(wl, prechecked=True, flat_update=True) for _ in range(2))
    for s in (eager, graphed):
        s.set_batch(batches(wl, 1)(0))
        s.step()
    graph = _graph_step(graphed)
    for k in range(1, 12):
        for s in (eager, graphed):
            s.set_batch(batches(wl, 1)(k))
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert torch.equal(eager.P.w32_arena, graphed.P.w32_arena) and torch.equal(eager.P.w16_arena, graphed.P.w16_arena), k
    a, b = eager.state(), graphed.state()
    assert (a.scale, a.opt_step, a.skipped_steps) == (b.scale, b.opt_step, b.skipped_steps) and 0 < a.skipped_steps < 11


@pytest.mark.parametrize("kw", [dict(teacher_top=8), dict(teacher_top=20, temperature=2.0, soft_weight=4.0, hard_weight=0.5, tail=True),
                                dict(teacher_top=1, vocab=11, tail=True), dict(teacher_top=64, hard_weight=1.0, vocab=20000, tokens=40)])
@pytest.mark.parametrize("opts", [dict(), dict(prechecked=True, flat_update=True)])
def test_iterations_of_a_student(kw, opts):
    wl = replace(HEAD, **kw)
    step = St.XentStep(wl, **opts)
    teacher_forced(step, wl, Mo.make_distill_head_fwd_bwd(wl.temperature, wl.soft_weight, wl.hard_weight, wl.tail), None, 4, batch_fn=lists(wl))
    step.forward_backward()
    assert step.logits.shape == (wl.tokens, wl.vocab) and np.isfinite(np32(step.logits)).all()


def test_captured_iterations_of_a_student():
    """With the loss finished by the launch that ends the iteration, as step() has it."""
    wl = replace(HEAD, teacher_top=20, tail=True, hard_weight=0.25)
    eager, graphed = (St.XentStep(wl, prechecked=True, flat_update=True) for _ in range(2))
    for s in (eager, graphed):
        s.set_batch(lists(wl, 1)(0))
        s.step()
    graph = _graph_step(graphed)
    for k in range(1, 6):
        for s in (eager, graphed):
            s.set_batch(lists(wl, 1)(k))
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert torch.equal(eager.P.w32_arena, graphed.P.w32_arena) and float(eager.loss) == float(graphed.loss), k
    eager.forward_backward()
    graphed.step()
    assert float(eager.loss) == float(graphed.loss)


@pytest.mark.parametrize("vocab,top,temperature", [(1003, 20, 1.0), (1003, 0, 0.5), (32768, 128, 2.0), (11, 11, 1.0)])
def test_scores(vocab, top, temperature):
    """Of the logits that the head's own product made, as 64 bits have them; tolerances of 2^-24 as counted where the operator is tested:
    200 + 8 |z|, an entropy times 1 + ln(vocab)."""
    wl = replace(HEAD, vocab=vocab)
    step = St.XentStep(wl)
    step.set_batch(wl.batch())
    before = step.P.w32_arena.clone()
    got = step.score(top, temperature)
    x = np32(step.rows16[:, :vocab]).astype(np.float64)
    c = float(np.float32(1.0 / temperature))
    logp, entropy, lse, ids, tops = L.token_logprobs(FP64, x, wl.batch()["targets"], c, top)
    tol = 2.0 ** -24 * (200 + 8 * np.abs(x).max(1) * c)
    for n, want, t in (("logp", logp, tol), ("entropy", entropy, tol * (1 + np.log(vocab))), ("lse", lse, tol)):
        assert np.all(np.abs(got[n].double().cpu().numpy() - want) <= t), n
    if top:
        assert np.array_equal(got["ids"].cpu().numpy(), ids)
        assert np.all(np.abs(got["top_logp"].double().cpu().numpy() - tops) <= tol[:, None])
    else:
        assert set(got) == {"logp", "entropy", "lse"}
    assert torch.equal(before, step.P.w32_arena)
    again = step.score(top, temperature)
    assert all(torch.equal(got[n], again[n]) and got[n].data_ptr() != again[n].data_ptr() for n in got)


def test_a_teacher_and_its_student():
    """The lists go from one model to the other on the device.  A student with the teacher's weights is where it should be: with all that
    matters listed and the rest as one class, loss and gradient are what rounding leaves.  p and q are each within 2^-24 (240 + 8 |z|) of
    the softmax that both come from, so the gradient is within twice that of S / rows, half a step of fp16's smallest besides, and the
    loss, a mean of sum q (ln q - ln p), within that of 0."""
    wl = replace(HEAD, teacher_top=32, tail=True, temperature=2.0)
    teacher, student = St.XentStep(replace(HEAD)), St.XentStep(wl)
    batch = HEAD.batch()
    teacher.set_batch(batch)
    lists_ = teacher.score(wl.teacher_top, wl.temperature)
    student.set_batch(dict(batch, teacher_ids=lists_["ids"], teacher_logp=lists_["top_logp"]))
    student.forward_backward()
    z = np.abs(np32(teacher.rows16[:, :wl.vocab])).max()
    unit = 2.0 ** -24 * (240 + 8 * z)
    assert abs(float(student.loss)) <= 2 * unit
    assert np.abs(np32(student.logits)).max() <= student.state().scale / wl.tokens * 0.5 * 2 * unit + 2.0 ** -25
    # another head's lists do move it
    other = St.XentStep(HEAD, masters={"w": wl.masters()["w"][::-1].copy(), "b": wl.masters()["b"]})
    other.set_batch(batch)
    lists_ = other.score(wl.teacher_top, wl.temperature)
    student.set_batch(dict(batch, teacher_ids=lists_["ids"], teacher_logp=lists_["top_logp"]))
    student.step()
    assert float(student.loss) > 0.01 and not torch.equal(student.P.w32["w"], teacher.P.w32["w"])


def test_a_policys_gradient_through_the_head_and_the_turned_stack():
    """Scores, the gradient that a policy's loss takes from them, the head's products and the stack's backward pass: all gradients as close
    to 64 bits as the oracle's with fp16 storage are."""
    wl = replace(BASE, rope_axes=1, causal=True, n_docs=7, qk_norm=True)
    head_wl = replace(HEAD, tokens=wl.tokens, d_model=wl.d_model)
    stack, head = St.TransformerStep(wl), St.XentStep(head_wl)
    batch, r = batches(wl)(0), np.random.default_rng(5)
    targets = r.integers(-1, head_wl.vocab, wl.tokens).astype(np.int32)        # (-1: a token that is no answer's)
    dlogp, dentropy, scale, c = r.standard_normal(wl.tokens).astype(np.float32), r.standard_normal(wl.tokens).astype(np.float32), 64.0, 0.5
    stack.set_batch(batch)
    head.targets.copy_(i32(targets))
    head.h.copy_(stack.forward())
    got = head.score(0, 1 / c)
    st = mp.scale_state_alloc()
    mp.mp_scale_state_init(st, 0, scale, 1)
    T, V, g = wl.tokens, head_wl.vocab, head.P.g16
    mp.mp_token_logprobs_bwd(T, V, head.rows16, head.ld_v, head.targets, c, got["entropy"], got["lse"], f32(dlogp), f32(dentropy), st, head.rows16)
    mp.mp_gemm_bwd_both(head.desc, head.rows16, head.P.w16["w"], stack.gbuf[0], head.desc, head.h, g["w"], g["b"], st, head.ws)
    stack.backward()

    def chain(P, w, hw, b):
        keep, grads = {}, {}
        pairs = wl.d_head // 2
        angles = b["positions"].astype(np.float64)[np.arange(pairs) % 1].T * wl.rope_base ** (-np.arange(pairs) / pairs)
        x, caches = b["x"], []
        for l in range(wl.n_layers):
            x, cache = Mo.encoder_layer_fwd(P, w, f"l{l}.", x, wl.n_seq, wl.seq_len, wl.n_heads,
                                            L.attention_ranges(T, b["doc_start"], True), angles)
            caches.append(cache)
        logits = L.linear_fwd(P, x, hw["w"], hw["b"])
        d = L.token_logprobs_bwd(P, logits, targets, c, dlogp.astype(P.acc), dentropy.astype(P.acc), scale)
        dh, grads["w"], grads["b"] = L.linear_bwd(P, d, x, hw["w"])
        for l in range(wl.n_layers - 1, -1, -1):
            dh = Mo.encoder_layer_bwd(P, w, f"l{l}.", dh, caches[l], grads)
        return grads

    w, hw, ob = _snapshot(stack)["w16"], _snapshot(head)["w16"], Mo.island_batch(MIXED, batch)
    g_ref, g64 = chain(MIXED, w, hw, ob), chain(FP64, _f64(w), _f64(hw), _f64(ob))
    for n, t in {**stack.P.g16, **head.P.g16}.items():
        e_gpu, e_orc = rel_fro(np32(t), g64[n]), rel_fro(g_ref[n], g64[n])
        assert e_gpu <= 3.0 * e_orc + GRAD_TOL, (n, e_gpu, e_orc)


def test_on_streams_of_their_own():
    wl, hw, other = replace(BASE, rope_axes=1, causal=True, qk_norm=True), replace(HEAD, teacher_top=9), torch.cuda.Stream()
    a, b, c, d = St.TransformerStep(wl), St.TransformerStep(wl), St.XentStep(hw), St.XentStep(hw)
    torch.cuda.synchronize()
    for k in range(3):
        for s, t in ((a, c), (b, d)):
            with torch.cuda.stream(other if s is b else torch.cuda.default_stream()):
                s.set_batch(batches(wl)(k))
                s.step()
                t.set_batch(lists(hw)(k))
                t.step()
                t.scores = t.score(5)
    torch.cuda.synchronize()
    assert torch.equal(a.P.w32_arena, b.P.w32_arena) and torch.equal(c.P.w32_arena, d.P.w32_arena) and float(c.loss) == float(d.loss)
    assert all(torch.equal(c.scores[n], d.scores[n]) for n in c.scores)


def test_a_batch_that_does_not_fit():
    wl = replace(HEAD, teacher_top=3)
    step = St.XentStep(wl)
    step.set_batch(lists(wl)(0))
    kept = step.teacher_ids.clone()
    for bad in (dict(teacher_ids=np.zeros((wl.tokens, 4), np.int32)), dict(teacher_logp=np.zeros((wl.tokens - 1, 3), np.float32))):
        with pytest.raises(ValueError, match="lists"):
            step.set_batch(dict(lists(wl)(1), **bad))
    assert torch.equal(kept, step.teacher_ids)

"""Whole training iterations with the operators of language models together: tokens, their embedding, attention under a mask in every
layer, and AdamW with moments in 32 or 8 bits; against the oracle step by step, and captured."""
from dataclasses import replace

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import steps as St
import mp_inputs as I
from oracle import MIXED
from oracle import models as Mo
from oracle import optimizer as O
from gpu_util import *
from test_gpu_configs import teacher_forced, _graph_step

ADAMW = I.OptCfg(kind="adamw", lr=1e-3, weight_decay=0.1)
ADAMW8 = replace(ADAMW, state_bits=8)
BASE = replace(I.C2_SMALL, n_layers=2, opt=ADAMW, scale=I.ScaleCfg(init_scale=2.0 ** 12, growth_interval=3))   # 200 tokens, 3 heads of 64


def batches(wl, seed=0):
    """A batch of other tokens and documents for each step."""
    def at(k):
        r, out = np.random.default_rng([seed, k]), {}
        out["target"] = r.standard_normal((wl.tokens, wl.d_model)).astype(np.float32)
        if wl.vocab:
            out["tokens"] = r.integers(0, wl.vocab, wl.tokens).astype(np.int32)
        else:
            out["x"] = r.standard_normal((wl.tokens, wl.d_model)).astype(np.float32)
        if wl.n_docs:
            out["doc_start"] = np.concatenate([[0], np.sort(r.integers(0, wl.tokens + 1, wl.n_docs - 1)), [wl.tokens]]).astype(np.int32)
        return out
    return at


def oracle_of(wl):
    return Mo.make_transformer_fwd_bwd(wl.n_layers, wl.n_seq, wl.seq_len, wl.n_heads, wl.causal)


@pytest.mark.parametrize("kw", [dict(causal=True, n_docs=7, vocab=301), dict(causal=True), dict(n_docs=4, d_model=256, n_heads=8),
                                dict(vocab=50021, seq_len=1, n_seq=61), dict(causal=True, n_docs=3, vocab=11, d_model=128, n_heads=1)])
@pytest.mark.parametrize("opts", [dict(), dict(prechecked=True, flat_update=True, two_streams=True)])
def test_iterations_against_the_oracle(kw, opts):
    wl = replace(BASE, **kw)
    step = St.TransformerStep(wl, **opts)
    teacher_forced(step, wl, oracle_of(wl), None, 4, batch_fn=batches(wl), grad_mode="vs_fp64")


@pytest.mark.parametrize("flat", [False, True])
def test_iterations_with_moments_in_8_bits(flat):
    """The oracle's update of the GPU's own gradients and states: codes and scales bit by bit."""
    wl = replace(BASE, causal=True, n_docs=7, vocab=301, opt=ADAMW8)
    step, batch_fn = St.TransformerStep(wl, prechecked=flat, flat_update=flat), batches(wl)
    P = step.P
    for k in range(5):
        step.set_batch(batch_fn(k))
        before = {n: dict(w32=np32(P.w32[n]), w16=np32(P.w16[n]), **{c: getattr(P, c)[n].cpu().numpy().copy() for c in ("m8", "v8", "ms", "vs")})
                  for n in P.names}
        s0 = step.state()
        step.forward_backward()
        if k == 2:
            P.g16["emb"].view(-1)[7:8].fill_(float("inf"))
            step.st[7:8].fill_(1)                                        # as a gradient's producer does
        tensors = [dict(before[n], g16=np32(P.g16[n]), w32=before[n]["w32"].copy()) for n in P.names]
        for t in tensors:
            t["m8"], t["v8"] = t["m8"].reshape(-1), t["v8"].reshape(-1)
        found = O.unscale_check_update8(MIXED, tensors, wl.opt, O.ScaleState(scale=float(s0.scale), opt_step=s0.opt_step))
        step.optimizer()
        assert found == int(k == 2) == step.state().hist_found_inf[k]
        for n, t in zip(P.names, tensors):
            for c in ("m8", "v8", "ms", "vs"):
                assert np.array_equal(getattr(P, c)[n].cpu().numpy().reshape(-1), t[c]), (k, n, c)
            w0 = before[n]["w32"]
            # (a step of the update is off by an ulp or two, so 2^-22 of it and of the master's own rounding)
            assert np.all(np.abs(np32(P.w32[n]).astype(np.float64) - t["w32"]) <= 2.0 ** -22 * (np.abs(t["w32"]) + np.abs(t["w32"] - w0)))


@pytest.mark.parametrize("opt", [ADAMW, ADAMW8])
def test_captured_iterations_take_every_batch(opt):
    """Replays with other tokens and other documents, eager iterations of another step between them: the eager step's bits, over
    overflows that the scale starts with."""
    wl = replace(BASE, causal=True, n_docs=7, vocab=301, opt=opt, scale=I.ScaleCfg(init_scale=2.0 ** 24, growth_interval=3))
    eager, graphed = (St.TransformerStep(wl, prechecked=True, flat_update=True) for _ in range(2))
    batch_fn = batches(wl, 1)
    graphed.set_batch(batch_fn(0))
    eager.set_batch(batch_fn(0))
    graphed.step()
    eager.step()
    graph = _graph_step(graphed)
    for k in range(1, 14):
        for s in (eager, graphed):
            s.set_batch(batch_fn(k))
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        assert torch.equal(eager.P.w32_arena, graphed.P.w32_arena) and torch.equal(eager.P.w16_arena, graphed.P.w16_arena), k
        if opt.state_bits == 8:
            assert all(torch.equal(eager.P.state8[c], graphed.P.state8[c]) for c in ("m8", "v8", "ms", "vs")), k
    a, b = eager.state(), graphed.state()
    assert (a.scale, a.opt_step, a.skipped_steps) == (b.scale, b.opt_step, b.skipped_steps) and 0 < a.skipped_steps < 13


@pytest.mark.parametrize("make", [lambda o: St.XentStep(replace(I.C4_SMALL, tokens=64, vocab=301, opt=o)),
                                  lambda o: St.LSTMStep(replace(I.C5_SMALL, opt=o)), lambda o: St.MLPStep(replace(I.C1, opt=o))])
def test_moments_in_8_bits_in_the_other_steps(make):
    """The same gradients in, so after one iteration from zero states the masters of both kinds agree: the moments of a first step are
    (1-b) g and (1-b) g^2 before they are encoded, and the step is taken with them."""
    a, b = make(replace(ADAMW, state_bits=32)), make(ADAMW8)
    for s in (a, b):
        s.set_batch(s.wl.batch())
        s.step()
    assert a.state().opt_step == b.state().opt_step == 1
    for n in a.P.names:
        assert torch.equal(a.P.g16[n], b.P.g16[n])
        x, y = np32(a.P.w32[n]).astype(np.float64), np32(b.P.w32[n]).astype(np.float64)
        # two statements of one formula: m / bc1 and lr m / bc1, sqrt(v / bc2) and sqrt(v) / sqrt(bc2): each step is within 8 roundings
        # of 2^-24 (1e-8 beside the root included, a root of at least 2^-24 |g| not being less accurate) and an ulp of the master
        assert np.all(np.abs(x - y) <= 2.0 ** -23 * np.abs(x) + 2.0 ** -20 * ADAMW.lr), n


def test_iterations_on_a_stream_of_their_own():
    wl, other = replace(BASE, causal=True, n_docs=7, vocab=301, opt=ADAMW8), torch.cuda.Stream()
    a, b = St.TransformerStep(wl), St.TransformerStep(wl)
    torch.cuda.synchronize()
    for k in range(3):
        a.set_batch(batches(wl)(k))
        a.step()
        with torch.cuda.stream(other):
            b.set_batch(batches(wl)(k))
            b.step()
    torch.cuda.synchronize()
    assert torch.equal(a.P.w32_arena, b.P.w32_arena) and float(a.loss) == float(b.loss)


def test_document_starts_that_do_not_fit():
    wl = replace(BASE, n_docs=4)
    step = St.TransformerStep(wl)
    with pytest.raises(ValueError, match="document starts"):
        step.set_batch(dict(wl.batch(), doc_start=np.array([0, wl.tokens], np.int32)))

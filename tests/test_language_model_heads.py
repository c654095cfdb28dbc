"""Turned heads and teachers' lists in the workloads: the oracle's gradients against differences, shapes, and what a step refuses before
anything is on a device (no GPU)."""
from dataclasses import replace
from types import SimpleNamespace

import numpy as np
import pytest

import mp_inputs as I
from oracle import FP64
from oracle import models as Mo
from paper_1805_10387_amd import steps as St

WL = replace(I.C2_SMALL, n_layers=2, d_model=16, n_heads=2, d_ff=24, seq_len=6, n_seq=3)
HEAD = replace(I.C4_SMALL, tokens=7, d_model=6, vocab=11)


@pytest.mark.parametrize("kw", [dict(rope_axes=1, causal=True, qk_norm=True), dict(rope_axes=2), dict(rope_axes=3, n_docs=4, qk_norm=True, vocab=9)])
def test_turned_heads_against_differences(kw):
    """Central differences of a step h in 64 bits: off by h^2 f''' / 6 and by 2^-52 L / h, both below 1e-8 of the gradients here."""
    wl = replace(WL, **kw)
    w = dict(wl.embedding(), **Mo.flatten_layers(wl.masters()))
    r = np.random.default_rng(0)
    w = {k: np.asarray(v, np.float64) + 0.1 * r.standard_normal(v.shape) for k, v in w.items()}
    f, batch = Mo.make_transformer_fwd_bwd(wl.n_layers, wl.n_seq, wl.seq_len, wl.n_heads, wl.causal, wl.rope_base), Mo.island_batch(FP64, wl.batch())
    _, g = f(FP64, w, batch, 1.0)
    assert set(g) == set(w) and all(g[k].shape == w[k].shape for k in w)
    for k in ["l0.wqkv", "l1.bqkv", "l0.wo"] + ["l0.qn_g", "l1.kn_g"] * wl.qk_norm:
        way, h = r.standard_normal(w[k].shape), 1e-5
        loss = [f(FP64, dict(w, **{k: w[k] + s * h * way}), batch, 1.0)[0] for s in (1, -1)]
        assert abs((loss[0] - loss[1]) / (2 * h) - float((g[k] * way).sum())) <= 1e-6 * np.sqrt((g[k] ** 2).sum()), k


def test_only_differences_of_positions_count():
    """On each axis: all tokens moved by the same amount see each other as before."""
    wl = replace(WL, rope_axes=2, n_docs=3, qk_norm=True)
    w = {k: np.asarray(v, np.float64) for k, v in Mo.flatten_layers(wl.masters()).items()}
    f, batch = Mo.make_transformer_fwd_bwd(wl.n_layers, wl.n_seq, wl.seq_len, wl.n_heads), Mo.island_batch(FP64, wl.batch())
    moved = dict(batch, positions=batch["positions"] + np.array([[5], [1000]]))
    a, b = f(FP64, w, batch, 1.0), f(FP64, w, moved, 1.0)
    assert abs(a[0] - b[0]) <= 1e-10 * a[0] and all(np.allclose(a[1][k], b[1][k], rtol=0, atol=1e-9 * np.abs(a[1][k]).max()) for k in w)
    turned = f(FP64, w, dict(batch, positions=batch["positions"][::-1].copy()), 1.0)
    assert abs(turned[0] - a[0]) > 1e-6 * a[0]


@pytest.mark.parametrize("kw", [dict(teacher_top=3), dict(teacher_top=4, temperature=2.0, soft_weight=4.0, hard_weight=0.5, tail=True)])
def test_a_students_gradient_against_differences(kw):
    wl = replace(HEAD, **kw)
    w = {k: np.asarray(v, np.float64) for k, v in wl.masters().items()}
    f, batch = Mo.make_distill_head_fwd_bwd(wl.temperature, wl.soft_weight, wl.hard_weight, wl.tail), Mo.island_batch(FP64, wl.batch())
    assert batch["teacher_logp"].dtype == np.float32
    _, g = f(FP64, w, batch, 1.0)
    r, h = np.random.default_rng(0), 1e-5
    for k in w:
        way = r.standard_normal(w[k].shape)
        loss = [f(FP64, dict(w, **{k: w[k] + s * h * way}), batch, 1.0)[0] for s in (1, -1)]
        assert abs((loss[0] - loss[1]) / (2 * h) - float((g[k] * way).sum())) <= 1e-6 * np.sqrt((g[k] ** 2).sum()), k


def test_workload_shapes():
    wl = replace(WL, rope_axes=3, n_docs=4, qk_norm=True)
    b = wl.batch()
    assert b["positions"].shape == (3, wl.tokens) and b["positions"].dtype == np.int32
    assert wl.n_params() == WL.n_params() + 2 * 2 * wl.d_head and wl.masters()[0]["qn_g"].shape == (wl.d_head,)
    starts = b["doc_start"][:-1][np.diff(b["doc_start"]) > 0]
    assert not b["positions"][:, starts].any()
    plain = replace(WL, rope_axes=1)
    assert np.array_equal(plain.batch()["positions"], np.tile(np.arange(6), 3)[None]) and "positions" not in WL.batch()
    assert set(WL.masters()[0]) == set(plain.masters()[0]) == set(wl.masters()[0]) - {"qn_g", "kn_g"}
    b = replace(HEAD, teacher_top=3).batch()
    assert b["teacher_ids"].shape == b["teacher_logp"].shape == (7, 3) and np.exp(b["teacher_logp"]).sum(1).max() < 1
    assert all(len(set(row)) == 3 for row in b["teacher_ids"].tolist()) and set(HEAD.batch()) == {"h", "targets"}


def test_what_a_stack_with_turned_heads_refuses(monkeypatch):
    def store(masters, adam, state_bits=32):
        raise KeyError("store")
    monkeypatch.setattr(St, "ParamStore", store)
    with pytest.raises(ValueError, match="rope_axes is 0"):
        St.TransformerStep(replace(I.C2_SMALL, qk_norm=True), masters={})
    with pytest.raises(ValueError, match="5 axes"):
        St.TransformerStep(replace(I.C2_SMALL, rope_axes=5), masters={})
    with pytest.raises(ValueError, match="head size 20"):
        St.TransformerStep(replace(I.C2_SMALL, d_model=160, n_heads=8, rope_axes=1), masters={})
    with pytest.raises(KeyError):
        St.TransformerStep(replace(I.C2_SMALL, rope_axes=3, qk_norm=True), masters={})


def test_a_workload_of_the_callers_own_without_the_new_fields(monkeypatch):
    def store(masters, adam, state_bits=32):
        raise KeyError("store")
    monkeypatch.setattr(St, "ParamStore", store)
    old = {k: v for k, v in vars(I.C2_SMALL).items() if k not in ("rope_axes", "rope_base", "qk_norm")}
    wl = SimpleNamespace(tokens=I.C2_SMALL.tokens, **dict(old, causal=True))
    with pytest.raises(KeyError):
        St.TransformerStep(wl, masters={"w": np.zeros(4, np.float32)})


def test_positions_that_do_not_fit_replace_nothing():
    step = St.TransformerStep.__new__(St.TransformerStep)
    step.wl = replace(I.C2_SMALL, rope_axes=2)                  # (nothing else is there: whatever set_batch did would fail)
    batch = step.wl.batch()
    for bad in (batch["positions"][:1], batch["positions"][:, 1:], batch["positions"].T, np.zeros(step.wl.tokens, np.int32)):
        with pytest.raises(ValueError, match="2 axes of 200 tokens"):
            step.set_batch(dict(batch, positions=bad))


def test_norms_without_their_weights_are_not_left_out():
    """Masters of the caller's own that do not have them: the forward pass says so."""
    step = St.TransformerStep.__new__(St.TransformerStep)
    step.wl, step.rope_axes, step.qk_norm, step.masked = replace(I.C2_SMALL, rope_axes=1, qk_norm=True), 1, True, True
    step.P = SimpleNamespace(w16={"l0.wqkv": None, "l0.bqkv": None})
    step.x0, step.act, step.trace = None, [dict(qkv=np.zeros((1, 1)), qk=np.zeros((1, 1)))], None
    step.d_qkv = step.d_rope = step.positions = step.freqs = None
    calls = []
    kept, St.B.mp_gemm_fwd = St.B.mp_gemm_fwd, lambda *a: calls.append(a)
    try:
        with pytest.raises(KeyError, match="l0.qn_g"):
            step.forward()
    finally:
        St.B.mp_gemm_fwd = kept
    assert len(calls) == 1

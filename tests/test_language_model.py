"""A stack on tokens with attention under a mask: the oracle's gradients against differences, and the workload's shapes."""
from dataclasses import replace

import numpy as np
import pytest

import mp_inputs as I
from oracle import FP64
from oracle import models as Mo

WL = replace(I.C2_SMALL, n_layers=2, d_model=16, n_heads=2, d_ff=24, seq_len=6, n_seq=3)


@pytest.mark.parametrize("kw", [dict(causal=True), dict(n_docs=4), dict(causal=True, n_docs=5, vocab=9), dict(vocab=7)])
def test_gradients_against_differences(kw):
    """Central differences of a step h in 64 bits: off by h^2 f''' / 6 and by 2^-52 L / h, both below 1e-8 of the gradients here."""
    wl = replace(WL, **kw)
    w = dict(wl.embedding(), **Mo.flatten_layers(wl.masters()))
    w, batch = {k: np.asarray(v, np.float64) for k, v in w.items()}, wl.batch()
    f = Mo.make_transformer_fwd_bwd(wl.n_layers, wl.n_seq, wl.seq_len, wl.n_heads, wl.causal)
    _, g = f(FP64, w, Mo.island_batch(FP64, batch), 1.0)
    assert set(g) == set(w) and all(g[k].shape == w[k].shape for k in w)
    r, h = np.random.default_rng(0), 1e-5
    for k in (["emb"] if wl.vocab else []) + ["l0.wqkv", "l1.wqkv", "l0.wo", "l1.bqkv"]:
        way = r.standard_normal(w[k].shape)
        loss = [f(FP64, dict(w, **{k: w[k] + s * h * way}), Mo.island_batch(FP64, batch), 1.0)[0] for s in (1, -1)]
        want = float((g[k] * way).sum())
        assert abs((loss[0] - loss[1]) / (2 * h) - want) <= 1e-6 * np.sqrt((g[k] ** 2).sum()), k


def test_packed_documents_do_not_see_each_other():
    wl = replace(WL, causal=True, n_docs=3, vocab=9)
    w = dict(wl.embedding(), **Mo.flatten_layers(wl.masters()))
    batch, f = wl.batch(), Mo.make_transformer_fwd_bwd(wl.n_layers, wl.n_seq, wl.seq_len, wl.n_heads, True)
    batch["doc_start"] = np.array([0, 5, 5, 18], np.int32)
    keeps = [{}, {}]
    for j, keep in enumerate(keeps):
        b = dict(batch, tokens=batch["tokens"].copy())
        b["tokens"][12] = (b["tokens"][12] + j) % wl.vocab       # row 12 of the last document: rows 12 to 17 only may change
        f(FP64, {k: np.asarray(v, np.float64) for k, v in w.items()}, Mo.island_batch(FP64, b), 1.0, keep)
    same = np.all(keeps[0]["y"] == keeps[1]["y"], axis=1)
    assert same[:12].all() and not same[12:].any()


def test_workload_shapes():
    wl = replace(WL, n_docs=4, vocab=9)
    b = wl.batch()
    assert b["tokens"].dtype == np.int32 and b["tokens"].shape == (wl.tokens,) and b["tokens"].max() < 9 and "x" not in b
    assert b["doc_start"].shape == (5,) and b["doc_start"][0] == 0 and b["doc_start"][-1] == wl.tokens and np.all(np.diff(b["doc_start"]) >= 0)
    assert wl.n_params() == WL.n_params() + 9 * 16 and set(WL.batch()) == {"x", "target"} and WL.embedding() == {}


@pytest.mark.parametrize("adam,bits", [(False, 8), (True, 16)])
def test_moments_that_there_are_not(adam, bits):
    from paper_1805_10387_amd import steps as St
    with pytest.raises(ValueError, match="moments"):
        St.ParamStore({"w": np.zeros(4, np.float32)}, adam=adam, state_bits=bits)

"""What the step classes make of their arguments before anything is on a device (no GPU)."""
from dataclasses import replace
from types import SimpleNamespace

import numpy as np
import pytest

import mp_inputs as I
from paper_1805_10387_amd import steps as St


class Stop(Exception):
    pass


def made(monkeypatch, opt):
    """(adam, state_bits) that a step with this optimizer asks its parameters' store for."""
    def store(masters, adam, state_bits=32):
        raise Stop(adam, state_bits)
    monkeypatch.setattr(St, "ParamStore", store)
    with pytest.raises(Stop) as e:
        St._StepBase({}, opt, I.ScaleCfg())
    return e.value.args


def test_an_optimizer_that_knows_no_state_bits(monkeypatch):
    """An object of the caller's own with the fields that there were before moments in 8 bits."""
    for kind, adam in (("sgd", False), ("adam", True), ("adamw", True)):
        opt = SimpleNamespace(kind=kind, lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0)
        assert made(monkeypatch, opt) == (adam, 32)
    assert made(monkeypatch, I.OptCfg(kind="adamw", state_bits=8)) == (True, 8)


@pytest.mark.parametrize("kw,says", [(dict(d_model=160, n_heads=8), "head size 20"), (dict(d_model=288, n_heads=2), "head size 144")])
@pytest.mark.parametrize("mask", [dict(causal=True), dict(n_docs=3)])
def test_a_head_size_without_a_kernel_is_refused_when_the_step_is_made(monkeypatch, kw, says, mask):
    """Not at its first iteration; without a mask the unfused chain takes any head size."""
    def store(masters, adam, state_bits=32):
        raise Stop()
    monkeypatch.setattr(St, "ParamStore", store)
    wl = replace(I.C2_SMALL, **kw)
    with pytest.raises(ValueError, match=says):
        St.TransformerStep(replace(wl, **mask), masters={})
    for ok in (wl, replace(I.C2_SMALL, **mask)):
        with pytest.raises(Stop):
            St.TransformerStep(ok, masters={})


def test_a_batch_that_does_not_fit_replaces_nothing():
    step = St.TransformerStep.__new__(St.TransformerStep)
    step.wl = replace(I.C2_SMALL, n_docs=4, vocab=11)          # (nothing else is there: whatever set_batch did would fail)
    batch = step.wl.batch()
    for starts in (np.array([0, 9], np.int32), np.zeros((5, 1), np.int32), [0, 1, 2, 3]):
        with pytest.raises(ValueError, match="document starts for 4"):
            step.set_batch(dict(batch, doc_start=starts))

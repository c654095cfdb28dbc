"""What a student's step makes of a batch before an iteration (no GPU: its buffers are on the host here)."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import mp_inputs as I
from paper_1805_10387_amd import steps as St

WL = replace(I.C4_SMALL, tokens=7, d_model=6, vocab=11, teacher_top=3)


@pytest.fixture
def step(monkeypatch):
    monkeypatch.setattr(St, "_h16", lambda x: torch.from_numpy(np.asarray(x, np.float32)).half())
    monkeypatch.setattr(St, "_i32", lambda x: torch.from_numpy(np.asarray(x).astype(np.int32)))
    s = St.XentStep.__new__(St.XentStep)
    s.wl = WL
    s.h, s.targets = torch.zeros(7, 6, dtype=torch.float16), torch.zeros(7, dtype=torch.int32)
    s.teacher_ids, s.teacher_logp = torch.zeros(7, 3, dtype=torch.int32), torch.zeros(7, 3)
    return s


def test_a_batch_is_taken(step):
    batch = WL.batch()
    step.set_batch(batch)
    assert np.array_equal(step.teacher_ids.numpy(), batch["teacher_ids"]) and np.array_equal(step.teacher_logp.numpy(), batch["teacher_logp"])
    assert np.array_equal(step.targets.numpy(), batch["targets"]) and np.array_equal(step.h.numpy(), batch["h"].astype(np.float16))


@pytest.mark.parametrize("bad", [dict(h=np.zeros((6, 6))), dict(h=np.zeros((7, 5))), dict(targets=np.zeros(6, np.int32)), dict(teacher_ids=np.zeros((7, 4), np.int32)),
                                 dict(teacher_logp=np.zeros((6, 3), np.float32)), dict(targets=None)])
def test_a_batch_that_does_not_fit_replaces_nothing(step, bad):
    """Whichever part it is: hidden states, targets and lists of two batches are never together."""
    step.set_batch(WL.batch())
    kept = [t.clone() for t in (step.h, step.targets, step.teacher_ids, step.teacher_logp)]
    batch = dict(WL.batch(), h=np.ones((7, 6)), targets=np.arange(7), teacher_ids=np.full((7, 3), 5, np.int32), teacher_logp=np.full((7, 3), -2, np.float32))
    with pytest.raises((ValueError, RuntimeError, KeyError)):
        step.set_batch({k: v for k, v in dict(batch, **bad).items() if v is not None})
    assert all(torch.equal(a, b) for a, b in zip(kept, (step.h, step.targets, step.teacher_ids, step.teacher_logp)))


def test_classes_of_lists_in_64_bits_keep_what_they_say(step):
    """What is no class stays none: cut to 32 bits 2^32 + 3 would be class 3, and the least of all class 0."""
    ids = np.array([[3, -1, 10], [2 ** 32 + 3, 2 ** 31, 2 ** 32], [-2 ** 63, 2 ** 63 - 1, -2 ** 32], [-2 ** 32 + 5, 2 ** 33 + 9, 0], [11, -100, 4], [-2 ** 31, 2 ** 31 - 1, 1],
                    [7, 8, 9]], np.int64)
    for given in (ids, torch.from_numpy(ids), torch.from_numpy(ids).t().contiguous().t()):
        step.teacher_ids.fill_(6)
        step.set_batch(dict(WL.batch(), teacher_ids=given))
        got, there = step.teacher_ids.numpy(), (ids >= 0) & (ids < WL.vocab)
        assert np.array_equal(got[there], ids[there]) and not ((got[~there] >= 0) & (got[~there] < WL.vocab)).any()

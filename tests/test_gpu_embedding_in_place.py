"""The embedding gradient added to a gradient in place: what the flag covers, and what stays as it is."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import _lib as ML
from oracle import MIXED
from oracle.numerics import half_bits
from gpu_util import *
from test_gpu_embedding import place

S16 = MIXED.store


@pytest.mark.parametrize("skew", [0, 1, 3, 8])
@pytest.mark.parametrize("rows", [0, 2, 300])
@pytest.mark.parametrize("bad", [None, 0, 6, 5000, 700 * 19 - 1])
def test_infinities_where_there_is_no_token_are_reported(rows, skew, bad):
    """As with a buffer of its own: the first and last elements, words and halves, at any alignment."""
    vocab, d = 700, 19
    second = S16(np.random.default_rng(skew).standard_normal((vocab, d)))
    if bad is not None:
        second.reshape(-1)[bad] = np.inf
    absent = np.where(np.arange(rows) % 2 == 0, -1, vocab)
    tokens, dy = i32(absent if rows else np.zeros(1)), place(np.ones((max(rows, 1), d)), 0)
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(rows, vocab, d), dtype=torch.uint8, device="cuda")
    for in_place in (False, True):
        st = mp.scale_state_alloc()
        mp.mp_scale_state_init(st, ML.MP_SCALE_BACKOFF, 1.0, 3)
        add = place(second, skew)
        dw = add if in_place else place(np.full((vocab, d), 7.0), skew)
        mp.mp_embedding_bwd(rows, vocab, d, tokens, dy, 1.0, dw, add=add, st=st, ws=ws)
        assert mp.scale_state_read(st).found_inf == int(bad is not None), in_place
        assert np.array_equal(bits(dw), half_bits(second))
        mp.mp_embedding_bwd(rows, vocab, d, tokens, dy, 1.0, dw, add=add, ws=ws)        # (without a state there is nothing to tell)
        assert np.array_equal(bits(dw), half_bits(second))


def test_in_place_is_the_same_with_and_without_a_state():
    vocab, d, rows = 300, 40, 5000
    r = np.random.default_rng(1)
    tokens, dy, second = i32(r.integers(0, vocab // 2, rows)), h16(S16(r.standard_normal((rows, d)))), S16(r.standard_normal((vocab, d)))
    ws = torch.empty(mp.mp_embedding_bwd_workspace_bytes(rows, vocab, d), dtype=torch.uint8, device="cuda")
    st = mp.scale_state_alloc()
    mp.mp_scale_state_init(st, ML.MP_SCALE_BACKOFF, 1.0, 3)
    a, b = h16(second), h16(second)
    mp.mp_embedding_bwd(rows, vocab, d, tokens, dy, 0.5, a, add=a, ws=ws)
    mp.mp_embedding_bwd(rows, vocab, d, tokens, dy, 0.5, b, add=b, st=st, ws=ws)
    assert torch.equal(a, b) and mp.scale_state_read(st).found_inf == 0 and np.array_equal(bits(a[vocab // 2:]), half_bits(second[vocab // 2:]))

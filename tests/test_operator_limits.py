"""Sizes whose launch would count more than 2^32 work items are refused on the host, with the reason (no GPU)."""
import ctypes as C

import pytest

from paper_1805_10387_amd import _lib as ML
from test_operator_refusals import A, bwd, desc, fwd

lib = ML.load()


@pytest.mark.parametrize("rows,d", [(2 ** 31 - 1, 17), (2 ** 31 - 1, 24), (2 ** 30, 32), (2 ** 29, 64)])
def test_embedding(rows, d):
    assert lib.mp_embedding_fwd(rows, 5, d, A, A, 1.0, A, None) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()


def test_embedding_gradient():
    assert lib.mp_embedding_bwd(1 << 24, 5, 1 << 28, A, A, 1.0, None, A, None, A, (1 << 64) - 1, None) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()


@pytest.mark.parametrize("kw", [dict(rows_q=2 ** 30, n_heads=2, n_kv_heads=1), dict(rows_k=2 ** 30, n_heads=2, n_kv_heads=1),
                                dict(rows_q=2 ** 27, n_heads=16, n_kv_heads=16), dict(rows_k=2 ** 27, n_heads=16, n_kv_heads=1)])
def test_attention(kw):
    d = desc(d_head=8, **dict(dict(ld_q=128, ld_k=128, ld_v=128, ld_ctx=128, ld_dq=128, ld_dk=128, ld_dv=128, ld_dctx=128), **kw))
    assert fwd(d) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()
    assert bwd(d) == ML.MP_E_INVAL and lib.mp_attention_masked_bwd_workspace_bytes(C.byref(d)) == 0


def test_decoding():
    assert lib.mp_state8_decode(2 ** 34 - 1023, A, A, None, None, A, None, None) == ML.MP_E_INVAL and b"large" in lib.mp_last_error()

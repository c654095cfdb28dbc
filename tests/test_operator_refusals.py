"""Refusals of masked attention, embedding and the 8-bit update: found on the host, before anything is enqueued (no GPU)."""
import ctypes as C
import os
import sys

import pytest

from paper_1805_10387_amd import _lib as ML

A = 256          # an aligned address that is never read
lib = ML.load()


def desc(**kw):
    v = dict(rows_q=10, rows_k=12, n_heads=4, n_kv_heads=2, d_head=64, ld_q=256, ld_k=128, ld_v=128, ld_ctx=256, ld_dq=256, ld_dk=128, ld_dv=128,
             ld_dctx=256, alpha=0.125, cap=0.0, reserved=0)
    v.update(kw)
    return ML.AttnDesc(*[v[n] for n, _ in ML.AttnDesc._fields_])


def fwd(d, mask=A, q=A, k=A, v=A, ctx=A, lse=A):
    return lib.mp_attention_masked_fwd(C.byref(d), mask, q, k, v, None, ctx, lse, None)


def bwd(d, mask=A, q=A, k=A, v=A, ctx=A, lse=A, do=A, dq=A, dk=A, dv=A, ws=A, n=1 << 30):
    return lib.mp_attention_masked_bwd(C.byref(d), mask, q, k, v, None, ctx, lse, do, dq, dk, dv, ws, n, None)


@pytest.mark.parametrize("kw", [dict(rows_q=-1), dict(rows_k=-1), dict(n_heads=0), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(d_head=0), dict(alpha=0.0),
                                dict(alpha=-1.0), dict(alpha=float("nan")), dict(alpha=float("inf")), dict(cap=-1.0), dict(cap=float("nan")),
                                dict(reserved=1), dict(ld_q=248), dict(ld_k=120), dict(ld_v=120), dict(ld_ctx=248), dict(n_heads=1 << 20)])
def test_attention_descriptions_that_make_no_sense(kw):
    assert fwd(desc(**kw)) == ML.MP_E_INVAL and bwd(desc(**kw)) == ML.MP_E_INVAL
    assert lib.mp_attention_masked_bwd_workspace_bytes(C.byref(desc(**kw))) == 0


@pytest.mark.parametrize("kw", [dict(d_head=60), dict(d_head=132, ld_q=1024, ld_ctx=1024, ld_k=512, ld_v=512), dict(ld_q=260), dict(ld_k=132), dict(ld_ctx=257)])
def test_attention_layouts_without_a_kernel(kw):
    assert fwd(desc(**kw)) == ML.MP_E_UNSUPPORTED and bwd(desc(**kw)) == ML.MP_E_UNSUPPORTED


def test_attention_pointers():
    for k in ("mask", "q", "k", "v", "ctx", "lse"):
        assert fwd(desc(), **{k: None}) == ML.MP_E_INVAL and b"NULL" in lib.mp_last_error()
    for k in ("mask", "q", "k", "v", "ctx", "lse", "do", "dq", "dk", "dv"):
        assert bwd(desc(), **{k: None}) == ML.MP_E_INVAL
    for k in ("mask", "q", "k", "v", "ctx"):
        assert fwd(desc(), **{k: A + 8}) == ML.MP_E_UNSUPPORTED and b"aligned" in lib.mp_last_error()
    for k in ("do", "dq", "dk", "dv"):
        assert bwd(desc(), **{k: A + 2}) == ML.MP_E_UNSUPPORTED
    for kw in (dict(ld_dq=248), dict(ld_dk=120), dict(ld_dv=64), dict(ld_dctx=0)):
        assert bwd(desc(**kw)) == ML.MP_E_INVAL
    assert bwd(desc(ld_dv=132)) == ML.MP_E_UNSUPPORTED
    need = lib.mp_attention_masked_bwd_workspace_bytes(C.byref(desc()))
    assert need >= 2 * 4 * 64 * 4
    assert bwd(desc(), ws=None) == bwd(desc(), ws=A + 4) == bwd(desc(), n=need - 1) == ML.MP_E_WORKSPACE
    # nothing to do: no pointer is looked at
    assert fwd(desc(rows_q=0), None, None, None, None, None, None) == ML.MP_OK
    assert bwd(desc(rows_q=0, rows_k=0), None, None, None, None, None, None, None, None, None, None) == ML.MP_OK


def test_masks():
    f = lib.mp_attention_mask_docs
    assert f(-1, 1, A, None, 0, 0, A, None) == f(4, -1, A, None, 0, 0, A, None) == f(4, 1, A, None, 0, -1, A, None) == ML.MP_E_INVAL
    assert f(4, 1, None, None, 0, 0, A, None) == f(4, 1, A, None, 0, 0, None, None) == f(4, 1, A, None, 0, 0, A + 8, None) == ML.MP_E_INVAL
    assert f(4, 1, A, A, 0, 0, A, None) == f(4, 1, A, A, 1, 3, A, None) == ML.MP_E_INVAL and b"prefix" in lib.mp_last_error()
    assert f(0, 0, None, None, 0, 0, A, None) == ML.MP_OK
    g = lib.mp_attention_mask_ranges
    assert g(-1, 4, A, A, A, None) == g(4, -1, A, A, A, None) == g(4, 4, None, A, A, None) == g(4, 4, A, None, A, None) == g(4, 4, A, A, None, None) == ML.MP_E_INVAL
    assert lib.mp_attention_mask_bytes(-1) == 0 and lib.mp_attention_mask_bytes(1) >= 64 * 8 + 16 and lib.mp_attention_mask_bytes(65) >= 128 * 8 + 32


def test_embedding():
    f, b = lib.mp_embedding_fwd, lib.mp_embedding_bwd
    assert f(-1, 5, 8, A, A, 1.0, A, None) == f(4, 0, 8, A, A, 1.0, A, None) == f(4, 5, 0, A, A, 1.0, A, None) == ML.MP_E_INVAL
    assert f(4, 5, 8, None, A, 1.0, A, None) == f(4, 5, 8, A, None, 1.0, A, None) == f(4, 5, 8, A, A, 1.0, None, None) == ML.MP_E_INVAL
    assert f(0, 5, 8, None, None, 1.0, None, None) == ML.MP_OK
    n = 1 << 40
    assert b(-1, 5, 8, A, A, 1.0, None, A, None, A, n, None) == b(4, 5, 8, None, A, 1.0, None, A, None, A, n, None) == ML.MP_E_INVAL
    assert b(4, 5, 8, A, None, 1.0, None, A, None, A, n, None) == b(4, 5, 8, A, A, 1.0, None, None, None, A, n, None) == ML.MP_E_INVAL
    assert b((1 << 24) + 1, 5, 8, A, A, 1.0, None, A, None, A, n, None) == b(4, 1 << 21, 8, A, A, 1.0, None, A, None, A, n, None) == ML.MP_E_UNSUPPORTED
    need = lib.mp_embedding_bwd_workspace_bytes(4, 5, 8)
    assert b(4, 5, 8, A, A, 1.0, None, A, None, None, n, None) == b(4, 5, 8, A, A, 1.0, None, A, None, A + 8, n, None) == ML.MP_E_WORKSPACE
    assert b(4, 5, 8, A, A, 1.0, None, A, None, A, need - 1, None) == ML.MP_E_WORKSPACE
    assert lib.mp_embedding_bwd_workspace_bytes(-1, 5, 8) == lib.mp_embedding_bwd_workspace_bytes(4, 0, 8) == 0


def test_update8():
    cfg = ML.OptCfg()
    t = (ML.TensorDesc8 * 1)()
    for k, _ in ML.TensorDesc8._fields_:
        setattr(t[0], k, 256)
    call = lambda: lib.mp_unscale_check_update8(t, 1, C.byref(cfg), A, 0, None)  # noqa: E731
    for kind in (ML.MP_OPT_SGD, 3, -1):
        cfg.kind = kind
        assert call() == ML.MP_E_INVAL and b"kind" in lib.mp_last_error()
    cfg.kind = ML.MP_OPT_ADAMW
    assert lib.mp_unscale_check_update8(t, 1, None, A, 0, None) == lib.mp_unscale_check_update8(t, 1, C.byref(cfg), None, 0, None) == ML.MP_E_INVAL
    assert lib.mp_unscale_check_update8(None, 1, C.byref(cfg), A, 0, None) == lib.mp_unscale_check_update8(t, -1, C.byref(cfg), A, 0, None) == ML.MP_E_INVAL
    assert lib.mp_unscale_check_update8(t, 1, C.byref(cfg), A, 2, None) == ML.MP_E_INVAL
    for k in ("g16", "w32", "w16", "m8", "v8", "ms", "vs"):
        setattr(t[0], k, None)
        assert call() == ML.MP_E_INVAL, k
        setattr(t[0], k, 256)
    for k, bad in (("g16", 257), ("w16", 257), ("w32", 258), ("ms", 258), ("vs", 257)):
        setattr(t[0], k, bad)
        assert call() == ML.MP_E_INVAL, k
        setattr(t[0], k, 256)
    e = lib.mp_unscale_check_update8_end
    assert e(t, 1, C.byref(cfg), A, 0, None, None, None, None) == e(t, 1, C.byref(cfg), A, 0, None, None, 258, None) == ML.MP_E_INVAL
    d = lib.mp_state8_decode
    assert d(4, None, A, None, None, A, None, None) == d(4, A, None, None, None, A, None, None) == d(4, None, None, A, None, None, A, None) == ML.MP_E_INVAL
    assert d(4, A, A, None, None, 258, None, None) == d(1 << 40, A, A, None, None, A, None, None) == ML.MP_E_INVAL
    assert d(4, None, None, None, None, None, None, None) == d(0, A, A, A, A, A, A, None) == ML.MP_OK


def test_structs_match_the_header():
    assert C.sizeof(ML.AttnDesc) == 64 and ML.AttnDesc.alpha.offset == 52 and C.sizeof(ML.TensorDesc8) == 64
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mp.h")).read()
    assert f"#define MP_STATE8_BLOCK {ML.MP_STATE8_BLOCK}\n" in hdr


def test_embedding_and_cap_at_their_ends():
    f, b = lib.mp_embedding_fwd, lib.mp_embedding_bwd
    assert f(4, 5, 8, A, A + 1, 1.0, A, None) == f(4, 5, 8, A, A, 1.0, A + 3, None) == ML.MP_E_INVAL
    assert b(4, 5, 8, A, A + 1, 1.0, None, A, None, A, 1 << 40, None) == b(4, 5, 8, A, A, 1.0, A + 1, A, None, A, 1 << 40, None) == ML.MP_E_INVAL
    for kw in (dict(cap=1025.0), dict(cap=1e-38, alpha=1.0), dict(cap=float("inf"))):
        d = desc(**kw)
        assert lib.mp_attention_masked_fwd(C.byref(d), A, A, A, A, None, A, A, None) in (ML.MP_E_UNSUPPORTED, ML.MP_E_INVAL)
        assert lib.mp_attention_masked_bwd_workspace_bytes(C.byref(d)) == 0

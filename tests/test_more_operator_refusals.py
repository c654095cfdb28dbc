"""Refusals of head norms with rotation, token log probabilities and distillation: found on the host, before anything is enqueued (no GPU)."""
import ctypes as C
import re

import pytest

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import _lib as ML

A = 256          # an aligned address that is never read
lib = ML.load()
BIG = 1 << 40


def rope(**kw):
    d = mp.rope_desc(10, 4, 2, 64)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def rope_fwd(d, q=A, k=A, gq=A, gk=A, pos=A, freqs=A, yq=A, yk=A):
    return lib.mp_qk_norm_rope_fwd(C.byref(d), q, k, gq, gk, pos, freqs, yq, yk, None)


def rope_bwd(d, q=A, k=A, gq=A, gk=A, pos=A, freqs=A, dyq=A, dyk=A, dq=A, dk=A, dgq=A, dgk=A, ws=A, n=BIG):
    return lib.mp_qk_norm_rope_bwd(C.byref(d), q, k, gq, gk, pos, freqs, dyq, dyk, dq, dk, dgq, dgk, None, ws, n, None)


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(n_heads=0), dict(n_kv_heads=0), dict(d_head=0), dict(rot=0), dict(rot=-4), dict(rot=66), dict(rot=7), dict(n_axes=0),
                                dict(n_axes=5), dict(adjacent=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(reserved=1), dict(ld_q=248),
                                dict(ld_k=120)])
def test_rotations_that_make_no_sense(kw):
    assert rope_fwd(rope(**kw)) == rope_bwd(rope(**kw)) == ML.MP_E_INVAL
    if not set(kw) & {"ld_q", "ld_k"}:
        assert lib.mp_qk_norm_rope_bwd_workspace_bytes(C.byref(rope(**kw))) == 0


@pytest.mark.parametrize("kw", [dict(d_head=60, rot=60), dict(d_head=264, ld_q=1056, ld_yq=1056, ld_dq=1056, ld_dyq=1056), dict(rot=62), dict(ld_q=260), dict(ld_k=132)])
def test_rotations_without_a_kernel(kw):
    assert rope_fwd(rope(**kw)) == rope_bwd(rope(**kw)) == ML.MP_E_UNSUPPORTED


def test_rotation_axes():
    d = mp.rope_desc(10, 4, 2, 64, n_axes=2, axis=[0, 1] * 16)
    assert lib.mp_qk_norm_rope_bwd_workspace_bytes(C.byref(d)) > 0
    d.axis[31] = 2
    assert rope_fwd(d) == rope_bwd(d) == ML.MP_E_INVAL and b"axis" in lib.mp_last_error()
    d.axis[31], d.axis[32] = 0, 200          # (behind the last pair)
    assert lib.mp_qk_norm_rope_bwd_workspace_bytes(C.byref(d)) > 0
    for bad in ([0] * 31, [0] * 31 + [256], [0] * 31 + [-1]):
        with pytest.raises(ValueError, match="axes"):
            mp.rope_desc(10, 4, 2, 64, axis=bad)


def test_rotation_pointers():
    for k in ("q", "k", "pos", "freqs", "yq", "yk", "gq", "gk"):
        assert rope_fwd(rope(), **{k: None}) == ML.MP_E_INVAL
    for k in ("q", "k", "yq", "yk", "gq", "gk"):
        assert rope_fwd(rope(), **{k: A + 8}) == ML.MP_E_UNSUPPORTED and b"aligned" in lib.mp_last_error()
    for k in ("q", "k", "pos", "freqs", "dyq", "dyk", "dq", "dk", "dgq", "dgk", "gq", "gk"):
        assert rope_bwd(rope(), **{k: None}) == ML.MP_E_INVAL
    for k in ("q", "k", "dyq", "dyk", "dq", "dk", "gq", "gk"):
        assert rope_bwd(rope(), **{k: A + 2}) == ML.MP_E_UNSUPPORTED
    for k in ("pos", "freqs"):
        assert rope_fwd(rope(), **{k: A + 2}) == rope_bwd(rope(), **{k: A + 2}) == ML.MP_E_INVAL
    for k in ("dgq", "dgk"):
        assert rope_bwd(rope(), **{k: A + 1}) == ML.MP_E_INVAL
    assert rope_bwd(rope(), gq=None, gk=None) == ML.MP_E_INVAL and b"together" in lib.mp_last_error()
    need = lib.mp_qk_norm_rope_bwd_workspace_bytes(C.byref(rope()))
    assert rope_bwd(rope(), ws=None) == rope_bwd(rope(), ws=A + 8) == rope_bwd(rope(), n=100) == ML.MP_E_WORKSPACE and need > 100
    # nothing to do: no pointer is looked at
    assert rope_fwd(rope(rows=0), None, None, None, None, None, None, None, None) == ML.MP_OK
    assert rope_bwd(rope(rows=0), None, None, None, None, None, None, None, None, None, None, None, None, None, 0) == ML.MP_OK


@pytest.mark.parametrize("field", ["ld_q", "ld_k", "ld_yq", "ld_yk", "ld_dyq", "ld_dyk", "ld_dq", "ld_dk"])
def test_rope_offsets_within_a_workgroup_fit_32_bits(field):
    calls = [rope_fwd] * ("d" not in field[3:]) + [rope_bwd] * ("y" not in field[3:] or "d" in field[3:])
    for call in calls:
        assert call(rope(**{field: 1 << 22})) == ML.MP_E_UNSUPPORTED and b"below" in lib.mp_last_error()


def test_rotation_of_too_many_rows():
    assert rope_fwd(rope(rows=2 ** 31 - 1)) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()


def lp(rows=4, vocab=100, top=5, x=A, ld=100, t=A, c=1.0, logp=A, entropy=A, lse=A, ids=A, tops=A, ws=A, n=BIG):
    return lib.mp_token_logprobs(rows, vocab, top, x, ld, t, c, logp, entropy, lse, ids, tops, ws, n, None)


def lp_bwd(rows=4, vocab=100, x=A, ld=100, t=A, c=1.0, entropy=A, lse=A, g=A, h=A, st=A, d=A):
    return lib.mp_token_logprobs_bwd(rows, vocab, x, ld, t, c, entropy, lse, g, h, st, d, None)


def test_token_logprobs():
    for kw in (dict(rows=-1), dict(vocab=0), dict(ld=99), dict(c=0.0), dict(c=-1.0), dict(c=float("nan")), dict(c=2.0 ** -9), dict(c=257.0)):
        assert lp(**kw) == lp_bwd(**kw) == ML.MP_E_INVAL, kw
    for kw in (dict(x=None), dict(t=None), dict(logp=None), dict(ids=None), dict(tops=None), dict(top=0), dict(top=-1), dict(top=101), dict(x=A + 1), dict(t=A + 2),
               dict(logp=A + 2), dict(entropy=A + 1), dict(lse=A + 2), dict(ids=A + 2), dict(tops=A + 2)):
        assert lp(**kw) == ML.MP_E_INVAL, kw
    assert lp(vocab=200, ld=200, top=129) == lp(vocab=(1 << 20) + 1, ld=1 << 21) == lp_bwd(vocab=(1 << 20) + 1, ld=1 << 21) == ML.MP_E_UNSUPPORTED
    need = lib.mp_token_logprobs_workspace_bytes(4, 100000, 5)
    assert need > 0 and lib.mp_token_logprobs_workspace_bytes(8192, 32000, 5) == 0
    for kw in (dict(ws=None), dict(ws=A + 8), dict(n=need // 2)):
        assert lp(vocab=100000, ld=100000, **kw) == ML.MP_E_WORKSPACE
    for bad in ((-1, 100, 5), (0, 100, 5), (4, 0, 0), (4, 100, -1), (4, 100, 101), (4, 1000, 129), (4, (1 << 20) + 1, 5)):
        assert lib.mp_token_logprobs_workspace_bytes(*bad) == 0
    assert lp(rows=0, x=None, t=None, logp=None, entropy=None, lse=None, ids=None, tops=None, ws=None) == ML.MP_OK
    for kw in (dict(x=None), dict(lse=None), dict(d=None), dict(g=None), dict(t=None), dict(g=None, t=None, h=None), dict(entropy=None), dict(x=A + 1), dict(d=A + 1),
               dict(lse=A + 2), dict(g=A + 2), dict(h=A + 1), dict(st=A + 2)):
        assert lp_bwd(**kw) == ML.MP_E_INVAL, kw
    assert lp_bwd(rows=0, x=None, lse=None, d=None) == ML.MP_OK
    assert lp(rows=2 ** 31 - 1, top=0, ids=None, tops=None) == lp_bwd(rows=2 ** 31 - 1) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()


def distill(d, x=A, ids=A, t=A, y=A, st=A, loss=A, dx=A, ws=A, n=BIG):
    parts = ML.MeanParts()
    a = lib.mp_distill_scaled(C.byref(d), x, ids, t, y, st, loss, dx, ws, n, None)
    b = lib.mp_distill_scaled_parts(C.byref(d), x, ids, t, y, st, dx, ws, n, C.byref(parts), None) if loss else a
    assert a == b
    return a


@pytest.mark.parametrize("kw", [dict(rows=0), dict(rows=-1), dict(vocab=0), dict(top=0), dict(top=-3), dict(ld=99), dict(inv_temperature=0.0), dict(inv_temperature=2.0 ** -9),
                                dict(inv_temperature=257.0), dict(inv_temperature=float("nan")), dict(weight=float("inf")), dict(weight=float("nan")),
                                dict(hard_weight=float("nan")), dict(tail=2), dict(tail=-1), dict(reserved=1)])
def test_distillations_that_make_no_sense(kw):
    d = mp.distill_desc(4, 100, 8)
    for k, v in kw.items():
        setattr(d, k, v)
    assert distill(d) == ML.MP_E_INVAL and lib.mp_distill_workspace_bytes(C.byref(d)) == 0


def test_distillation():
    assert distill(mp.distill_desc(4, 1000, 129)) == distill(mp.distill_desc(4, (1 << 20) + 1, 8)) == ML.MP_E_UNSUPPORTED
    d = mp.distill_desc(4, 100, 8, hard_weight=0.5)
    for k in ("x", "ids", "t", "y", "st", "loss", "dx"):
        assert distill(d, **{k: None}) == ML.MP_E_INVAL, k
    for kw in (dict(x=A + 1), dict(dx=A + 1), dict(ids=A + 2), dict(t=A + 2), dict(y=A + 2), dict(st=A + 2)):
        assert distill(d, **kw) == ML.MP_E_INVAL, kw
    assert lib.mp_distill_scaled(C.byref(d), A, A, A, A, A, A + 2, A, A, BIG, None) == ML.MP_E_INVAL
    for vocab in (100, 140000):
        d = mp.distill_desc(4, vocab, 8)
        need = lib.mp_distill_workspace_bytes(C.byref(d))
        assert need >= 16 and distill(d, ws=None) == distill(d, ws=A + 8) == distill(d, n=15) == ML.MP_E_WORKSPACE
    assert lib.mp_distill_scaled(None, A, A, A, A, A, A, A, A, BIG, None) == ML.MP_E_INVAL and lib.mp_distill_workspace_bytes(None) == 0
    assert distill(mp.distill_desc(2 ** 31 - 1, 140000, 8), n=1 << 60) == ML.MP_E_INVAL and b"too many" in lib.mp_last_error()


def test_structs_and_limits_match_the_header():
    import os
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mp.h")).read()
    assert C.sizeof(ML.RopeDesc) == 68 + 128 and ML.RopeDesc.axis.offset == 68 and C.sizeof(ML.DistillDesc) == 36
    for name in ("MP_ROPE_AXES", "MP_ROPE_PAIRS", "MP_TOP_MAX"):
        assert hdr.split(f"#define {name} ")[1].split()[0] == str(getattr(ML, name)), name
    assert "#define MP_VOCAB_MAX (1 << 20)" in hdr and ML.MP_VOCAB_MAX == 1 << 20


def needed(call):
    assert call() == ML.MP_E_WORKSPACE
    return int(re.search(rb"of (\d+) bytes", lib.mp_last_error()).group(1))


ROWS = [1, 2, 3, 7, 8, 9, 61, 64, 65, 127, 128, 129, 255, 256, 257, 300, 512, 513, 1000, 1024, 1025, 4095, 4096, 4097, 8192, 12289, 16384, 16385, 70000]


@pytest.mark.parametrize("d_head,rot", [(64, 64), (128, 64), (80, 40), (256, 256), (24, 4)])
def test_rotation_workspaces_serve_fewer_rows(d_head, rot):
    sizes = [lib.mp_qk_norm_rope_bwd_workspace_bytes(C.byref(mp.rope_desc(r, 4, 2, d_head, rot=rot))) for r in ROWS]
    assert sizes == sorted(sizes)
    for r, size in zip(ROWS, sizes):
        assert needed(lambda: rope_bwd(mp.rope_desc(r, 4, 2, d_head, rot=rot), ws=None)) <= size


@pytest.mark.parametrize("vocab", [1000, 65529, 65530, 65536, 65537, 100000, 131071, 135161, 200001, 1 << 20])
def test_vocabulary_workspaces_serve_fewer_rows(vocab):
    sizes, lp_sizes = [], []
    for r in ROWS:
        sizes.append(lib.mp_distill_workspace_bytes(C.byref(mp.distill_desc(r, vocab, 100))))
        lp_sizes.append(lib.mp_token_logprobs_workspace_bytes(r, vocab, 100))
        for ld, x in ((vocab, A), (vocab, A + 2), ((vocab + 7) // 8 * 8, A), (vocab + 1, A)):
            assert needed(lambda: distill(mp.distill_desc(r, vocab, 100, ld=ld), x=x, ws=None)) <= sizes[-1]
            if vocab > 65536:            # (up to there a call may need none)
                assert needed(lambda: lp(r, vocab, 100, x=x, ld=ld, ws=None)) <= lp_sizes[-1]
    assert sizes == sorted(sizes) and lp_sizes == sorted(lp_sizes)

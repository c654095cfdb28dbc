"""Distillation from a teacher's lists: loss and seed gradient against 64 bits over vocabularies, lists, temperatures, hard labels,
alignments; lists that end early, repeat a class or name all; captured, in place, with the partial sums' form."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import _lib as ML
from oracle import FP64
from oracle import layers as L
from gpu_util import *
from test_gpu_token_logprobs import place


def problem(seed, rows, vocab, k, short=False, sharp=2.0):
    r = np.random.default_rng([seed, rows, vocab, k])
    t = r.standard_normal((rows, vocab)) * sharp
    x = (0.7 * t + r.standard_normal((rows, vocab))).astype(np.float16)
    lp = t - np.log(np.exp(t).sum(1, keepdims=True))
    ids = np.argsort(-lp, 1)[:, :k].astype(np.int32)
    teacher = np.take_along_axis(lp, ids, 1).astype(np.float32)
    if k > ids.shape[1]:
        raise ValueError
    if short:
        ids[np.arange(k)[None] >= r.integers(0, k + 1, (rows, 1))] = -1
    return x, ids, teacher, r.integers(0, vocab, rows).astype(np.int32)


def state(scale):
    st = mp.scale_state_alloc()
    mp.mp_scale_state_init(st, ML.MP_SCALE_STATIC, scale, 1)
    return st


def call(x, ids, teacher, targets, c=1.0, w=1.0, hard=0.0, tail=False, scale=2.0 ** 12, ld=None, offset=0, in_place=False):
    rows, vocab = x.shape
    view, ld = place(x, ld, offset)
    desc = mp.distill_desc(rows, vocab, ids.shape[1], ld=ld, inv_temperature=c, weight=w, hard_weight=hard, tail=tail)
    buf = torch.full((rows * ld + 24,), 9.0, dtype=torch.float16, device="cuda")
    d = view if in_place else torch.as_strided(buf, (rows, vocab), (ld, 1), 8 + (0 if in_place is None else offset))
    ws, loss = torch.full((mp.mp_distill_workspace_bytes(desc) // 4 + 4,), float("nan"), device="cuda"), empty32(1)
    mp.mp_distill_scaled(desc, view, i32(ids), f32(teacher), i32(targets) if hard else None, state(scale), loss, d, ws)
    return loss, d, buf


def check(x, ids, teacher, targets, c=1.0, w=1.0, hard=0.0, tail=False, scale=2.0 ** 12, **kw):
    """Errors in 2^-24: an exponent has c2 rounded twice (of the difference of two logits) and one rounding; an exponential 2; a sum up to 128
    terms a lane, 6 + 4 + 48 over lanes, waves and chunks, entries 8; a logarithm 4, the teacher's exponentials and their sum 20, products
    8: 240 + 8 |z| of each probability, twice for a quotient of two.  The gradient has half a step of fp16 besides, the loss a mean over
    rows of differences of logarithms that are up to |z| + ln(vocab) + |ln q|."""
    loss, d, buf = call(x, ids, teacher, targets, c, w, hard, tail, scale, **kw)
    rows, vocab = x.shape
    x64, t64, c, w, hard = x.astype(np.float64), teacher.astype(np.float64), *(float(np.float32(v)) for v in (c, w, hard))
    want_loss, want = L.distill_scaled(FP64, x64, ids, t64, scale, c, w, hard, targets, tail)
    lp, _ = L._log_softmax(FP64, x64 * c)
    p, p1 = np.exp(lp), np.exp(L._log_softmax(FP64, x64)[0])
    z = np.where(np.isfinite(x64), np.abs(x64), 0).max(1) * max(c, 1.0)
    unit = 2.0 ** -24 * (480 + 16 * z)[:, None]
    size = np.zeros_like(p)
    for i in range(rows):
        ok = (ids[i] >= 0) & (ids[i] < vocab)
        if not ok.any():
            continue
        q = np.exp(t64[i][ok]) if tail else np.exp(t64[i][ok] - t64[i][ok].max()) / np.exp(t64[i][ok] - t64[i][ok].max()).sum()
        rest = np.ones(vocab, bool)
        rest[ids[i][ok]] = False
        left = max(0.0, 1 - q.sum()) if tail and rest.any() else 0.0
        # (what is added up, each term by its size: a weight below 0 makes no term smaller, so |w|)
        size[i] += abs(w) * c * (p[i] * (q.sum() + left) + (left * p[i] * rest / max(p[i][rest].sum(), 1e-300) if left else 0))
        np.add.at(size[i], ids[i][ok], abs(w) * c * q)
    if hard:
        for i, t in enumerate(targets):
            if 0 <= t < vocab:
                size[i] += hard * p1[i]
                size[i, t] += hard
    tol = 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + unit * size * (scale / rows)
    err = np.abs(np32(d).astype(np.float64) - want) - tol
    assert err.max() <= 0, (err.max(), np.unravel_index(err.argmax(), err.shape))
    each = (abs(w) + abs(hard)) * unit[:, 0] * (2 + 2 * z + np.log(vocab) + np.abs(np.where(np.isfinite(t64), t64, 0)).max(1))
    # (inf where a target is a class that cannot be, on both sides)
    assert loss.item() == float(want_loss) or abs(loss.item() - float(want_loss)) <= each.mean() + 2.0 ** -20 * abs(float(want_loss)), (loss.item(), want_loss)
    return loss, d, buf


SHAPES = [(1, 1, 1), (3, 7, 3), (5, 100, 8), (61, 1000, 8), (4, 2049, 64), (3, 8192, 128), (2, 16391, 20), (3, 32768, 64), (2, 32767, 5), (2, 50021, 100), (3, 65536, 3), (2, 131071, 30),
          (1, 131072, 128), (33, 40000, 16), (2, 140000, 10), (300, 500, 4)]


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_vocabularies(shape, tail):
    check(*problem(1, *shape), tail=tail)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("c,w,hard", [(0.5, 4.0, 0.0), (0.5, 4.0, 0.3), (1.0, 0.7, 0.3), (1 / 0.7, 1.0, 1.0), (2.0 ** -8, 1.0, 0.0), (4.0, 0.0, 1.0)])
@pytest.mark.parametrize("shape", [(7, 1003, 9), (2, 40007, 20), (2, 132000, 7)], ids=str)
def test_temperatures_and_hard_labels(shape, tail, c, w, hard):
    x, ids, teacher, targets = problem(2, *shape)
    targets[0] = ids[0, 2]                                                # a listed one
    targets[1] = -1 if shape[0] == 2 else shape[1]
    check(x, ids, teacher, targets, c, w, hard, tail)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("offset", [0, 1, 3, 7])
@pytest.mark.parametrize("in_place", [False, True, None])
def test_alignment_and_in_place(offset, tail, in_place):
    loss, d, buf = check(*problem(3, 9, 2003, 12), tail=tail, hard=0.5, ld=2011, offset=offset, in_place=in_place)
    if in_place is not True:
        left = buf.clone()
        torch.as_strided(left, d.shape, d.stride(), d.storage_offset()).fill_(9.0)
        assert torch.all(left == 9.0)


@pytest.mark.parametrize("vocab", [1003, 40000])
@pytest.mark.parametrize("in_place", [False, True])
def test_in_place_over_many_rows(vocab, in_place):
    """More rows than workgroups, so each takes several."""
    x, ids, teacher, targets = problem(4, 2500 if vocab < 2000 else 600, vocab, 3)
    a = call(x, ids, teacher, targets, tail=True, in_place=in_place)
    rows = [0, 1, len(x) // 2, len(x) - 1]
    b = call(x[rows], ids[rows], teacher[rows], targets[rows], tail=True, scale=2.0 ** 12 * len(rows) / len(x))
    assert torch.equal(a[1][rows], b[1])


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("vocab", [60, 3000, 140000])
def test_lists(vocab, tail):
    """Lists that end early or hold nothing, that name a class several times, that the teacher gives nothing, with entries out of range."""
    x, ids, teacher, targets = problem(5, 9, vocab, 20)
    ids[0, 5:] = -1
    ids[1] = -1
    ids[2, :] = ids[2, 0]
    teacher[2] = np.log(0.04)
    ids[3, ::2] = ids[3, 1]
    teacher[3] -= 3
    ids[4, 3], ids[4, 7], ids[4, 9] = vocab, -2 ** 31, 2 ** 31 - 1
    teacher[5, 4:] = -np.inf
    ids[6] = np.arange(20) + 8                                            # side by side in few pieces
    teacher[6] -= 2
    ids[7], targets[7] = -1, -1
    targets[6] = 30
    check(x, ids, teacher, targets, tail=tail)
    loss, d, _ = check(x, ids, teacher, targets, c=0.5, hard=0.5, tail=tail)
    assert torch.all(d[7] == 0)


@pytest.mark.parametrize("vocab", [1, 8, 100, 128])
def test_lists_that_name_every_class(vocab):
    """Nothing is left for others: no term in r, though the teacher's probabilities add up to 1 only nearly."""
    x, ids, teacher, targets = problem(6, 4, vocab, vocab)
    check(x, ids, teacher - np.float32(1e-3), targets, tail=True)
    if vocab > 1:                                                         # each row's one other class cannot be
        x[np.arange(4), ids[:, -1]] = -np.inf
        check(x, ids[:, :-1], (teacher - np.float32(1e-3))[:, :-1], targets, tail=True)


def test_a_student_who_is_sure():
    """Nearly all of p in A: p_rest is 1e-9, where 1 minus a sum has nothing of it left."""
    x, ids, teacher, targets = problem(7, 6, 5000, 4)
    x = np.clip(x, -4, 4)
    for i in range(6):
        x[i, ids[i]] = 26 + np.arange(4)
    check(x, ids, teacher, targets, tail=True)
    check(x, ids, teacher, targets, tail=True, c=0.25, hard=1.0)


def test_large_logits():
    x, ids, teacher, targets = problem(8, 4, 900, 5)
    check((x * 2000).astype(np.float16), ids, teacher, targets)
    check((x * 2000).astype(np.float16), ids, teacher, targets, tail=True, hard=0.5, c=0.25)


@pytest.mark.parametrize("vocab", [200, 140000])
def test_non_finite_rows(vocab):
    x, ids, teacher, targets = problem(9, 8, vocab, 4)
    x[0, 100], x[1, 7], x[2] = np.nan, np.inf, -np.inf
    x[3, 5:] = -np.inf                                                    # classes that cannot be
    ids[3] = [0, 1, 2, 3]
    teacher[4, 1] = np.nan
    ids[5], x[5, 3] = -1, np.nan
    x[6, ids[6, 1]] = -np.inf                                             # a listed class that the student rules out
    loss, d, _ = call(x, ids, teacher, targets, tail=True)
    d = np32(d)
    assert np.isnan(d[[0, 1, 2]]).all() and np.isfinite(d[3]).all() and np.isnan(d[4]).all() and np.all(d[5] == 0) and np.isfinite(d[[6, 7]]).all()
    assert np.isnan(loss.item())
    loss, _, _ = call(x[6:], ids[6:], teacher[6:], targets[6:])
    assert loss.item() == np.inf


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("shape", SHAPES + [(70, 131071, 100), (400, 20000, 64)], ids=str)
def test_hard_labels_at_temperature_2(shape, tail):
    """Where one exponential serves both: all vocabularies, a student who is sure of listed and of other classes, far logits, -inf."""
    x, ids, teacher, targets = problem(11, *shape)
    check(x, ids, teacher, targets, 0.5, 4.0, 0.5, tail)
    sure = np.clip(x, -4, 4)
    sure[0, ids[0, 0]] = 40                                               # its other classes' p at temperature 1 are below 2^-50
    sure[-1, targets[-1]] = 3000
    check(sure, ids, teacher, targets, 0.5, -1.0, 0.5, tail)
    if shape[1] > 100 and shape[2] < shape[1] // 2:
        x = (x * 2000).astype(np.float16)
        x[0, ::3] = -np.inf
        x[0, ids[0]] = 1.0
        check(x, ids, teacher, targets, 0.5, 4.0, 0.5, tail)


@pytest.mark.parametrize("vocab", [200, 140000])
def test_non_finite_rows_at_temperature_2(vocab):
    x, ids, teacher, targets = problem(12, 5, vocab, 4)
    x[0, 100], x[1, 7], x[2] = np.nan, np.inf, -np.inf
    ids[3], targets[3], x[3, 3] = -1, -1, np.nan
    for tail in (False, True):
        loss, d, _ = call(x, ids, teacher, targets, c=0.5, hard=0.5, tail=tail)
        d = np32(d)
        assert np.isnan(d[[0, 1, 2]]).all() and np.all(d[3] == 0) and np.isfinite(d[4]).all() and np.isnan(loss.item())


def test_overflow_shows():
    """A gradient beyond fp16 becomes infinite, as every seed gradient does: the loss scale's policy sees it."""
    x, ids, teacher, targets = problem(10, 1, 50, 2)
    _, d, _ = call(x, ids, teacher, targets, scale=2.0 ** 24)
    assert torch.isinf(d).any()


@pytest.mark.parametrize("rows,vocab", [(70, 3001), (2, 140000)])
def test_parts_and_capture(rows, vocab):
    x, ids, teacher, targets = problem(11, rows, vocab, 16)
    view, ld = place(x)
    desc = mp.distill_desc(rows, vocab, 16, inv_temperature=0.5, weight=4.0, hard_weight=0.5, tail=True)
    args = [i32(ids), f32(teacher), i32(targets)]
    st = state(2.0 ** 10)
    n = mp.mp_distill_workspace_bytes(desc)
    ws, ws2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    d, loss, loss2, d2 = torch.empty_like(view), empty32(1), empty32(1), torch.empty_like(view)

    def go():
        parts = mp.mp_distill_scaled_parts(desc, view, *args, st, d, ws)
        mp.mp_loss_scale_update_mean(st, parts, loss)

    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for k in range(4):
        view.copy_(torch.from_numpy(problem(20 + k, rows, vocab, 16)[0]))
        args[0].copy_(torch.from_numpy(problem(30 + k, rows, vocab, 16)[1]))
        graph.replay()
        mp.mp_distill_scaled(desc, view, *args, st, loss2, d2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(loss, loss2) and torch.equal(d, d2), k


def test_gradient_against_differences():
    """As the token log probabilities' test: e^2 |f'''| / 6 with |f'''| below 8 a row of both terms, half a step of each gradient."""
    x, ids, teacher, targets = problem(12, 8, 60, 6)
    x = np.round(x.astype(np.float64) * 16) / 16
    kw = dict(hard=0.5, tail=True, scale=8.0)
    _, d, _ = call(x, ids, teacher, targets, **kw)
    way = np.round(np.random.default_rng(0).uniform(-1, 1, x.shape) * 4) / 4
    f = [call(x + e * way, ids, teacher, targets, **kw)[0].item() * 8 for e in (2.0 ** -3, -2.0 ** -3)]
    bound = 8 * 8 * 2.0 ** -6 / 6 + 2.0 ** -11 * np.abs(np32(d)).sum() + 2 * 2.0 ** -24 * 600 * 12 * 8 / 2.0 ** -2
    assert abs((np32(d).astype(np.float64) * way).sum() - (f[0] - f[1]) / 2.0 ** -2) <= bound


def test_teacher_to_student():
    """The teacher's top alternatives are the student's lists as they are: a student with the teacher's logits has nothing to learn."""
    rows, vocab, k = 40, 5003, 32
    x = problem(13, rows, vocab, 1)[0]
    view, ld = place(x)
    ids, top = torch.empty(rows, k, dtype=torch.int32, device="cuda"), empty32(rows, k)
    ws = torch.empty(mp.mp_token_logprobs_workspace_bytes(rows, vocab, k), dtype=torch.uint8, device="cuda")
    mp.mp_token_logprobs(rows, vocab, k, view, ld, None, 0.5, None, None, None, ids, top, ws)
    desc = mp.distill_desc(rows, vocab, k, inv_temperature=0.5, tail=True)
    d, loss = torch.empty_like(view), empty32(1)
    ws = torch.empty(mp.mp_distill_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    mp.mp_distill_scaled(desc, view, ids, top, None, state(float(rows)), loss, d, ws)
    # probabilities that are equal but for 480 + 16 |z| roundings, of a distribution that adds up to 1
    unit = 2.0 ** -24 * (480 + 16 * np.abs(x.astype(np.float64)).max())
    assert abs(loss.item()) <= 4 * unit * np.log(vocab) and d.float().abs().max().item() <= unit + 2.0 ** -25

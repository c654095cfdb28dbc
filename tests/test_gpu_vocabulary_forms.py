"""Log probabilities and distillation in each form that rows and vocabulary choose: the forms for many rows that only large calls reach."""
import functools

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from gpu_util import *
import test_gpu_distill as D
import test_gpu_token_logprobs as T


def test_more_rows_than_the_longest_forms_launch_could_count():
    """2^23 + 5 short rows, each with 64 lanes: the rows of a smaller call over and over, bit by bit."""
    rows, vocab, ld, few = (1 << 23) + 5, 3, 8, 1021
    x = T.rows_of("ties", few, ld).astype(np.float16)
    which = torch.arange(rows, device="cuda") % few
    small, t = torch.from_numpy(x).cuda(), i32(np.arange(few) % 4 - 1)
    big, targets = small[which], t[which]

    def run(n, logits, t):
        out = [empty32(n) for _ in range(3)] + [torch.empty(n, 2, dtype=torch.int32, device="cuda"), empty32(n, 2)]
        mp.mp_token_logprobs(n, vocab, 2, logits, ld, t, 1.0, *out)
        return out

    for a, b in zip(run(few, small, t), run(rows, big, targets)):
        assert torch.equal(a[which], b)


# ------------------------------------------------------------------------------------ log probabilities
# 65 rows and more of 16385 to 32768 classes take the form with four waves and 16 pieces a lane, and 8193 to 16384 the one with 8, however many rows
MANY = [(66, 20000), (65, 32753), (5, 12001), (3, 16384)]


@pytest.mark.parametrize("kind", ["plain", "ties", "banned", "equal", "one lane", "descending"])
@pytest.mark.parametrize("rows,vocab", MANY)
def test_scores(kind, rows, vocab):
    """No list; shares of it that each wave finds a bound for, up to 24; one bound of all beyond."""
    x, targets = T.rows_of(kind, rows, vocab), np.random.default_rng(1).integers(0, vocab, rows)
    for top in (0, 8, 24, 25, 128):
        T.check(x, targets, top)


@pytest.mark.parametrize("top", [8, 24, 25, 128])
@pytest.mark.parametrize("there", [130, 900])
@pytest.mark.parametrize("rows,vocab", MANY)
def test_few_classes_that_can_be(rows, vocab, there, top):
    """With some of the waves only, or fewer for a wave than its share of the list."""
    x = np.full((rows, vocab), -np.inf)
    x[:, 1024:1024 + there] = T.rows_of("plain", rows, there)
    T.check(x, np.arange(rows) + 1000, top)


@pytest.mark.parametrize("offset", [0, 1, 4, 7])
@pytest.mark.parametrize("rows,vocab", [(65, 16387), (65, 32749), (9, 16380)])
def test_any_alignment(offset, rows, vocab):
    T.check(T.rows_of("plain", rows, vocab), np.arange(rows) * 4, 11, ld=vocab + 5, offset=offset)


@pytest.mark.parametrize("rows,vocab", MANY)
def test_non_finite_scores(rows, vocab):
    """As they come: the first rows of the call, all others plain."""
    x = T.rows_of("plain", rows, vocab)
    bad = np.concatenate([x[:3]] * 3)
    bad[0, 3], bad[1, [5, 20, 30]], bad[1, 7], bad[2, 11] = np.nan, np.nan, np.inf, np.inf
    bad[3], bad[4, 1:], bad[5, 13], bad[6], bad[7] = -np.inf, -np.inf, -np.inf, np.nan, np.inf
    bad[8, ::2] = -np.inf
    bad = np.concatenate([bad, x])[:max(rows, 9)]
    got, _, _ = T.check(bad, np.arange(len(bad)) % 14, 25)
    assert got["logp"][4].item() == -np.inf and np.isfinite(got["logp"][9:].cpu().numpy()).all()


# ------------------------------------------------------------------------------------------ distillation
# 65 rows and more of 65537 to 135160 classes: a row in the registers of 12 waves, two pieces to a word of the map
LONG = [(66, 65537, 30), (65, 131071, 100), (65, 135160, 3)]


@functools.lru_cache(2)
def problem(rows, vocab, k):
    return D.problem(1, rows, vocab, k)


def fresh(*shape):
    return [x.copy() for x in problem(*shape)]


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("shape", LONG + [(5, 12001, 30), (70, 16384, 128)], ids=str)
def test_distillation(shape, tail):
    D.check(*fresh(*shape), tail=tail)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("c,w,hard", [(0.5, 4.0, 0.0), (0.5, 4.0, 0.3), (1.0, 0.7, 0.3), (1 / 0.7, 1.0, 1.0), (4.0, 0.0, 1.0)])
@pytest.mark.parametrize("shape", [LONG[0], (5, 12001, 30)], ids=str)
def test_temperatures_and_hard_labels(shape, tail, c, w, hard):
    x, ids, teacher, targets = fresh(*shape)
    targets[0], targets[1], targets[2] = ids[0, 2], -1, shape[1]
    D.check(x, ids, teacher, targets, c, w, hard, tail)


@pytest.mark.parametrize("tail", [False, True])
def test_other_temperatures_of_the_longest(tail):
    D.check(*fresh(*LONG[2]), c=1 / 3, w=9.0, hard=0.5, tail=tail)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("c,hard", [(1.0, 0.0), (0.5, 0.5), (0.7, 0.5)])
def test_lists_side_by_side(tail, c, hard):
    """Entries that share a word of the map, in one of its pieces and in both, with the target between them; a class named several times, lists
    that end early, hold nothing or name what is no class.  A row of 65537 begins an element further on in its piece than the one before."""
    x, ids, teacher, targets = fresh(*LONG[0])
    rows, vocab, k = LONG[0]
    ids[0, 5:] = -1
    ids[1] = -1
    ids[2, :] = ids[2, 0]
    teacher[2] = np.log(0.03)
    ids[3, ::2] = ids[3, 1]
    teacher[3] -= 3
    ids[4, 3], ids[4, 7], ids[4, 9] = vocab, -2 ** 31, 2 ** 31 - 1
    teacher[5, 4:] = -np.inf
    for i in range(6, 22):                       # both pieces of a word and the next word's first one
        ids[i], targets[i] = 16 * 100 + np.arange(k), 16 * 100 + i
        teacher[i] -= 3
    for i in range(22, 38):                      # one class of a word, the target elsewhere in it
        ids[i, 1:], ids[i, 0], targets[i] = -1, 16 * 200 + 5, 16 * 200 + i - 22
    for i in range(38, 54):                      # the ends of the row
        ids[i], targets[i] = np.concatenate([np.arange(k // 2), vocab - 1 - np.arange(k // 2)]), vocab - 1 - (i - 38)
        teacher[i] -= 3
    ids[54], targets[54] = -1, -1
    for i in range(55, 60):                      # twice in one word, in its two pieces
        ids[i, ::3], ids[i, 1::3] = 16 * 300 + 2, 16 * 300 + 11
        teacher[i] -= 3
    loss, d, _ = D.check(x, ids, teacher, targets, c=c, hard=hard, tail=tail)
    assert torch.all(d[54] == 0)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("in_place", [False, True, None])
def test_distillation_at_any_alignment_and_in_place(offset, tail, in_place):
    x, ids, teacher, targets = fresh(*LONG[0])
    loss, d, buf = D.check(x, ids[:, :12], teacher[:, :12], targets, tail=tail, hard=0.5, ld=x.shape[1] + 6, offset=offset, in_place=in_place)
    if in_place is not True:
        left = buf.clone()
        torch.as_strided(left, d.shape, d.stride(), d.storage_offset()).fill_(9.0)
        assert torch.all(left == 9.0)


@pytest.mark.parametrize("c,hard", [(1.0, 0.0), (0.5, 0.5), (0.7, 0.5)])
def test_non_finite_distillation(c, hard):
    x, ids, teacher, targets = fresh(*LONG[0])
    k = ids.shape[1]
    x[0, 100], x[1, 7], x[2] = np.nan, np.inf, -np.inf
    x[3, k:] = -np.inf                                                    # classes that cannot be
    ids[3], targets[3] = np.arange(k), 4
    teacher[4, 1] = np.nan
    ids[5], targets[5], x[5, 3] = -1, -1, np.nan
    x[6, ids[6, 1]] = -np.inf                                             # a listed class that the student rules out
    targets[6] = ids[6, 0]
    loss, d, _ = D.call(x, ids, teacher, targets, c=c, hard=hard, tail=True)
    d = np32(d)
    assert np.isnan(d[[0, 1, 2, 4]]).all() and np.all(d[5] == 0) and np.isfinite(d[3]).all() and np.isfinite(d[6:]).all() and np.isnan(loss.item())
    for v in (x, ids, teacher, targets):
        v[:6] = v[7]
    loss, _, _ = D.call(x, ids, teacher, targets, c=c, hard=hard)
    assert loss.item() == np.inf


@pytest.mark.parametrize("tail", [False, True])
def test_the_same_rows_in_registers_and_in_chunks(tail):
    """70 rows of 100000 classes are each held whole, 4 of them cut into chunks: both as near to 64 bits, both alike in place."""
    x, ids, teacher, targets = D.problem(4, 70, 100000, 9)
    for rows in (np.arange(70), np.array([0, 1, 35, 69])):
        part = [v[rows] for v in (x, ids, teacher, targets)]
        scale = 2.0 ** 12 * len(rows) / 70
        loss, d, _ = D.check(*part, hard=0.5, c=0.7, tail=tail, scale=scale)
        loss2, d2, _ = D.call(*part, hard=0.5, c=0.7, tail=tail, scale=scale, in_place=True)
        assert torch.equal(d, d2) and torch.equal(loss, loss2)


@pytest.mark.parametrize("vocab", [500, 65537, 140000])
def test_lists_to_which_the_teacher_gives_nothing(vocab):
    """All entries -inf: q = 0.  Renormalised such a row has neither loss nor gradient; with the rest all of the teacher is there, L = -ln p_rest.
    Tolerances as counted in the distillation's own tests: 2^-24 (480 + 16 |z|), times p r + r p / p_rest or what the logarithms are up to."""
    rows, scale = 66, 2.0 ** 12
    x, ids, teacher, targets = D.problem(14, rows, vocab, 5)
    teacher[:] = -np.inf
    loss, d, _ = D.call(x, ids, teacher, targets, scale=scale)
    assert loss.item() == 0 and torch.all(d == 0)
    loss, d, _ = D.call(x, ids, teacher, targets, scale=scale, tail=True)
    x = x.astype(np.float64)
    p = np.exp(x - np.log(np.exp(x).sum(1, keepdims=True)))
    rest = p.copy()
    np.put_along_axis(rest, ids, 0.0, 1)
    p_rest = rest.sum(1, keepdims=True)
    want, z = (p - rest / p_rest) * (scale / rows), np.abs(x).max(1, keepdims=True)
    unit = 2.0 ** -24 * (480 + 16 * z)
    assert np.all(np.abs(np32(d) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + unit * (p + rest / p_rest) * (scale / rows))
    assert abs(loss.item() + np.log(p_rest).mean()) <= (unit * (2 + 2 * z + np.log(vocab))).mean()

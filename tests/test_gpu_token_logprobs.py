"""Log probabilities of given tokens, entropies, alternatives and their gradient: against 64 bits, exact order of the alternatives with
ties and non-finite logits, any alignment, rows cut into chunks, captured, in place."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import _lib as ML
from oracle import FP64
from oracle import layers as L
from gpu_util import *


def place(x, ld=None, offset=0):
    """x [rows, vocab] on the device with rows ld apart, `offset` elements behind a 16-byte boundary; what is around it is NaN."""
    rows, vocab = x.shape
    ld = ld or vocab
    buf = torch.full((rows * ld + offset + 8,), float("nan"), dtype=torch.float16, device="cuda")
    view = torch.as_strided(buf, (rows, vocab), (ld, 1), offset)
    view.copy_(torch.from_numpy(x.astype(np.float16)))
    return view, ld


def call(x, targets, top, c=1.0, ld=None, offset=0):
    rows, vocab = x.shape
    view, ld = place(x, ld, offset)
    out = dict(logp=empty32(rows), entropy=empty32(rows), lse=empty32(rows), ids=torch.full((rows, top), -7, dtype=torch.int32, device="cuda") if top else None,
               top=empty32(rows, top) if top else None)
    ws = torch.full((mp.mp_token_logprobs_workspace_bytes(rows, vocab, top) // 4 + 4,), float("nan"), device="cuda")
    mp.mp_token_logprobs(rows, vocab, top, view, ld, i32(targets), c, out["logp"], out["entropy"], out["lse"], out["ids"], out["top"], ws)
    return out, view, ld


def check(x, targets, top, c=1.0, ld=None, offset=0):
    """Errors in 2^-24: an exponent c2 x - ref has c2 rounded twice (2 of the difference of two logits, up to twice the largest) and one
    rounding; exponential 2; up to 128 terms a lane, 6 + 4 over lanes and waves, 48 chunks; logarithm 4, products 4: 200 + 8 |z|.  An
    entropy weighs them by |y|, whose mean is at most ln(vocab) + 1."""
    x = x.astype(np.float16).astype(np.float64)
    got, view, ld = call(x, targets, top, c, ld, offset)
    c = float(np.float32(c))
    logp, entropy, lse, ids, tops = L.token_logprobs(FP64, x, np.asarray(targets), c, top)
    finite = np.where(np.isfinite(x), np.abs(x), 0).max(1) * c
    tol = 2.0 ** -24 * (200 + 8 * finite)
    for name, want, t in (("logp", logp, tol), ("lse", lse, tol), ("entropy", entropy, tol * (1 + np.log(x.shape[1])))):
        g = got[name].double().cpu().numpy()
        assert np.array_equal(np.isnan(g), np.isnan(want)) and np.array_equal(np.isinf(g), np.isinf(want)), (name, g, want)
        ok = np.isfinite(want)
        assert np.all(np.abs(g[ok] - want[ok]) <= t[ok]), (name, np.abs(g[ok] - want[ok]).max(), t[ok].min())
    if top:
        assert np.array_equal(got["ids"].cpu().numpy(), ids)
        g = got["top"].double().cpu().numpy()
        assert np.array_equal(np.isnan(g), np.isnan(tops)) and np.array_equal(np.isneginf(g), np.isneginf(tops))
        ok = np.isfinite(tops)
        assert np.all(np.abs(g[ok] - tops[ok]) <= np.broadcast_to(tol[:, None], g.shape)[ok])
    return got, view, ld


def rows_of(kind, rows, vocab, seed=0):
    r = np.random.default_rng([seed, rows, vocab])
    x = r.standard_normal((rows, vocab)) * 2.5
    if kind == "peaked":
        x[np.arange(rows), r.integers(0, vocab, rows)] += 20
    elif kind == "ties":
        x = np.round(x)
    elif kind == "equal":
        x[:] = -3.25
    elif kind == "zeros":
        x = np.where(r.random((rows, vocab)) < 0.5, 0.0, -0.0)
    elif kind == "banned":
        x[r.random((rows, vocab)) < 0.7] = -np.inf
        x[:, vocab // 2] = 1.0
    elif kind == "ascending":
        x = np.sort(x, 1)
    elif kind == "descending":
        x = -np.sort(-x, 1)
    elif kind == "far":
        x = r.uniform(-60000, 60000, (rows, vocab))
    elif kind == "one lane":
        x[:, : min(vocab, 8)] += 30                                       # the best of all in one 16-byte piece
    return x


@pytest.mark.parametrize("kind", ["plain", "peaked", "ties", "equal", "zeros", "banned", "ascending", "descending", "far", "one lane"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (3, 7, 7), (4, 64, 20), (5, 1000, 8), (2, 4099, 128), (3, 32768, 20), (2, 32767, 64), (260, 2049, 5), (1, 50021, 100), (2, 131071, 8)],
                         ids=str)
def test_values(kind, shape):
    rows, vocab, top = shape
    targets = np.random.default_rng(1).integers(0, vocab, rows)
    targets[-1] = vocab - 1
    check(rows_of(kind, rows, vocab), targets, top)


@pytest.mark.parametrize("kind", ["plain", "ties", "banned", "ascending", "one lane"])
@pytest.mark.parametrize("top", [31, 32, 33, 63, 65, 100, 127, 128])
@pytest.mark.parametrize("vocab", [128, 510, 700, 1021, 1777])
def test_long_lists_of_short_rows(kind, top, vocab):
    """Between the ways that the bound is found in, and lists as long as the pieces are many."""
    check(rows_of(kind, 3, vocab), [0, vocab // 2, vocab - 1], top)


@pytest.mark.parametrize("top", [1, 20, 24, 25, 32, 33, 48, 49, 64, 65, 128])
@pytest.mark.parametrize("vocab", [2500, 6000, 20000, 50021, 70001])
@pytest.mark.parametrize("there", [130, 512, 900])
def test_few_classes_that_can_be(there, vocab, top):
    """The finite ones side by side, so with some of the waves only: as many as the list, or fewer for some waves; rows many and few."""
    for rows in (2, 1030 if vocab < 4096 else 3):
        x = np.full((rows, vocab), -np.inf)
        first = min(1024, vocab - there)
        x[:, first:first + there] = rows_of("plain", rows, there)
        check(x, np.arange(rows) % vocab, top)


@pytest.mark.parametrize("rows", [1023, 1024])
@pytest.mark.parametrize("vocab,ld,top", [(2049, 2049, 128), (4090, 4097, 20), (4096, 4096, 100), (3001, 3001, 0)])
def test_many_rows(rows, vocab, ld, top):
    check(rows_of("plain", rows, vocab), np.arange(rows) % vocab, top, ld=ld, offset=3 if ld > vocab else 0)


@pytest.mark.parametrize("offset", range(8))
@pytest.mark.parametrize("vocab,ld", [(1001, 1001), (4096, 4101), (40, 57), (33000, 33003)])
def test_any_alignment(offset, vocab, ld):
    check(rows_of("plain", 9, vocab), np.arange(9) * 4, 11, ld=ld, offset=offset)


@pytest.mark.parametrize("c", [0.5, 1.0 / 0.7, 2.0 ** -8, 2.0 ** 8])
def test_temperatures(c):
    check(rows_of("plain", 4, 3001), [0, 1, 2, 3000], 6, c)
    check(rows_of("plain", 1, 70001), [69999], 6, c)


def test_targets_that_there_are_not():
    got, _, _ = check(rows_of("plain", 5, 100), [-1, 100, 99, -2 ** 31, 2 ** 31 - 1], 0)
    assert got["logp"][[0, 1, 3, 4]].tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("vocab", [40, 5000, 66000])
def test_non_finite_rows(vocab):
    x = rows_of("plain", 9, vocab)
    x[0, 3] = np.nan
    x[1, [5, 20, 30]] = np.nan
    x[1, 7] = np.inf
    x[2, 11] = np.inf
    x[3] = -np.inf
    x[4, 1:] = -np.inf                                                    # one class is certain
    x[5, 13] = -np.inf
    x[6] = np.nan
    x[7] = np.inf
    x = x.astype(np.float16)
    x.view(np.uint16)[0, 9] = 0xFE01                                      # a NaN with its sign set, with a payload
    got, _, _ = check(x, [0, 1, 2, 3, 0, 13, 5, 5, 5], 25)
    # (a certain class: its exponent y is what is left of c2 x - ref, up to 2^-24 of |c2 x| < 32, s = 2^y, and log2 s and t / s round s, s
    # and y to 2^-24 each)
    assert abs(got["entropy"][4].item()) <= 2.0 ** -22 and abs(got["logp"][4].item()) <= 2.0 ** -22 and got["logp"][5].item() == -np.inf


def test_single_outputs():
    x = rows_of("plain", 3, 500)
    full, view, ld = call(x, [1, 2, 3], 4)
    for name in ("logp", "entropy", "lse"):
        out = empty32(3)
        kw = {n: (out if n == name else None) for n in ("logp", "entropy", "lse")}
        mp.mp_token_logprobs(3, 500, 0, view, ld, i32([1, 2, 3]) if name == "logp" else None, 1.0, **kw)
        assert torch.equal(out, full[name])
    ids, top = torch.empty(3, 4, dtype=torch.int32, device="cuda"), empty32(3, 4)
    mp.mp_token_logprobs(3, 500, 4, view, ld, None, 1.0, None, None, None, ids, top)
    assert torch.equal(ids, full["ids"]) and torch.equal(top, full["top"])


# ------------------------------------------------------------------------------------------------------ gradient
def gradient(x, targets, c, g, h, scale=2.0 ** 10, ld=None, offset=0, in_place=False, no_state=False):
    rows, vocab = x.shape
    out, view, ld = call(x, targets, 0, c, ld, offset)
    st = None
    if not no_state:
        st = mp.scale_state_alloc()
        mp.mp_scale_state_init(st, ML.MP_SCALE_STATIC, scale, 1)
    buf = torch.full((rows * ld + 24,), 9.0, dtype=torch.float16, device="cuda")
    d = view if in_place else torch.as_strided(buf, (rows, vocab), (ld, 1), 8 + (0 if in_place is None else offset))
    mp.mp_token_logprobs_bwd(rows, vocab, view, ld, i32(targets) if g is not None else None, c, out["entropy"] if h is not None else None, out["lse"],
                             None if g is None else f32(g), None if h is None else f32(h), st, d)
    return d, buf, ld


def check_gradient(x, targets, c, g, h, scale=2.0 ** 10, **kw):
    """Half a step of fp16, and of each term p (g + h (ln p + entropy)): the errors of lse and entropy that the call is given, 200 + 8 |z| and
    that times ln(vocab) + 1 of them, and as many again of its own exponent."""
    x = x.astype(np.float16).astype(np.float64)
    d, buf, ld = gradient(x, targets, c, g, h, scale, **kw)
    g0, h0 = (np.zeros(len(x)) if v is None else np.asarray(v, np.float32).astype(np.float64) for v in (g, h))
    want = L.token_logprobs_bwd(FP64, x, np.asarray(targets), float(np.float32(c)), g0, h0, scale)
    lp, _ = L._log_softmax(FP64, x * c)
    p = np.exp(lp)
    lp = np.where(p == 0, 0, lp)
    logv = 1 + np.log(x.shape[1])
    size = scale * c * p * (np.abs(g0)[:, None] + np.abs(h0)[:, None] * (np.abs(lp) + 2 * logv))
    tol = 2.0 ** -11 * np.abs(want) + 2.0 ** -25 + 2.0 ** -24 * (400 + 16 * np.where(np.isfinite(x), np.abs(x), 0).max(1) * c)[:, None] * size
    err = np.abs(np32(d).astype(np.float64) - want) - tol
    assert err.max() <= 0, (err.max(), np.unravel_index(err.argmax(), err.shape))
    return d, buf, ld


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 7), (6, 1000), (2, 32768), (5, 4099), (1, 131071)])
@pytest.mark.parametrize("which", ["both", "logp", "entropy"])
def test_gradient(rows, vocab, which):
    r = np.random.default_rng(rows)
    g, h = r.standard_normal(rows), r.standard_normal(rows) * 0.1
    check_gradient(rows_of("peaked" if rows % 2 else "banned", rows, vocab), r.integers(0, vocab, rows), 0.8, g if which != "entropy" else None, h if which != "logp" else None)


@pytest.mark.parametrize("offset", [0, 1, 5])
@pytest.mark.parametrize("in_place", [False, True, None])
def test_gradient_alignment_and_in_place(offset, in_place):
    """None: the gradient lies at another alignment than the logits."""
    x, targets = rows_of("plain", 7, 2003), [0, 5, 2002, -1, 2003, 1000, 7]
    d, buf, ld = check_gradient(x, targets, 1.0, np.ones(7), np.full(7, 0.2), ld=2010, offset=offset, in_place=in_place)
    if in_place is not True:
        left = buf.clone()
        torch.as_strided(left, d.shape, d.stride(), d.storage_offset()).fill_(9.0)
        assert torch.all(left == 9.0)                                     # nothing else was written


def test_gradient_without_a_state_is_unscaled():
    x = rows_of("plain", 3, 333)
    a, _, _ = gradient(x, [1, 2, 3], 1.0, np.ones(3), None, no_state=True)
    b, _, _ = gradient(x, [1, 2, 3], 1.0, np.ones(3), None, scale=1.0)
    assert torch.equal(a, b)


def test_rows_that_are_left_out_have_no_gradient_whatever_they_hold():
    x = rows_of("plain", 6, 100)
    x[1], x[2, 4], x[3, 5] = np.nan, np.inf, np.nan
    d, _, _ = gradient(x, [3, 3, -1, 3, 3, 100], 1.0, [1, 0, 1, 0, 1, 1], [0, 0, 0, 0.5, 0, 0])
    d = np32(d)
    assert np.all(d[[1, 2, 5]] == 0) and np.isnan(d[3]).all() and np.isfinite(d[[0, 4]]).all()


def test_gradient_against_differences():
    """(f(x + e) - f(x - e)) / 2 of the calls' own sums, e = 2^-3 in fp16 exactly: off by e^2 f''' / 6 with |f'''| below 4 here, and by
    the sums' own 2^-24 (200 + 8 |z|) (1 + ln vocab) of 8 rows over 2^-3."""
    r = np.random.default_rng(3)
    x = np.round(r.standard_normal((8, 60)) * 16) / 16
    targets, g, h = r.integers(0, 60, 8), r.standard_normal(8), r.standard_normal(8)
    d, _, _ = gradient(x, targets, 1.0, g, h, scale=1.0)
    way = np.round(r.uniform(-1, 1, x.shape) * 4) / 4
    f = []
    for e in (2.0 ** -3, -2.0 ** -3):
        out, _, _ = call(x + e * way, targets, 0)
        f.append((out["logp"].double().cpu().numpy() * g + out["entropy"].double().cpu().numpy() * h).sum())
    want = (f[0] - f[1]) / 2.0 ** -2
    assert abs((np32(d).astype(np.float64) * way).sum() - want) <= 8 * 4 * 2.0 ** -6 / 6 + 8 * 2.0 ** -24 * 300 * 6 / 2.0 ** -2 + 2.0 ** -11 * np.abs(np32(d)).sum()


# ------------------------------------------------------------------------------------------------------- as used
@pytest.mark.parametrize("rows,vocab", [(2, 40000), (30, 1000)])
def test_captured_and_replayed(rows, vocab):
    view, ld = place(rows_of("plain", rows, vocab))
    t, d = i32(np.arange(rows)), torch.empty_like(view)
    st = mp.scale_state_alloc()
    mp.mp_scale_state_init(st, ML.MP_SCALE_STATIC, 8.0, 1)

    def go(ws):
        o = [empty32(rows), empty32(rows), empty32(rows), torch.empty(rows, 9, dtype=torch.int32, device="cuda"), empty32(rows, 9), torch.empty_like(view)]
        mp.mp_token_logprobs(rows, vocab, 9, view, ld, t, 1.0, *o[:5], ws)
        mp.mp_token_logprobs_bwd(rows, vocab, view, ld, t, 1.0, o[1], o[2], o[0], o[1], st, o[5])
        return o

    ws = [torch.empty(mp.mp_token_logprobs_workspace_bytes(rows, vocab, 9), dtype=torch.uint8, device="cuda") for _ in range(2)]
    go(ws[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = go(ws[0])
    for k in range(4):
        view.copy_(torch.from_numpy(rows_of("ties" if k == 2 else "plain", rows, vocab, k + 1).astype(np.float16)))
        graph.replay()
        got = [x.clone() for x in out]
        want = go(ws[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_two_streams_with_workspaces_of_their_own():
    x = [place(rows_of("plain", 3, 40000, s))[0] for s in (1, 2)]
    run = lambda v: _top(v, torch.empty(mp.mp_token_logprobs_workspace_bytes(3, 40000, 16), dtype=torch.uint8, device="cuda"))  # noqa: E731
    want = [run(v) for v in x]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for k in range(2):
        with torch.cuda.stream(streams[k]):
            got[k] = run(x[k])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def _top(view, ws):
    rows, vocab = view.shape
    out = torch.empty(rows, 16, dtype=torch.int32, device="cuda"), empty32(rows, 16)
    mp.mp_token_logprobs(rows, vocab, 16, view, vocab, None, 1.0, None, None, None, *out, ws)
    return out


def test_the_longest_rows():
    """2^20 classes, and rows that lie beyond 2^31 elements."""
    check(rows_of("plain", 1, 1 << 20), [(1 << 20) - 1], 128)
    rows, vocab = 2100, 1 << 20
    x = torch.full((rows, vocab), -60000.0, dtype=torch.float16, device="cuda")
    x[rows - 1, vocab - 1] = 1.0
    x[rows - 1, 5] = 0.0
    out = [empty32(rows) for _ in range(3)] + [torch.empty(rows, 2, dtype=torch.int32, device="cuda"), empty32(rows, 2)]
    ws = torch.empty(mp.mp_token_logprobs_workspace_bytes(rows, vocab, 2), dtype=torch.uint8, device="cuda")
    t = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    mp.mp_token_logprobs(rows, vocab, 2, x, vocab, t, 1.0, *out, ws)
    assert out[3][-1].tolist() == [vocab - 1, 5] and out[3][0].tolist() == [0, 1]
    assert abs(out[0][-1].item() + np.log1p(np.exp(-1.0))) < 1e-6 and abs(out[0][0].item() + 20 * np.log(2)) < 1e-4
    g = torch.ones(rows, device="cuda")
    mp.mp_token_logprobs_bwd(rows, vocab, x, vocab, t, 1.0, None, out[2], g, None, None, x)
    assert abs(x[-1, 5].item() + 0.26894) < 1e-3 and abs(x[-1, -1].item() - 0.26894) < 1e-3 and x[-1, 6].item() == 0

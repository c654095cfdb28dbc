"""Embedding lookup and its gradient through the C ABI against the oracle.

Forward is one fp32 product and one rounding: equal bits.  Backward: at most half a step of the result (2^-11), and of the sum of n rows
n 2^-24 times the sum of their magnitudes; with a second gradient one more rounding of each of the two values."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import _lib as ML
from oracle import FP64, MIXED
from oracle import layers as L
from oracle.numerics import half_bits
from gpu_util import *

S16 = MIXED.store


def tokens_of(kind, rows, vocab, r):
    if kind == "spread":
        return r.integers(0, vocab, rows)
    if kind == "zipf":
        return np.minimum((vocab ** r.random(rows)).astype(np.int64) - 1, vocab - 1)
    if kind == "same":
        return np.full(rows, vocab - 1)
    if kind == "pads":                                   # half of them no token at all
        return np.where(r.random(rows) < 0.5, r.choice([-1, vocab, 2 ** 31 - 1, -2 ** 31], rows), r.integers(0, vocab, rows))
    if kind == "none":
        return np.full(rows, -1)
    return np.arange(rows) % vocab                       # "in turn"


def place(x, skew):
    """The array on the device, `skew` elements behind a 16-byte boundary."""
    t = torch.empty(x.size + 16, dtype=torch.float16, device="cuda")
    t[skew:skew + x.size] = h16(x).view(-1)
    return t[skew:skew + x.size].view(x.shape)


def check(rows, vocab, d, kind, scale=1.5, add=False, skew=0, seed=0):
    r = np.random.default_rng(seed + rows + vocab + d)
    tok = tokens_of(kind, rows, vocab, r).astype(np.int32)
    w, dy, second = S16(r.standard_normal((vocab, d))), S16(r.standard_normal((rows, d))), S16(r.standard_normal((vocab, d)))
    tokens, y = i32(tok), place(np.full((rows, d), 7.0), skew)
    mp.mp_embedding_fwd(rows, vocab, d, tokens, place(w, skew), scale, y)
    assert np.array_equal(bits(y), half_bits(L.embedding_fwd(MIXED, tok, w, scale))), "forward"
    dw, ws = place(np.full((vocab, d), 7.0), skew), torch.empty(mp.mp_embedding_bwd_workspace_bytes(rows, vocab, d), dtype=torch.uint8, device="cuda")
    mp.mp_embedding_bwd(rows, vocab, d, tokens, place(dy, skew), scale, dw, ws=ws)
    ok = (tok >= 0) & (tok < vocab)
    ref, mag, n = np.zeros((vocab, d)), np.zeros((vocab, d)), np.zeros(vocab)
    np.add.at(ref, tok[ok], scale * dy[ok].astype(np.float64))
    np.add.at(mag, tok[ok], scale * np.abs(dy[ok]).astype(np.float64))
    np.add.at(n, tok[ok], 1)
    bound = 2.0 ** -11 * np.abs(ref) + (n[:, None] + 2) * 2.0 ** -24 * mag + 2.0 ** -25
    assert np.all(np.abs(np32(dw) - ref) <= bound), "backward"
    assert torch.all(dw[torch.from_numpy(n == 0).cuda()] == 0)
    again = torch.empty_like(dw)
    mp.mp_embedding_bwd(rows, vocab, d, tokens, place(dy, skew), scale, again, ws=ws)
    assert torch.equal(again, dw), "two calls"
    if add:
        other, tied = place(second, skew), place(second, skew)
        mp.mp_embedding_bwd(rows, vocab, d, tokens, place(dy, skew), scale, again, add=other, ws=ws)
        mp.mp_embedding_bwd(rows, vocab, d, tokens, place(dy, skew), scale, tied, add=tied, ws=ws)
        assert np.array_equal(bits(again), half_bits(S16(np32(dw) + second))), "with a second gradient"
        assert torch.equal(again, tied), "in place"


@pytest.mark.parametrize("kind", ["spread", "zipf", "same", "pads", "none", "in turn"])
@pytest.mark.parametrize("rows", [1, 31, 32, 33, 64, 65, 500, 2047, 2048, 2049, 5000])
def test_row_counts(rows, kind):
    check(rows, 97, 24, kind, add=True)


@pytest.mark.parametrize("d,skew", [(1, 0), (7, 0), (8, 0), (8, 1), (24, 3), (64, 0), (192, 4), (515, 0), (512, 0), (520, 0), (1024, 1), (1032, 0)])
def test_widths_and_alignments(d, skew):
    check(300, 61, d, "zipf", scale=d ** 0.5, add=True, skew=skew)


@pytest.mark.parametrize("rows,vocab", [(40, 1), (3, 30000), (5000, 30000), (65536, 100), (65537, 3), (70000, 2 ** 21 - 1), (140000, 50000)])
def test_many_tokens_and_words(rows, vocab):
    """Up to several levels of merging, the largest vocabulary."""
    check(rows, vocab, 2 if vocab < 2 ** 20 else 1, "zipf")
    check(rows, vocab, 1, "same")


@pytest.mark.parametrize("rows", [7, 8, 9, 15, 16, 17, 127, 129, 257, 511, 1025])
@pytest.mark.parametrize("kind,d,skew", [("same", 9, 1), ("zipf", 17, 0), ("pads", 8, 3)])
def test_pieces_and_parts(rows, kind, d, skew):
    check(rows, 13, d, kind, add=True, skew=skew)


@pytest.mark.parametrize("rows,d", [(20000, 840), (70000, 500), (100003, 672), (140000, 1027)])
@pytest.mark.parametrize("kind", ["zipf", "pads", "same"])
def test_long_chunks(rows, d, kind):
    """Chunks of 16, 32, 64 positions (more rows and columns than the oracle is quick for: the sums in 64 bits on the device)."""
    vocab, r = 3001, np.random.default_rng(rows)
    tok = torch.from_numpy(tokens_of(kind, rows, vocab, r).astype(np.int32)).cuda()
    dy = torch.randn(rows, d, device="cuda", generator=torch.Generator("cuda").manual_seed(rows)).half()
    dw, ws = empty16(vocab, d), torch.empty(mp.mp_embedding_bwd_workspace_bytes(rows, vocab, d), dtype=torch.uint8, device="cuda")
    mp.mp_embedding_bwd(rows, vocab, d, tok, dy, 0.5, dw, ws=ws)
    ok = (tok >= 0) & (tok < vocab)
    at, x = tok[ok].long(), 0.5 * dy[ok].double()
    order = torch.argsort(at, stable=True)
    count = torch.bincount(at, minlength=vocab)
    end = torch.cumsum(count, 0)

    def sums(v):
        out = torch.zeros(vocab, *v.shape[1:], dtype=torch.float64, device="cuda")
        for t in torch.nonzero(count > 50).flatten().tolist():          # (adding these one by one takes a second)
            out[t] = v[order[end[t] - count[t]:end[t]]].sum(0)
        few = count[at] <= 50
        return out.index_add_(0, at[few], v[few])
    ref, mag, n = sums(x), sums(x.abs()), sums(torch.ones(at.numel(), dtype=torch.float64, device="cuda"))
    assert torch.all((dw.double() - ref).abs() <= 2.0 ** -11 * ref.abs() + (n[:, None] + 2) * 2.0 ** -24 * mag + 2.0 ** -25)
    again = torch.empty_like(dw)
    mp.mp_embedding_bwd(rows, vocab, d, tok, dy, 0.5, again, ws=ws)
    assert torch.equal(again, dw)


def test_three_rounds_of_merging():
    check(2048 * 32 * 32 + 5000, 50000, 3, "zipf")


def test_offsets_beyond_32_bits():
    """A table of 2.2e9 elements: the rows of a few tokens, and zeros everywhere else."""
    vocab, d = 2000003, 1100
    w, dw = (torch.zeros(vocab, d, dtype=torch.float16, device="cuda") for _ in range(2))
    tok = [vocab - 1, 5, 1960000, vocab - 1]
    r = np.random.default_rng(1)
    rows, dy, y = S16(r.standard_normal((4, d))), S16(r.standard_normal((4, d))), empty16(4, d)
    rows[3] = rows[0]
    w[torch.tensor(tok, device="cuda")] = h16(rows)
    mp.mp_embedding_fwd(4, vocab, d, i32(tok), w, 2.0, y)
    assert np.array_equal(bits(y), half_bits(S16(2 * rows)))
    dw[::1000] = 7
    mp.mp_embedding_bwd(4, vocab, d, i32(tok), h16(dy), 1.0, dw, ws=ws_bytes(mp.mp_embedding_bwd_workspace_bytes(4, vocab, d)))
    want = {vocab - 1: S16((dy[0].astype(np.float32) + dy[3]).astype(np.float32)), 5: dy[1], 1960000: dy[2]}
    for t, x in want.items():
        assert np.array_equal(bits(dw[t]), half_bits(x)), t
        dw[t] = 0
    assert all(int(torch.count_nonzero(dw[i:i + 100000])) == 0 for i in range(0, vocab, 100000))


@pytest.mark.parametrize("other", [0, 3])
def test_the_second_gradient_where_there_is_no_token(other):
    """It is copied, whatever its alignment beside dw's, and its infinities are reported."""
    vocab, d = 700, 19
    second = S16(np.random.default_rng(other).standard_normal((vocab, d)))
    for bad in (None, 0, vocab * d - 1, 5000):
        if bad is not None:
            second.reshape(-1)[bad] = -np.inf
        st = mp.scale_state_alloc()
        mp.mp_scale_state_init(st, ML.MP_SCALE_BACKOFF, 1.0, 3)
        dw, ws = place(np.full((vocab, d), 7.0), 1), torch.empty(mp.mp_embedding_bwd_workspace_bytes(2, vocab, d), dtype=torch.uint8, device="cuda")
        mp.mp_embedding_bwd(2, vocab, d, i32([-1, vocab]), place(np.ones((2, d)), 0), 1.0, dw, add=place(second, other), st=st, ws=ws)
        assert np.array_equal(bits(dw), half_bits(second)) and mp.scale_state_read(st).found_inf == int(bad is not None)
        if bad is not None:
            second.reshape(-1)[bad] = 1


def test_no_rows():
    dw, ws = torch.full((5, 8), 7.0, dtype=torch.float16, device="cuda"), torch.empty(1024, dtype=torch.uint8, device="cuda")
    mp.mp_embedding_bwd(0, 5, 8, None, None, 1.0, dw, ws=ws)
    assert torch.all(dw == 0)
    mp.mp_embedding_fwd(0, 5, 8, None, dw, 1.0, None)


@pytest.mark.parametrize("d", [8, 9])
def test_overflow_is_flagged_and_kept(d):
    """A sum beyond fp16 is an infinity in its own row and sets the flag; a clean gradient does not.  A sum over several chunks, and
    an infinite second gradient of an absent word, too."""
    st, ws = mp.scale_state_alloc(), torch.empty(mp.mp_embedding_bwd_workspace_bytes(300, 7, d), dtype=torch.uint8, device="cuda")
    for rows, value, add, want in ((4, 1.0, None, 0), (4, 30000.0, None, 1), (300, 300.0, None, 1), (4, 1.0, 1.0, 0), (4, 1.0, np.inf, 1)):
        mp.mp_scale_state_init(st, ML.MP_SCALE_BACKOFF, 2.0 ** 15, 10)
        dw, tok = empty16(7, d), i32(np.full(rows, 3))
        second = None if add is None else torch.zeros(7, d, dtype=torch.float16, device="cuda")
        if add is not None:
            second[6, d - 1] = add
        mp.mp_embedding_bwd(rows, 7, d, tok, torch.full((rows, d), value, dtype=torch.float16, device="cuda"), 1.0, dw, add=second, st=st, ws=ws)
        assert mp.scale_state_read(st).found_inf == want, (rows, value, add)
        assert torch.all(torch.isfinite(dw[[0, 1, 2, 4, 5]]))
        assert torch.all(torch.isinf(dw[3])) == (value * rows > 65519)


def test_captured_and_replayed_with_other_tokens():
    rows, vocab, d = 3000, 500, 64
    r = np.random.default_rng(1)
    dy, w, tokens = h16(S16(r.standard_normal((rows, d)))), h16(S16(r.standard_normal((vocab, d)))), i32(np.zeros(rows))
    out = [[empty16(rows, d), empty16(vocab, d), torch.empty(mp.mp_embedding_bwd_workspace_bytes(rows, vocab, d), dtype=torch.uint8, device="cuda")]
           for _ in range(2)]

    def both(o):
        mp.mp_embedding_fwd(rows, vocab, d, tokens, w, 2.0, o[0])
        mp.mp_embedding_bwd(rows, vocab, d, tokens, dy, 2.0, o[1], ws=o[2])
    both(out[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out[0])
    for kind in ("zipf", "same", "pads", "spread"):
        tokens.copy_(i32(tokens_of(kind, rows, vocab, r)))
        graph.replay()
        both(out[1])
        torch.cuda.synchronize()
        assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]), kind

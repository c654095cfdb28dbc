"""Masked attention through the C ABI against the oracle in 64 bits, element by element.

Tolerances are sums of the roundings that the calls state, each at most half a step (fp16 2^-11, fp32 2^-24 of a value):
  scores   E = (d + 16) 2^-24 alpha sum |q k|  (fp32 sums and their scaling, in any order) + 2^-21 cap (the capped score: 1 - 2 / (..)
           and its two hardware functions) + 2^-23 |bias|, the largest over a row's keys
  ctx      2^-11 |ctx| (stored) + (2^-11 + 2 E + n 2^-24) sum p |v|  (probabilities rounded as operands; a score's error shifts p and
           the sum; fp32 sums over n keys) + 2^-24 sum |v| (those below fp16's normal range, over a sum of at least 1) + 2^-25
  ds       (2^-11 + 4 E + 2^-20) |ds| + 2^-25 + p (d 2^-24 sum |dctx v| + sum |dctx| (2^-11 |ctx| + the error of ctx))
           (+ 2^-20 p |dp - delta| where scores are capped: 1 - tanh^2)
  dq, dk   2^-11 |.| + alpha sum (error of ds + n 2^-24 |ds|) |k|, |q|;   dv   2^-11 |dv| + sum ((2^-11 + 4 E + 2^-20 + n 2^-24) p
           + 2^-35) |dctx|  (probabilities times 1024 as operands)
  lse      E + 2^-21 (1 + |lse|)
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from oracle import FP64, MIXED
from oracle import layers as L
from gpu_util import *

S16 = MIXED.store


def documents(rows, seed, mean, front=0, back=0):
    """Starts of documents that fill [front, rows - back), an empty one among them."""
    r = np.random.default_rng(seed)
    at, out = front, [front]
    while at < rows - back:
        at = min(rows - back, at + int(r.integers(1, 2 * mean)))
        out.append(at)
    out.insert(len(out) // 2, out[len(out) // 2])
    return np.asarray(out, np.int32)


class Problem:
    """Inputs on both sides.  apart: q, k and v in matrices of their own with wider rows, else one fused projection."""

    def __init__(self, rows, heads, kv_heads, d, seed=0, keys=None, cap=0.0, bias=False, apart=False, spread=1.0):
        r = np.random.default_rng(seed)
        self.rows, self.keys, self.h, self.g, self.d = rows, rows if keys is None else keys, heads, kv_heads, d
        self.cap, self.slopes = cap, np.float32(2.0 ** -(1 + np.arange(heads))) if bias else None
        n = lambda *s: S16(r.standard_normal(s))  # noqa: E731
        self.q, self.k, self.v = S16(spread * n(rows, heads * d)), n(self.keys, kv_heads * d), n(self.keys, kv_heads * d)
        self.do = S16(0.5 * n(rows, heads * d))
        self.alpha = float(np.float32(1.0 / np.sqrt(d)))
        self.apart = apart or self.keys != rows
        w, wk = heads * d, kv_heads * d

        def place(x, extra):
            t = torch.full((x.shape[0], x.shape[1] + extra), float("nan"), dtype=torch.float16, device="cuda")
            t[:, :x.shape[1]] = h16(x)
            return t
        if self.apart:
            self.dev = [place(self.q, 8), place(self.k, 16), place(self.v, 24)]
            ld = [w + 8, wk + 16, wk + 24]
            self.dq, self.dk, self.dv = (torch.full((n_, m), 7.0, dtype=torch.float16, device="cuda") for n_, m in
                                         ((rows, w + 16), (self.keys, wk), (self.keys, wk + 8)))
            ld_d = [w + 16, wk, wk + 8]
        else:
            x = h16(np.concatenate([self.q, self.k, self.v], 1))
            self.dev, ld = [x, x[:, w:], x[:, w + wk:]], [w + 2 * wk] * 3
            y = torch.full((rows, w + 2 * wk), 7.0, dtype=torch.float16, device="cuda")
            self.dq, self.dk, self.dv, ld_d = y, y[:, w:], y[:, w + wk:], [w + 2 * wk] * 3
        self.ddo = place(self.do, 8)
        self.ctx = torch.full((rows, w + 8), 7.0, dtype=torch.float16, device="cuda")
        self.lse = torch.full((heads, rows), 7.0, device="cuda")
        self.desc = mp.attn_desc(rows, self.keys, heads, kv_heads, d, *ld, w + 8, self.alpha, cap, *ld_d, w + 8)
        self.mask = torch.empty(mp.mp_attention_mask_bytes(rows), dtype=torch.uint8, device="cuda")
        self.ws = torch.empty(mp.mp_attention_masked_bwd_workspace_bytes(self.desc), dtype=torch.uint8, device="cuda")
        self.dslopes = f32(self.slopes) if bias else None

    def docs(self, start, causal=False, prefix=None, window=0):
        self.lo, self.hi = L.attention_ranges(self.rows, start, causal, prefix, window)
        self.keep = i32(start), None if prefix is None else i32(prefix)
        mp.mp_attention_mask_docs(self.rows, len(start) - 1, self.keep[0], self.mask, self.keep[1], causal, window)
        return self

    def ranges(self, lo, hi):
        self.lo, self.hi = np.maximum(lo, 0), np.minimum(hi, self.keys)
        mp.mp_attention_mask_ranges(self.rows, self.keys, i32(lo), i32(hi), self.mask)
        return self

    def run(self):
        mp.mp_attention_masked_fwd(self.desc, self.mask, *self.dev, self.dslopes, self.ctx, self.lse)
        mp.mp_attention_masked_bwd(self.desc, self.mask, *self.dev, self.dslopes, self.ctx, self.lse, self.ddo, self.dq, self.dk, self.dv, self.ws)
        return self

    def results(self):
        w, wk = self.h * self.d, self.g * self.d
        return dict(ctx=self.ctx[:, :w], lse=self.lse, dq=self.dq[:, :w], dk=self.dk[:, :wk], dv=self.dv[:, :wk])

    def check(self, what=""):
        f8 = lambda x: np.asarray(x, np.float64)  # noqa: E731
        q, k, v, do = f8(self.q), f8(self.k), f8(self.v), f8(self.do)
        ctx, c = L.masked_attention_fwd(FP64, q, k, v, self.lo, self.hi, self.h, self.g, self.cap, self.slopes)
        dq, dk, dv = L.masked_attention_bwd(FP64, do, c)
        d, n, a = self.d, max(self.keys, self.rows), self.alpha
        cols = np.arange(self.keys)[None]
        seen = (cols >= self.lo[:, None]) & (cols < self.hi[:, None])
        q3, k3, v3, p, ds = np.abs(c["q"]), np.abs(c["k"]), np.abs(c["v"]), c["p"], np.abs(c["ds"])
        split = lambda t: t.reshape(t.shape[0], self.h, d).transpose(1, 0, 2)  # noqa: E731
        flat = lambda t: t.transpose(1, 0, 2).reshape(t.shape[1], t.shape[0] * t.shape[2])  # noqa: E731
        shared = lambda t: t.reshape(self.g, self.h // self.g, t.shape[1], d).sum(1)  # noqa: E731
        e = (d + 16) * 2.0 ** -24 * a * (q3 @ k3.transpose(0, 2, 1)) + 2.0 ** -21 * self.cap
        if self.slopes is not None:
            e = e + 2.0 ** -23 * f8(self.slopes)[:, None, None] * np.abs(np.arange(self.rows)[:, None] - cols)
        E = np.where(seen, e, 0).max(2, initial=0)[..., None]
        e_ctx = (2.0 ** -11 + 2 * E + n * 2.0 ** -24) * (p @ v3) + 2.0 ** -24 * (seen.astype(float) @ v3) + 2.0 ** -25
        do3, c3 = np.abs(split(do)), np.abs(split(ctx))
        e_ds = ((2.0 ** -11 + 4 * E + 2.0 ** -20) * ds + 2.0 ** -25 * seen +
                p * (d * 2.0 ** -24 * (do3 @ v3.transpose(0, 2, 1)) + (do3 * (2.0 ** -11 * c3 + e_ctx)).sum(-1, keepdims=True)))
        if self.cap:
            e_ds = e_ds + 2.0 ** -20 * p * np.abs(split(do) @ c["v"].transpose(0, 2, 1) - (split(do) * split(ctx)).sum(-1, keepdims=True))
        e_ds = e_ds + n * 2.0 ** -24 * ds
        e_p = (2.0 ** -11 + 4 * E + 2.0 ** -20 + n * 2.0 ** -24) * p + 2.0 ** -35 * seen
        T = lambda t: t.transpose(0, 2, 1)  # noqa: E731
        bounds = dict(ctx=flat(e_ctx), lse=E[..., 0] + 2.0 ** -21 * (1 + np.abs(np.where(np.isinf(c["lse"]), 0, c["lse"]))),
                      dq=flat(a * (e_ds @ k3)), dk=flat(shared(a * (T(e_ds) @ q3))), dv=flat(shared(T(e_p) @ do3)))
        for name, ref in dict(ctx=ctx, lse=c["lse"], dq=dq, dk=dk, dv=dv).items():
            got = self.results()[name].double().cpu().numpy()
            bound = bounds[name] + (0 if name == "lse" else 2.0 ** -11 * np.abs(ref) + 2.0 ** -25)
            assert np.array_equal(np.isinf(got), np.isinf(ref)), (what, name)
            fin = ~np.isinf(ref)
            worst = (np.abs(got - np.where(fin, ref, 0)) / bound)[fin].max(initial=0)
            assert worst <= 1, (what, name, worst)
        # beside the results nothing was written
        w, wk = self.h * d, self.g * d
        assert torch.all(self.ctx[:, w:] == 7)
        if self.apart:
            assert torch.all(self.dq[:, w:] == 7) and torch.all(self.dv[:, wk:] == 7)
        return self


@pytest.mark.parametrize("rows", [1, 2, 31, 33, 63, 64, 65, 127, 128, 129, 200, 385])
@pytest.mark.parametrize("mask", ["whole", "causal", "prefix", "window", "both window"])
def test_rows_around_the_tiles(rows, mask):
    p = Problem(rows, 2, 1, 64, seed=rows)
    kw = dict(whole={}, causal=dict(causal=True), prefix=dict(causal=True), window=dict(causal=True, window=max(1, rows // 3)),
              **{"both window": dict(window=1 + rows // 5)})[mask]
    start = documents(rows, rows, max(1, rows // 3))
    if mask == "prefix":
        kw["prefix"] = np.arange(len(start) - 1, dtype=np.int32) * 7 - 3
    p.docs(start, **kw).run().check(mask)


@pytest.mark.parametrize("d", [8, 16, 24, 32, 40, 64, 72, 96, 104, 128])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (3.0, False), (0.0, True), (5.0, True)])
def test_head_sizes_and_scores(d, cap, bias):
    p = Problem(150, 4, 2, d, seed=d, cap=cap, bias=bias, spread=3.0 if cap else 1.0, apart=d % 16 == 0)
    p.docs(documents(150, d, 40, front=3, back=9), causal=bool(d % 16)).run().check()


@pytest.mark.parametrize("cap,spread", [(0.01, 1.0), (0.5, 8.0), (1024.0, 30.0)])
def test_small_and_large_caps(cap, spread):
    Problem(150, 2, 1, 64, seed=5, cap=cap, spread=spread).docs([0, 60, 150], causal=True).run().check()


@pytest.mark.parametrize("heads,kv", [(1, 1), (5, 5), (6, 2), (8, 1), (16, 4)])
def test_head_layouts(heads, kv):
    Problem(170, heads, kv, 64, seed=heads).docs([0, 100, 170], causal=True).run().check()
    Problem(70, heads, kv, 128, seed=heads, apart=True).docs([0, 1, 70]).run().check()


@pytest.mark.parametrize("rows,keys", [(1, 300), (300, 1), (70, 200), (129, 64), (5, 0), (64, 65)])
def test_intervals_of_other_keys(rows, keys):
    """Queries over keys of another length (a decoder over an encoder's states), intervals of any kind, some empty, turned round or
    out of range; keys that nobody sees get zero gradients."""
    r = np.random.default_rng(rows + keys)
    lo, hi = (r.integers(-5, keys + 6, rows) for _ in range(2))
    lo[0], hi[0] = 0, max(keys - 1, 0)
    p = Problem(rows, 4, 2, 32, seed=keys, keys=keys).ranges(lo, hi).run().check()
    unseen = np.ones(keys, bool)
    for a, b in zip(p.lo, p.hi):
        unseen[a:max(a, b)] = False
    for t in ("dk", "dv"):
        assert torch.all(p.results()[t][torch.from_numpy(unseen).cuda()] == 0)


@pytest.mark.parametrize("n_docs", [0, 1])
def test_rows_that_see_nothing(n_docs):
    """No document, or one that is empty: ctx 0, lse -inf, all gradients 0."""
    p = Problem(130, 2, 2, 64).docs(np.zeros(n_docs + 1, np.int32)).run()
    r = p.results()
    assert all(torch.all(r[k] == 0) for k in ("ctx", "dq", "dk", "dv")) and torch.all(r["lse"] == -np.inf)


@pytest.mark.parametrize("d,cap", [(64, 0.0), (128, 4.0)])
def test_longer_documents(d, cap):
    """Many tiles of keys: running maxima that move, statistics of long rows."""
    p = Problem(1500, 2, 1, d, seed=d, cap=cap, spread=4.0)
    p.docs([0, 1400, 1500], causal=True).run().check()
    p.docs([0, 700, 1499], window=300).run().check()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_hidden_is_not_felt(bad, d):
    """Rows of no document, other documents and later keys may hold NaN and infinities: every row that does not see them keeps its bits,
    and rows that do see them show it."""
    start = [4, 90, 200, 310]

    def run(spoil):
        p = Problem(320, 2, 1, d, seed=9)
        for which, rows in spoil.items():
            t = dict(q=p.dev[0][:, :p.h * d], k=p.dev[1][:, :d], v=p.dev[2][:, :d], do=p.ddo[:, :p.h * d])[which]
            t[rows] = bad
        return p.docs(start, causal=True).run().results()
    clean = run({})
    pads = torch.cat([torch.arange(0, 4), torch.arange(310, 320)]).cuda()
    got = run(dict(q=pads, k=pads, v=pads, do=pads))
    for k in clean:
        assert torch.equal(clean[k], got[k]), k
    # a whole document of it: the others do not feel it
    doc = torch.arange(90, 200).cuda()
    other = torch.tensor([r for r in range(320) if not 90 <= r < 200]).cuda()
    got = run(dict(q=doc, k=doc, v=doc, do=doc))
    for k in clean:
        a, b = (clean[k][:, other], got[k][:, other]) if k == "lse" else (clean[k][other], got[k][other])
        assert torch.equal(a, b), k
    # one key, that later rows of its document see: earlier rows keep what does not come from later ones
    for which in ("k", "v"):
        got = run({which: torch.tensor([150]).cuda()})
        early = torch.tensor([r for r in range(320) if not 150 <= r < 200]).cuda()
        for name in ("ctx", "dq"):
            assert torch.equal(clean[name][early], got[name][early]), (which, name)
        assert torch.equal(clean["lse"][:, early], got["lse"][:, early])
        if which == "v" or bad != bad:              # (an infinite key may be one that takes no part, or takes all)
            assert not torch.any(torch.isfinite(got["ctx"][150:200]).all(1))
    # a gradient row: it reaches its own dq and the keys it sees, and no other document's
    got = run(dict(do=torch.tensor([150]).cuda()))
    assert not torch.any(torch.isfinite(got["dq"][150])) and not torch.any(torch.isfinite(got["dv"][90:151]).all(1))
    assert torch.equal(clean["dv"][200:], got["dv"][200:]) and torch.equal(clean["dk"][:90], got["dk"][:90]) and torch.equal(clean["dv"][151:], got["dv"][151:])


def test_large_scores_and_one_sided_rows():
    """Scores of several hundred: one key takes a row; probabilities that underflow."""
    p = Problem(200, 2, 2, 64, seed=3, spread=60.0)
    p.docs([0, 200], causal=True).run().check()


def test_two_calls_give_the_same_bits_and_streams_do_not_mix():
    p = Problem(700, 8, 2, 64, seed=5).docs(documents(700, 5, 90), causal=True).run()
    first = {k: v.clone() for k, v in p.results().items()}
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        p.run()
    torch.cuda.current_stream().wait_stream(s)
    for k, v in p.results().items():
        assert torch.equal(first[k], v), k


def test_captured_and_replayed_with_other_documents():
    """One capture of mask, forward and backward; the documents are data, and each replay follows them.  Eager calls in between."""
    p, q = (Problem(300, 4, 2, 64, seed=6) for _ in range(2))
    start = i32([0, 300, 300, 300])
    p.docs([0, 300, 300, 300], causal=True).run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mp.mp_attention_mask_docs(300, 3, start, p.mask, causal=True)
        p.run()
    for s in ([0, 10, 200, 300], [5, 5, 6, 290], [0, 128, 256, 300], [0, 300, 300, 300]):
        start.copy_(i32(s))
        graph.replay()
        q.docs(s, causal=True).run()
        torch.cuda.synchronize()
        for k, v in p.results().items():
            assert torch.equal(v, q.results()[k]), (s, k)


@pytest.mark.parametrize("d,kv,cap,bias", [(32, 512, 0.0, False), (64, 256, 0.0, False), (64, 512, 5.0, True), (40, 256, 0.0, True), (96, 256, 3.0, False),
                                           (128, 256, 0.0, True)])
def test_as_many_workgroups_as_one_team_takes(d, kv, cap, bias):
    """1024 workgroups of queries (2 x 512 heads), 512 and more of keys: one team each, heads that share keys summed in registers."""
    p = Problem(129, 512, kv, d, seed=d, cap=cap, bias=bias, spread=2.0 if cap else 1.0)
    p.docs([0, 50, 50, 128], causal=d != 64).run().check()
    p.docs([2, 129], causal=True, window=40).run().check()


@pytest.mark.parametrize("rows,window", [(4224, 70), (4170, 0), (8193, 65)])
def test_more_than_64_tiles_of_queries(rows, window):
    """The tiles that see a key are found 64 at a time; their number is odd for some keys."""
    start = [0, rows] if window else np.concatenate([np.arange(0, rows, 100), [rows]])
    p = Problem(rows, 1, 1, 8, seed=rows).docs(start, causal=True, window=window).run()
    q, k, v = (torch.from_numpy(np.asarray(x, np.float64)).cuda() for x in (p.q, p.k, p.v))
    at = torch.arange(rows, device="cuda")
    seen = (at[None] >= i32(p.lo)[:, None]) & (at[None] < i32(p.hi)[:, None])
    prob = torch.softmax((p.alpha * q @ k.T).masked_fill(~seen, -np.inf), 1)
    do = torch.from_numpy(np.asarray(p.do, np.float64)).cuda()
    dp = do @ v.T
    ds = prob * (dp - (prob * dp).sum(1, keepdim=True))
    # (errors of a key's sums by the oracle's check: half a step of each of p, ds and of ctx in delta, all of the magnitudes' sums)
    r = p.results()
    for name, ref, mag in (("dk", p.alpha * ds.T @ q, p.alpha * (ds.abs() + prob * (do.abs() @ (prob @ v).abs().T).diagonal()[:, None]).T @ q.abs()),
                           ("dv", prob.T @ do, prob.T @ do.abs())):
        assert torch.all((r[name].double() - ref).abs() <= 2.0 ** -9 * mag + 2.0 ** -11 * ref.abs() + 2.0 ** -20), name


def test_offsets_beyond_32_bits():
    """Rows so far apart that elements lie beyond 2^31: the first and last rows of a long matrix against the same rows packed."""
    rows, ld = 40000, 65536                       # 2.6e9 elements
    big = torch.empty(rows, ld, dtype=torch.float16, device="cuda")
    r = np.random.default_rng(7)
    x = S16(r.standard_normal((rows, 3 * 8)))
    big[:, :24] = h16(x)
    small = Problem(rows, 1, 1, 8, apart=True)
    mask = torch.empty(mp.mp_attention_mask_bytes(rows), dtype=torch.uint8, device="cuda")
    mp.mp_attention_mask_docs(rows, 3, i32([0, 200, 39800, 40000]), mask, causal=True, window=50)
    outs = []
    for t, l in ((big, ld), (h16(x), 24)):
        desc = mp.attn_desc(rows, rows, 1, 1, 8, l, l, l, 8, 0.3)
        ctx, lse, d = empty16(rows, 8), empty32(1, rows), torch.empty_like(t)
        ws = torch.empty(mp.mp_attention_masked_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
        mp.mp_attention_masked_fwd(desc, mask, t, t[:, 8:], t[:, 16:], None, ctx, lse)
        mp.mp_attention_masked_bwd(desc, mask, t, t[:, 8:], t[:, 16:], None, ctx, lse, small.ddo[:, :8].contiguous(), d, d[:, 8:], d[:, 16:], ws)
        outs.append((ctx, lse, d[:, :24].clone()))
        del d
    for a, b in zip(*outs):
        assert torch.equal(a, b)

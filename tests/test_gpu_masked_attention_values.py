"""Masked attention at the ends of its numbers: infinities in visible places, gradients far below and above fp16's middle, masks made for
other keys; bounds as stated in test_gpu_masked_attention.py."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from oracle import MIXED
from gpu_util import *
from test_gpu_masked_attention import Problem

S16 = MIXED.store


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("d,bias,heads", [(64, False, 2), (128, False, 2), (64, True, 2), (40, False, 512)])
@pytest.mark.parametrize("causal", [False, True])
def test_what_is_visible_and_not_finite_is_felt(bad, cap, d, bias, heads, causal):
    """One element of one key, or of one query: every row that sees it has no finite ctx, lse or dq, in whole tiles and in others, whatever
    the sign of its scores and whether or not they are capped; the other rows keep their bits, and some dk shows it too."""
    start, at = [0, 300, 320], 70                  # queries 0 .. 255 see whole tiles of keys unless causal
    rows = torch.arange(320, device="cuda")

    def run(which):
        p = Problem(320, heads, heads // 2, d, seed=9, cap=cap, bias=bias)
        if which == "k":
            p.dev[1][at, 5] = bad
        if which == "q":
            p.dev[0][at, 5] = bad
        if which == "no sign":                     # the key's score is -inf (or +inf) for every query
            p.dev[0][:, 5] = 1.0
            p.dev[1][at, 5] = bad
        if which == "row":                         # a query all of whose scores have one sign
            p.dev[1][:, 5] = 1.0
            p.dev[0][at, 5] = bad
        return p.docs(start, causal=causal).run().results()
    clean = run(None)
    for which in ("k", "q", "no sign", "row"):
        got = run(which)
        see = (rows < 300) & ((rows >= at) if causal else (rows >= 0)) if which in ("k", "no sign") else rows == at
        for name in ("ctx", "dq"):
            assert not torch.any(torch.isfinite(got[name][see][:, :d])), (which, name)
        assert torch.all(torch.isnan(got["lse"][0, see])), which
        assert not torch.all(torch.isfinite(got["dk"][:300, :d])), which
        assert torch.all(torch.isfinite(got["dk"][300:])) and torch.all(torch.isfinite(got["dv"][300:]))
        assert torch.all(torch.isfinite(got["ctx"][~see][:, :d])) and torch.all(torch.isfinite(got["lse"][0, ~see])), which
        if which in ("k", "q"):                    # (the others have changed finite elements too)
            for name in ("ctx", "dq"):
                assert torch.equal(clean[name][~see], got[name][~see]), (which, name)
            assert torch.equal(clean["lse"][:, ~see], got["lse"][:, ~see])


def small_gradients(rows, heads, kv, d, size):
    """Many keys of almost even weight, queries and gradients that point one way: every ds = p (dp - delta) is near size / rows."""
    p = Problem(rows, heads, kv, d, seed=3, apart=True)
    r = np.random.default_rng(4)
    p.q, p.k, p.v = S16(1 + 0.1 * r.standard_normal(p.q.shape)), S16(0.02 * r.standard_normal(p.k.shape)), S16(r.standard_normal(p.v.shape))
    p.do = S16(size * (1 + 0.1 * r.standard_normal(p.do.shape)))
    for dev, host in zip(p.dev + [p.ddo], (p.q, p.k, p.v, p.do)):
        dev[:, :host.shape[1]] = h16(host)
    return p


@pytest.mark.parametrize("rows,heads,kv,d", [(4096, 2, 2, 64), (4096, 2, 1, 128), (4096, 64, 64, 8)])
def test_gradients_of_scores_below_the_end_of_fp16(rows, heads, kv, d):
    """ds near 2^-27, whose sums over 4096 queries fp16 has.  Rounded to fp16 times 2^10, a ds is off by 2^-11 of itself and 2^-35 where
    that is below fp16's normal range; delta by the rounding of ctx (2^-11 |ctx|) and its own of it; otherwise as the bounds of the
    masked attention tests, whose scores' error E is below 2^-20 here."""
    p = small_gradients(rows, heads, kv, d, 2.0 ** -15 / d ** 0.5).docs([0, rows]).run()
    got = p.results()
    T = lambda x, n: torch.from_numpy(np.asarray(x, np.float64)).cuda().view(-1, n, d).transpose(0, 1).contiguous()  # noqa: E731
    q, k, v, do = T(p.q, heads), T(p.k, kv), T(p.v, kv), T(p.do, heads)
    dk, mag = torch.zeros_like(k), torch.zeros_like(k)
    for h in range(heads):
        g = h // (heads // kv)
        pr = torch.softmax(p.alpha * (q[h] @ k[g].T.contiguous()), 1)
        ctx = pr @ v[g]
        ds = pr * (do[h] @ v[g].T.contiguous() - (do[h] * ctx).sum(1, keepdim=True))
        e = (2.0 ** -11 + 2.0 ** -17) * ds.abs() + 2.0 ** -35 + pr * ((do[h].abs() * (2.0 ** -10 * ctx.abs() + 2.0 ** -24)).sum(1, keepdim=True) + d * 2.0 ** -24 * (do[h].abs() @ v[g].abs().T.contiguous()))
        dq, bound = p.alpha * ds @ k[g], p.alpha * e @ k[g].abs()
        cols = slice(h * d, h * d + d)
        assert torch.all((got["dq"][:, cols].double() - dq).abs() <= bound + 2.0 ** -11 * dq.abs() + 2.0 ** -25)
        dk[g] += p.alpha * ds.T.contiguous() @ q[h]
        mag[g] += p.alpha * e.T.contiguous() @ q[h].abs()
        assert ds.abs().median() < 2.0 ** -25
    got_dk = got["dk"].double().view(rows, kv, d).transpose(0, 1)
    assert torch.all((got_dk - dk).abs() <= mag + 2.0 ** -11 * dk.abs() + 2.0 ** -25)
    assert torch.all(mag + 2.0 ** -25 <= 0.25 * dk.abs().amax((1, 2), keepdim=True))       # (what the bound would let pass)


@pytest.mark.parametrize("heads,kv,d", [(2, 1, 64), (2, 2, 128), (4, 1, 128), (512, 256, 40)])
@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_gradients_of_scores_above_64(heads, kv, d, cap):
    """Gradients so large that ds times 2^10 is beyond fp16, though ds is not: in some workgroups (keys and queries of one document) and
    not in others."""
    rows = 129 if heads > 4 else 400
    p = Problem(rows, heads, kv, d, seed=heads, cap=cap, spread=2.0, apart=True)
    p.do[: rows // 2] *= 256
    p.ddo[:, :p.do.shape[1]] = h16(p.do)
    p.docs([0, rows // 2, rows], causal=True).run().check()
    first = {k: v.clone() for k, v in p.results().items()}
    p.run()
    assert all(torch.equal(first[k], v) for k, v in p.results().items())


@pytest.mark.parametrize("d,heads", [(64, 2), (128, 2), (40, 512)])
@pytest.mark.parametrize("keys", [0, 1, 63, 64, 100, 130, 200, 299])
def test_a_mask_made_for_more_keys(d, heads, keys):
    """A mask of rows_q rows serves calls of fewer keys than it was made for: they see what of their intervals is there."""
    rows = 300
    p = Problem(rows, heads, heads // 2, d, seed=keys, keys=keys)
    r = np.random.default_rng(keys)
    lo = np.minimum(r.integers(0, 40, rows), 20) * (np.arange(rows) % 3 == 0)
    hi = np.full(rows, 300) - r.integers(0, 30, rows) * (np.arange(rows) >= 128)
    mp.mp_attention_mask_ranges(rows, 300, i32(lo), i32(hi), p.mask)
    p.lo, p.hi = lo, np.minimum(hi, keys)
    p.run().check()
    p.docs([0, rows]).lo[:] = 0                     # one whole document of 300 rows, whose mask is made from the document
    p.hi[:] = keys
    p.run().check()


@pytest.mark.parametrize("d,heads,rows", [(64, 2, 130), (128, 2, 130), (40, 512, 130)])
@pytest.mark.parametrize("cap", [0.02, 1.0])
def test_capped_scores_under_a_large_bias(d, heads, rows, cap):
    """Keys some thousands of rows away, whose bias is 10^3 to 10^5 caps: what the cap leaves of a gradient does not come out of their sum."""
    keys = 6000 if heads == 2 else 1500
    p = Problem(rows, heads, heads // 2, d, seed=d, keys=keys, cap=cap, bias=heads == 2, spread=cap)
    if heads > 2:
        p.slopes = np.float32(0.5 / (1 + np.arange(heads) % 7))
        p.dslopes = f32(p.slopes)
    lo = keys - 60 + np.arange(rows) % 50
    p.ranges(lo, lo + 1 + np.arange(rows) % 8).run().check()

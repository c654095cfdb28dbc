"""Pins of the oracle's masked attention, embedding and AdamW / 8-bit optimizer states (no GPU)."""
import numpy as np
import pytest
import torch

import mp_inputs as I
from oracle import FP32, FP64, MIXED
from oracle import layers as L
from oracle import optimizer as O


def _problem(seed, rows=23, keys=23, h=4, g=2, d=8):
    r = np.random.default_rng(seed)
    return r.standard_normal((rows, h * d)), r.standard_normal((keys, g * d)), r.standard_normal((keys, g * d)), r.standard_normal((rows, h * d))


def test_ranges_of_documents():
    start = [2, 5, 5, 11, 12]
    lo, hi = L.attention_ranges(14, start)
    assert list(zip(lo, hi)) == [(0, 0)] * 2 + [(2, 5)] * 3 + [(5, 11)] * 6 + [(11, 12)] + [(0, 0)] * 2
    lo, hi = L.attention_ranges(14, start, causal=True, prefix=[2, 9, 3, 0])
    assert list(zip(lo[2:12], hi[2:12])) == [(2, 4), (2, 4), (2, 5), (5, 8), (5, 8), (5, 8), (5, 9), (5, 10), (5, 11), (11, 12)]
    lo, hi = L.attention_ranges(14, start, causal=True, window=2)
    assert list(zip(lo[5:11], hi[5:11])) == [(5, 6), (5, 7), (6, 8), (7, 9), (8, 10), (9, 11)]
    lo, hi = L.attention_ranges(14, start, window=3)
    assert list(zip(lo[5:11], hi[5:11])) == [(5, 8), (5, 9), (5, 10), (6, 11), (7, 11), (8, 11)]


@pytest.mark.parametrize("cap,bias", [(0.0, False), (1.5, False), (0.0, True), (2.0, True)])
def test_masked_attention_against_autograd(cap, bias):
    """Values and gradients against torch's own differentiation of the formula in 64 bits."""
    h, g, d = 4, 2, 8
    q, k, v, do = _problem(1)
    lo, hi = L.attention_ranges(23, [1, 9, 10, 21], causal=True, prefix=[3, 0, 2])
    slopes = np.array([0.5, 0.25, 0.125, 0.0625]) if bias else None
    ctx, cache = L.masked_attention_fwd(FP64, q, k, v, lo, hi, h, g, cap, slopes)
    grads = L.masked_attention_bwd(FP64, do, cache)
    tq, tk, tv = (torch.tensor(x, dtype=torch.float64, requires_grad=True) for x in (q, k, v))
    outs = []
    for i in range(h):
        a, j = slice(i * d, i * d + d), slice(i // (h // g) * d, i // (h // g) * d + d)
        s = tq[:, a] @ tk[:, j].T / np.sqrt(d)
        s = cap * torch.tanh(s / cap) if cap else s
        if bias:
            s = s - slopes[i] * (torch.arange(23)[:, None] - torch.arange(23)[None]).abs()
        c = torch.arange(23)[None]
        hide = (c < torch.tensor(lo)[:, None]) | (c >= torch.tensor(hi)[:, None])
        p = torch.softmax(s.masked_fill(hide, -1e300), 1).masked_fill(hide, 0)
        outs.append(p @ tv[:, j])
    out = torch.cat(outs, 1)
    out.backward(torch.tensor(do))
    assert np.allclose(ctx, out.detach().numpy(), atol=1e-12)
    for got, ref in zip(grads, (tq, tk, tv)):
        assert np.allclose(got, ref.grad.numpy(), atol=1e-12)
    assert np.all(ctx[0] == 0) and np.all(ctx[21:] == 0) and np.all(np.isneginf(cache["lse"][:, 21:]))


def test_masked_attention_is_the_unmasked_one_where_everything_is_seen():
    """Against the encoder layers' attention, sequence by sequence."""
    r = np.random.default_rng(2)
    n_seq, s, h, d = 3, 7, 2, 4
    qkv, do = r.standard_normal((n_seq * s, 3 * h * d)), r.standard_normal((n_seq * s, h * d))
    ref, c0 = L.attention_fwd(FP64, qkv, n_seq, s, h)
    lo, hi = L.attention_ranges(n_seq * s, np.arange(n_seq + 1) * s)
    w = h * d
    ctx, c1 = L.masked_attention_fwd(FP64, qkv[:, :w], qkv[:, w:2 * w], qkv[:, 2 * w:], lo, hi, h, h)
    assert np.allclose(ctx, ref, atol=1e-13)
    assert np.allclose(np.concatenate(L.masked_attention_bwd(FP64, do, c1), 1), L.attention_bwd(FP64, do, c0), atol=1e-13)


def test_embedding_against_autograd():
    r = np.random.default_rng(3)
    w, tokens, dy = r.standard_normal((11, 5)), np.array([3, 0, 3, -1, 10, 11, 3]), r.standard_normal((7, 5))
    tw = torch.tensor(w, requires_grad=True)
    ok = torch.tensor((tokens >= 0) & (tokens < 11))
    y = torch.where(ok[:, None], 2.5 * tw[torch.tensor(np.where(ok, tokens, 0))], 0.0)
    y.backward(torch.tensor(dy))
    assert np.allclose(L.embedding_fwd(FP64, tokens, w, 2.5), y.detach().numpy())
    assert np.allclose(L.embedding_bwd(FP64, tokens, dy, 11, 2.5), tw.grad.numpy())


def test_adamw_against_torch():
    r = np.random.default_rng(4)
    w = r.standard_normal(37)
    p = torch.nn.Parameter(torch.tensor(w))
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    cfg = I.OptCfg(kind="adamw", lr=1e-2, beta2=0.99, weight_decay=0.1)
    st = O.ScaleState(scale=4.0)
    t = dict(w32=w.copy(), w16=w.copy(), m=np.zeros(37), v=np.zeros(37))
    for _ in range(7):
        g = r.standard_normal(37)
        p.grad = torch.tensor(g)
        opt.step()
        assert O.unscale_check_update(FP64, [dict(t, g16=g * 4.0)], cfg, st) == 0
        st.opt_step += 1
        assert np.allclose(t["w32"], p.detach().numpy(), rtol=0, atol=1e-13)


@pytest.mark.parametrize("P", [FP32, FP64])
def test_codes_are_fixed_points_and_nearest(P):
    """Encoding what codes stand for gives the codes back; any value is decoded to within half a step of its root, the largest of
    a block exactly (to a rounding), and a positive second moment never becomes 0."""
    r = np.random.default_rng(5)
    m8 = r.integers(-127, 128, 1000).astype(np.int8)
    v8 = r.integers(1, 256, 1000).astype(np.uint8)
    m8[::256], v8[::256] = 127, 255
    ms, vs = r.uniform(1e-6, 1e3, 4).astype(P.acc), r.uniform(1e-6, 1e3, 4).astype(P.acc)
    m, v = O.state8_decode(P, m8, ms, False), O.state8_decode(P, v8, vs, True)
    a, sa, b, sb = O.state8_encode(P, m, np.sqrt(v))
    assert np.array_equal(a, m8) and np.array_equal(b, v8) and np.allclose(sa, ms, rtol=1e-6) and np.allclose(sb, vs, rtol=1e-6)
    x, y = r.standard_normal(700) ** 3, r.standard_normal(700) ** 6
    a, sa, b, sb = O.state8_encode(P, x, np.sqrt(y))
    dx, dy = O.state8_decode(P, a, sa, False), O.state8_decode(P, b, sb, True)
    big = lambda s: np.repeat(np.asarray(s, np.float64), 256)[:700]  # noqa: E731
    assert np.all(np.abs(np.sqrt(np.abs(dx) / big(sa)) - np.sqrt(np.abs(x) / big(sa))) <= 0.5 / 127 + 1e-6)
    assert np.all(np.abs((dy / big(sb) ** 2) ** 0.25 - (y / big(sb) ** 2) ** 0.25) <= np.where(b == 1, 1.0, 0.5) / 255 + 1e-6)
    assert np.all((dy > 0) == (y > 0)) and np.all(np.sign(dx) * np.sign(x) >= 0)
    z = O.state8_encode(P, np.zeros(5), np.zeros(5))
    assert not any(np.any(t) for t in z)


def test_adam_in_8_bits_follows_adam():
    """The codes' error is a per cent of a moment, and so is the update's: over 50 steps of noisy gradients the masters stay within
    five per cent of the distance they have moved."""
    r = np.random.default_rng(6)
    w = r.standard_normal(600)
    a = dict(w32=w.copy(), w16=w.copy(), m=np.zeros(600), v=np.zeros(600))
    b = dict(w32=w.copy(), w16=w.copy(), m8=np.zeros(600, np.int8), v8=np.zeros(600, np.uint8), ms=np.zeros(3), vs=np.zeros(3))
    cfg, st = I.OptCfg(kind="adamw", lr=1e-2, weight_decay=0.01), O.ScaleState(scale=1.0)
    size = np.exp(r.standard_normal(600))
    for _ in range(50):
        g = size * (1 + r.standard_normal(600))
        O.unscale_check_update(FP64, [dict(a, g16=g)], cfg, st)
        O.unscale_check_update8(FP64, [dict(b, g16=g)], cfg, st)
        st.opt_step += 1
    assert np.linalg.norm(a["w32"] - b["w32"]) <= 0.05 * np.linalg.norm(a["w32"] - w)

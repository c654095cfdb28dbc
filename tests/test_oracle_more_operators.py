"""Pins of the oracle's head norms with rotation, token log probabilities and distillation (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import FP64, MIXED
from oracle import layers as L


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_norm_rope_against_autograd(norm, adjacent):
    r = np.random.default_rng(1)
    rows, heads, d, rot = 7, 3, 12, 8
    x, dy, g = r.standard_normal((rows, heads * d)), r.standard_normal((rows, heads * d)), r.standard_normal(d) if norm else None
    angles = r.integers(-50, 50, (rows, 1)) * r.random((1, rot // 2))
    y, cache = L.norm_rope_fwd(FP64, x, heads, g, 1e-3, angles, adjacent)
    dx, dg = L.norm_rope_bwd(FP64, dy, cache)
    tx = torch.tensor(x, requires_grad=True)
    tg = torch.tensor(np.ones(d) if g is None else g, requires_grad=True)
    n = tx.reshape(rows, heads, d)
    if norm:
        n = n / torch.sqrt((n ** 2).mean(-1, keepdim=True) + 1e-3) * tg
    at = np.arange(rot).reshape(-1, 2) if adjacent else np.arange(rot).reshape(2, -1).T
    z = torch.complex(n[..., at[:, 0]], n[..., at[:, 1]]) * torch.exp(1j * torch.tensor(angles))[:, None]
    out = n.clone()
    out[..., at[:, 0]], out[..., at[:, 1]] = z.real, z.imag
    out.reshape(rows, -1).backward(torch.tensor(dy))
    assert np.allclose(y, out.detach().numpy().reshape(rows, -1), atol=1e-13)
    assert np.allclose(dx, tx.grad.numpy(), atol=1e-12)
    assert dg is None if g is None else np.allclose(dg, tg.grad.numpy(), atol=1e-12)


def test_rotation_keeps_lengths_and_only_distances_count():
    r = np.random.default_rng(2)
    q, k = r.standard_normal((2, 1, 16))
    f = 10000.0 ** (-np.arange(8) / 8)
    at = lambda v, pos: L.norm_rope_fwd(FP64, v, 1, None, 0, pos * f[None])[0]  # noqa: E731
    assert np.isclose(np.linalg.norm(at(q, 1000.0)), np.linalg.norm(q))
    assert np.isclose((at(q, 1007.0) * at(k, 1000.0)).sum(), (at(q, 7.0) * at(k, 0.0)).sum())


def test_token_logprobs_against_torch():
    r = np.random.default_rng(3)
    x = MIXED.store(r.standard_normal((5, 9)) * 3).astype(np.float64)
    x[1, 2:5] = -np.inf
    x[2, :4] = [1.5, 1.5, -0.0, 0.0]
    x[3] = 0.25
    targets = np.array([3, 0, -1, 8, 9])
    logp, entropy, lse, ids, top = L.token_logprobs(FP64, x, targets, 0.5, 9)
    lp = torch.log_softmax(torch.tensor(x) * 0.5, 1).numpy()
    assert np.allclose(logp, [lp[0, 3], lp[1, 0], 0, lp[3, 8], 0]) and np.allclose(lse, torch.logsumexp(torch.tensor(x) * 0.5, 1).numpy())
    assert np.allclose(entropy, torch.special.entr(torch.tensor(np.exp(lp))).sum(1).numpy())
    assert list(ids[3]) == list(range(9)) and np.allclose(top, np.take_along_axis(lp, ids, 1))
    where = list(ids[2])
    assert where.index(0) + 1 == where.index(1) and where.index(2) + 1 == where.index(3) and sorted(where) == list(range(9))
    nan = L.token_logprobs(FP64, np.array([[0.0, np.nan, np.inf, -np.inf, np.nan]]), np.array([0]), 1.0, 5)
    assert list(nan[3][0]) == [1, 4, 2, 0, 3] and np.isnan(nan[0][0]) and np.isnan(nan[1][0])
    none = L.token_logprobs(FP64, np.full((1, 3), -np.inf), np.array([0]), 1.0, 3)
    assert np.isneginf(none[2][0]) and np.isnan(none[0][0]) and np.isnan(none[1][0])


@pytest.mark.parametrize("temperature", [1.0, 0.5])
def test_token_logprobs_gradient_against_autograd(temperature):
    r = np.random.default_rng(4)
    x, g, h = r.standard_normal((6, 11)), r.standard_normal(6), r.standard_normal(6)
    x[2, 3] = -np.inf
    targets = np.array([0, 4, 10, -1, 11, 7])
    got = L.token_logprobs_bwd(FP64, x, targets, 1 / temperature, g, h, 8.0)
    tx = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(tx / temperature, 1)
    total = sum(g[i] * lp[i, t] for i, t in enumerate(targets) if 0 <= t < 11)
    safe = torch.where(torch.isinf(lp), 0.0, lp)
    total = total - (torch.tensor(h)[:, None] * torch.exp(lp) * safe).sum()
    total.backward()
    want = 8.0 * tx.grad.numpy()
    assert np.allclose(got, np.nan_to_num(want), atol=1e-12)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("hard", [0.0, 0.3])
@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_distillation_against_autograd(tail, hard, temperature):
    r = np.random.default_rng(5)
    rows, vocab, k = 6, 13, 4
    x, t = r.standard_normal((rows, vocab)), torch.log_softmax(torch.tensor(r.standard_normal((rows, vocab)) * 2), 1).numpy()
    ids = np.argsort(-t, 1)[:, :k]
    teacher = np.take_along_axis(t, ids, 1)
    ids[1, 2:] = -1                                                       # a list that ends early
    ids[2] = [-1, 13, 20, -5]                                             # none
    ids[3] = [4, 4, 7, 4]                                                 # one class three times
    teacher[3] = np.log([0.1, 0.2, 0.3, 0.15])
    targets = np.array([0, 1, 2, 4, -1, 13])
    loss, got = L.distill_scaled(FP64, x, ids, teacher, 16.0, 1 / temperature, 1.7, hard, targets, tail)
    tx = torch.tensor(x, requires_grad=True)
    total = 0
    for i in range(rows):
        q = torch.zeros(vocab, dtype=torch.float64)
        for j, v in zip(ids[i], teacher[i]):
            if 0 <= j < vocab:
                q[j] += np.exp(v)
        p = torch.softmax(tx[i] / temperature, 0)
        if q.sum() > 0:
            if not tail:
                q = q / q.sum()
            named = torch.tensor(np.isin(np.arange(vocab), ids[i]))
            kl = (q[named] * (q[named].log() - p[named].log())).sum()
            if tail:
                kl = kl + (1 - q.sum()) * ((1 - q.sum()).log() - p[~named].sum().log())
            total = total + 1.7 * kl
        if 0 <= targets[i] < vocab:
            total = total - hard * torch.log_softmax(tx[i], 0)[targets[i]]
    (total / rows * 16.0).backward()
    assert np.isclose(loss, float(total.detach()) / rows) and np.allclose(got, tx.grad.numpy(), atol=1e-12)


def test_distillation_from_oneself_costs_nothing():
    r = np.random.default_rng(6)
    x = r.standard_normal((3, 8))
    lp = torch.log_softmax(torch.tensor(x), 1).numpy()
    for k, tail in ((3, True), (8, True), (8, False)):                    # (all eight listed: nothing is left to the others)
        ids = np.argsort(-lp, 1)[:, :k]
        loss, d = L.distill_scaled(FP64, x, ids, np.take_along_axis(lp, ids, 1), 1.0, tail=tail)
        assert abs(loss) < 1e-14 and np.abs(d).max() < 1e-15

"""Moments in 8 bits over thousands of steps, as iterations are configured (state_bits = 8), against moments in 32 bits (no GPU).

Rounding without bias makes each step's code a martingale's increment: its variance is at most D^2 / 4, D the distance of two codes
(4 v / q of a second moment), and the moment forgets it at 1 - beta2 a step, so a v of code q has a relative variance of at most
(4 / q)^2 / 4 / (2 (1 - beta2)), and the mean of n of them a standard deviation of (4 / q) / 2 / sqrt(2 (1 - beta2) n).  Bounds are five of
these (and 1 % for sums in fp32 and what a block's moving scale adds)."""
import numpy as np
import pytest

import mp_inputs as I
from oracle import FP32
from oracle import optimizer as O

N = 1024


class Run:
    """Both kinds side by side, gradients N(0, 1), those of every other element times `size(step)`."""

    def __init__(self, beta2, seed=0):
        z = lambda kind, n=N: np.zeros(n, kind)  # noqa: E731
        self.r, self.st = np.random.default_rng(seed), O.ScaleState(scale=1.0)
        self.cfg = I.OptCfg(kind="adamw", lr=1e-3, beta2=beta2, state_bits=8)
        self.a = dict(w32=z(np.float32), w16=z(np.float32), m=z(np.float32), v=z(np.float32))
        self.b = dict(w32=z(np.float32), w16=z(np.float32), m8=z(np.int8), v8=z(np.uint8), ms=z(np.float32, N // 256), vs=z(np.float32, N // 256))
        self.half = np.arange(N) % 2 == 1

    def steps(self, n, size):
        for _ in range(n):
            g = self.r.standard_normal(N).astype(np.float32)
            g[self.half] *= np.float32(size)
            O.unscale_check_update(FP32, [dict(self.a, g16=g)], self.cfg, self.st)
            O.unscale_check_update8(FP32, [dict(self.b, g16=g)], self.cfg, self.st)
            self.st.opt_step += 1
        return self

    def ratio(self, which):
        """Mean v of 8 bits over that of 32, and the bound on its distance from 1."""
        v, code = O.state8_decode(FP32, self.b["v8"], self.b["vs"], True)[which], np.median(self.b["v8"][which])
        n = int(np.count_nonzero(which))
        return v.mean() / self.a["v"][which].mean(), 5 * (4 / code) / 2 / np.sqrt(2 * (1 - self.cfg.beta2) * n) + 0.01


def test_steady_gradients():
    run = Run(0.999).steps(4000, 1.0)
    ratio, bound = run.ratio(np.ones(N, bool))
    assert bound <= 0.1 and abs(ratio - 1) <= bound


def test_gradients_that_become_smaller():
    """Half a block's gradients a tenth from step 1500 on: their second moments come down with the 32-bit ones."""
    run = Run(0.999).steps(1500, 1.0).steps(5000, 0.1)
    for which in (run.half, ~run.half):
        ratio, bound = run.ratio(which)
        assert bound <= 0.3 and abs(ratio - 1) <= bound, (ratio, bound)


def test_weights_whose_gradients_become_zero_stop():
    """From step 500 on half a block has none.  A first moment m0 then moves its weight by 10 m0 in all; each of its steps' rounding has
    a variance of at most m sm / 127^2 (codes of m lie 2 sqrt(m sm) / 127 apart), ten times over: 10 sqrt(10 sm m0) / 127, which five
    times is below half of 10 m0 where m0 >= sm / 16.  So medians over the elements agree to that half."""
    run = Run(0.99).steps(500, 1.0)
    at = run.a["w32"].copy(), run.b["w32"].copy()
    m0 = np.abs(run.a["m"][run.half])
    assert np.median(m0) >= np.abs(run.a["m"]).max() / 16
    run.steps(1000, 0.0)
    moved = run.b["w32"].copy()
    run.steps(2000, 0.0)
    a, b = (np.median(np.abs(x - y)[run.half]) for x, y in ((run.a["w32"], at[0]), (run.b["w32"], at[1])))
    assert abs(b - a) <= 0.5 * a
    assert np.array_equal(run.b["w32"][run.half], moved[run.half])          # and no further


@pytest.mark.parametrize("top", [1.0, 3e-7])
def test_codes_are_the_value_in_the_mean(top):
    """A value's codes over many steps: their mean is the value to five deviations of at most half a step of the code each; the block's
    largest and zero are always themselves, and a second moment's code is never 0 unless it is."""
    r, steps = np.random.default_rng(1), 4000
    m, root = np.zeros(256), np.zeros(256)
    m[:250] = top * r.uniform(-1, 1, 250) ** 3
    root[:250] = top * np.abs(r.uniform(0.01, 1, 250)) ** 2
    m[17], root[18] = -top, top
    m, root = m.astype(np.float32), root.astype(np.float32)
    sums = np.zeros((2, 256))
    for t in range(1, steps + 1):
        m8, ms, v8, vs = O.state8_encode_unbiased(FP32, m, root, t)
        assert m8[17] == -127 and v8[18] == 255 and not m8[250:].any() and not v8[250:].any() and v8[:250].min() >= 1
        dm, dv = O.state8_decode(FP32, m8, ms, False), O.state8_decode(FP32, v8, vs, True)
        assert np.all(np.abs(np.abs(m8) - np.sqrt(np.abs(m) / top) * 127) <= 1.001) and np.all(np.abs(v8 - np.sqrt(root / top) * 255) <= 1.001)
        sums += dm, dv
    q, k = np.floor(np.sqrt(np.abs(m) / top) * 127), np.floor(np.sqrt(root / top) * 255)
    for got, want, step in ((sums[0], m, (2 * q + 1) / 127 ** 2 * top), (sums[1], root.astype(np.float64) ** 2, ((k + 1) ** 4 - k ** 4) / 255 ** 4 * top ** 2)):
        assert np.all(np.abs(got / steps - want) <= 5 * 0.5 * step / np.sqrt(steps) + 1e-5 * np.abs(want))


def test_what_rounds_is_even_and_does_not_repeat():
    """Means, and correlations from step to step, between neighbours, between m's and v's and between blocks: 0 to five deviations."""
    ms, vs = np.array([1e-3, 0.37, 2.0], np.float32), np.array([2e-3, 1.1, 2.0], np.float32)
    u, v = (np.array(x) for x in zip(*(O.state8_uniforms(ms, vs, t) for t in range(1, 3001))))
    c = lambda a, b: abs(((a - 0.5) * (b - 0.5)).mean(dtype=np.float64)) * 12 * np.sqrt(a.size)  # noqa: E731
    for x in (u, v):
        assert 0 < x.min() and x.max() < 1 and abs(x.mean(dtype=np.float64) - 0.5) * np.sqrt(12 * x.size) <= 5
        assert c(x[1:], x[:-1]) <= 5 and c(x[2:], x[:-2]) <= 5 and c(x[:, :, 1:], x[:, :, :-1]) <= 5 and c(x[:, 0], x[:, 1]) <= 5
    assert c(u, v) <= 5 and c(u[1:], v[:-1]) <= 5

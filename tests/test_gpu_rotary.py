"""Norms of queries and keys with the rotation by position: values and gradients against 64 bits, layouts, axes, far positions, in place,
captured, on other streams."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import _lib as ML
from oracle import FP64
from oracle import layers as L
from gpu_util import *

EPS = 1e-6


class Problem:
    """Queries and keys as columns of one projection [q | k | v], positions, weights, and everything in 64 bits."""

    def __init__(self, seed, rows, heads, kv, d, rot=None, axis=None, adjacent=False, norm=True, far=0, scale=1.0):
        r = np.random.default_rng(seed)
        self.rows, self.heads, self.kv, self.d, self.rot, self.norm, self.adjacent = rows, heads, kv, d, rot or d, norm, adjacent
        n = self.rot // 2
        self.axis = [0] * n if axis is None else axis
        axes = max(self.axis) + 1
        self.pos = (r.integers(-20, 4000, (axes, rows)) + far).astype(np.int32)
        self.freqs = 10000.0 ** (-np.arange(n) / n)
        self.qkv, self.dy = (r.standard_normal((rows, (heads + 2 * kv) * d)) * scale).astype(np.float16), (r.standard_normal((rows, (heads + kv) * d)) / 4).astype(np.float16)
        self.g = [(1 + 0.2 * r.standard_normal(d)).astype(np.float16) if norm else None for _ in range(2)]
        self.angles = np.stack([self.pos[a].astype(np.float64) * f for a, f in zip(self.axis, self.freqs)], 1)
        ld = (heads + 2 * kv) * d
        self.desc = mp.rope_desc(rows, heads, kv, d, rot=rot, n_axes=axes, axis=self.axis, adjacent=adjacent, eps=EPS, ld_q=ld, ld_k=ld, ld_yq=(heads + kv) * d,
                                 ld_yk=(heads + kv) * d, ld_dq=(heads + kv) * d, ld_dk=(heads + kv) * d)
        dev = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
        self.t = dict(x=dev(self.qkv), dy=dev(self.dy), gq=dev(self.g[0]), gk=dev(self.g[1]), pos=dev(self.pos), freqs=dev(self.freqs))

    def forward(self, y=None, x=None, desc=None):
        t, kq = self.t, self.heads * self.d
        x = t["x"] if x is None else x
        y = empty16(self.rows, (self.heads + self.kv) * self.d) if y is None else y
        mp.mp_qk_norm_rope_fwd(desc or self.desc, x, x[:, kq:], t["gq"], t["gk"], t["pos"], t["freqs"], y, y[:, kq:])
        return y

    def backward(self, d=None, dy=None, st=None, ws=None):
        t, kq = self.t, self.heads * self.d
        dy = t["dy"] if dy is None else dy
        d = empty16(*dy.shape) if d is None else d
        dg = [empty16(self.d) for _ in range(2)] if self.norm else [None, None]
        if ws is None:
            ws = torch.full((mp.mp_qk_norm_rope_bwd_workspace_bytes(self.desc) // 4 + 1,), float("nan"), device="cuda")
        mp.mp_qk_norm_rope_bwd(self.desc, t["x"], t["x"][:, kq:], t["gq"], t["gk"], t["pos"], t["freqs"], dy, dy[:, kq:], d, d[:, kq:], *dg, st=st, ws=ws)
        return (d, *dg)

    def exact(self):
        """(y, dx, dgq, dgk) and what their errors are measured by, each in 64 bits."""
        kq, ke = self.heads * self.d, (self.heads + self.kv) * self.d
        out = []
        for h, a, e, g in ((self.heads, 0, kq, self.g[0]), (self.kv, kq, ke, self.g[1])):
            x, dy, g = self.qkv[:, a:e].astype(np.float64), self.dy[:, a:e].astype(np.float64), None if g is None else g.astype(np.float64)
            y, c = L.norm_rope_fwd(FP64, x, h, g, EPS, self.angles, self.adjacent)
            dx, dg = L.norm_rope_bwd(FP64, dy, c)
            ones = np.ones_like(self.angles)
            # both members of a pair, taken absolutely
            pair = lambda v: np.abs(_pairs(np.abs(v.reshape(self.rows, h, self.d)), 2 * ones.shape[1], self.adjacent)).reshape(self.rows, -1)  # noqa: E731
            n = x if g is None else (c["x"] * c["r"] * g).reshape(self.rows, -1)
            sy, u = pair(n), pair(dy)
            if g is None:
                sdx, sdg = u, None
            else:
                u3, hat = u.reshape(c["x"].shape), np.abs(c["x"] * c["r"])
                v = u3 * np.abs(g)
                sdx = (c["r"] * (v + hat * (v * hat).mean(-1, keepdims=True))).reshape(self.rows, -1)
                sdg = (u3 * hat).sum((0, 1))
            out.append((y, dx, dg, sy, sdx, sdg))
        cat = lambda i: np.concatenate([o[i] for o in out], 1)  # noqa: E731
        return dict(y=cat(0), dx=cat(1), dg=[o[2] for o in out], sy=cat(3), sdx=cat(4), sdg=[o[5] for o in out])


def _pairs(n, rot, adjacent):
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
    s = n.copy()
    s[..., a] = s[..., b] = n[..., a] + n[..., b]
    return s


def close(got, want, size, roundings, what=""):
    """Within half a step of fp16 (2^-11 of the value, 2^-25 among subnormals) and so many roundings of fp32 of what was summed."""
    err = np.abs(np32(got).astype(np.float64) - want) - (2.0 ** -11 * np.abs(want) + 2.0 ** -25 + roundings * 2.0 ** -24 * size)
    assert err.max(initial=-1) <= 0, (what, err.max(), np.unravel_index(err.argmax(), err.shape))


def check(p, y=None, grads=None):
    """Roundings of 2^-24.  A value: sum of squares 16 a lane and 6 over lanes, halved by the root, 11; root, eps and mean 3; two products 2;
    an angle in revolutions rounded below 1/2, so 2 pi / 2 in radians, 3.2; sine and cosine 4; products and sum 2: 26.  An input gradient: the
    turn back 10; two norms' factors 2 x 14; mean of products 22 + 3; 6 products: 70.  A weight gradient: an item 26; up to 64 items a lane,
    6 over lanes, 4 waves, 64 workgroups: 170."""
    e = p.exact()
    if y is not None:
        close(y, e["y"], e["sy"], 26, "y")
    if grads is not None:
        close(grads[0], e["dx"], e["sdx"], 70, "dx")
        for got, want, size in zip(grads[1:], e["dg"], e["sdg"]):
            if want is not None:
                close(got, want, size, 170, "dg")


SHAPES = [dict(rows=1, heads=16, kv=4, d=128), dict(rows=37, heads=4, kv=4, d=32), dict(rows=300, heads=8, kv=2, d=64), dict(rows=61, heads=4, kv=4, d=80, rot=40),
          dict(rows=5, heads=3, kv=1, d=8, rot=4), dict(rows=130, heads=1, kv=1, d=24, rot=12), dict(rows=19, heads=2, kv=2, d=40), dict(rows=7, heads=2, kv=1, d=72),
          dict(rows=33, heads=5, kv=3, d=96, rot=64), dict(rows=2049, heads=2, kv=1, d=256), dict(rows=4, heads=2, kv=2, d=256, rot=252), dict(rows=3, heads=1, kv=1, d=248, rot=8),
          dict(rows=1100, heads=1, kv=2, d=16), dict(rows=2, heads=40, kv=8, d=128, rot=32)]


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(str(v) for v in s.values()))
def test_values_and_gradients(shape, norm, adjacent):
    p = Problem(1, norm=norm, adjacent=adjacent, **shape)
    check(p, p.forward(), p.backward())


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("rows", [2, 7, 8, 9, 255, 257, 513, 1000, 1025, 4097, 16384, 16385, 20011, 33000])
@pytest.mark.parametrize("heads", [dict(heads=2, kv=1, d=64), dict(heads=1, kv=1, d=40), dict(heads=1, kv=1, d=256)], ids=lambda s: f"d{s['d']}")
def test_blocks_of_tokens(norm, rows, heads):
    """Workgroups of 1 to 16 tokens, the last one of fewer; several blocks a workgroup beyond 16384 tokens (8192 of heads of 256)."""
    p = Problem(5, rows=rows, norm=norm, **heads)
    check(p, p.forward(), p.backward())


@pytest.mark.parametrize("axis", [[0, 1] * 16, [0] * 8 + [1] * 12 + [2] * 12, [3, 0, 2, 1] * 8])
@pytest.mark.parametrize("adjacent", [False, True])
def test_several_axes(axis, adjacent):
    p = Problem(2, 77, 4, 2, 64, axis=axis, adjacent=adjacent)
    check(p, p.forward(), p.backward())


@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 5000, -(1 << 31) + 30])
def test_far_positions(far):
    """pos freq in 64 bits is off by 2^-52 of up to 2^31, so 2^-21 a turn more at the last two: 8 roundings of 2^-24."""
    p = Problem(3, 50, 2, 2, 64, far=far)
    e = p.exact()
    close(p.forward(), e["y"], e["sy"], 26 + 8 * 6.3, "y")


@pytest.mark.parametrize("scale", [1e-4, 60.0])
def test_sizes_of_values(scale):
    p = Problem(4, 40, 3, 1, 64, scale=scale)
    check(p, p.forward(), p.backward())


def test_rows_of_zeros_and_non_finite_ones():
    p = Problem(5, 6, 2, 1, 32)
    p.qkv[1] = 0
    p.qkv[2, 5] = np.inf
    p.qkv[3, 40] = np.nan
    p.t["x"].copy_(torch.from_numpy(p.qkv))
    st = mp.scale_state_alloc()
    mp.mp_scale_state_init(st, ML.MP_SCALE_STATIC, 1.0, 1)
    y, (d, dgq, dgk) = np32(p.forward()), p.backward(st=st)
    assert np.all(y[1] == 0) and np.isnan(y[2, :32]).any() and np.isnan(y[3, 32:64]).all() and np.isfinite(np.delete(y, [2, 3], 0)).all()
    assert np.isfinite(y[2, 32:]).all() and np.isfinite(y[3, :32]).all()
    assert np.isfinite(np32(d)[[0, 1, 4, 5]]).all() and not np.isfinite(np32(dgq)).all()
    assert mp.scale_state_read(st).found_inf == 1


def test_flag_of_overflowing_weight_gradients():
    p = Problem(6, 64, 2, 1, 32)
    st = mp.scale_state_alloc()
    mp.mp_scale_state_init(st, ML.MP_SCALE_STATIC, 1.0, 1)
    p.backward(st=st)
    assert mp.scale_state_read(st).found_inf == 0
    p.t["dy"].copy_(torch.full_like(p.t["dy"], 60000.0))
    p.t["x"].copy_(torch.full_like(p.t["x"], 1.0))
    p.backward(st=st)
    assert mp.scale_state_read(st).found_inf == 1


@pytest.mark.parametrize("norm", [True, False])
def test_in_place(norm):
    p = Problem(7, 90, 4, 2, 64, norm=norm)
    y, grads = p.forward(), p.backward()
    dy = p.t["dy"].clone()
    in_place = p.backward(d=dy, dy=dy)
    assert all(a is None or torch.equal(a, b) for a, b in zip(grads, in_place))
    x = p.t["x"].clone()
    ld, kq = x.shape[1], p.heads * p.d
    desc = mp.rope_desc(p.rows, p.heads, p.kv, p.d, eps=EPS, ld_q=ld, ld_k=ld, ld_yq=ld, ld_yk=ld)
    p.forward(y=x, x=x, desc=desc)
    ke = kq + p.kv * p.d
    assert torch.equal(x[:, :ke], y) and torch.equal(x[:, ke:], p.t["x"][:, ke:])      # (values are left as they were)


def test_columns_and_rows_around_the_outputs_stay():
    p = Problem(8, 21, 2, 2, 32)
    ld, kq = 4 * 32 + 24, 64
    desc = mp.rope_desc(p.rows, 2, 2, 32, eps=EPS, ld_q=p.desc.ld_q, ld_k=p.desc.ld_k, ld_yq=ld, ld_yk=ld)
    out = torch.full((p.rows + 2, ld), 7.0, dtype=torch.float16, device="cuda")
    mp.mp_qk_norm_rope_fwd(desc, p.t["x"], p.t["x"][:, kq:], p.t["gq"], p.t["gk"], p.t["pos"], p.t["freqs"], out[1:, 8:], out[1:, 8 + kq:])
    assert torch.equal(out[1:-1, 8:8 + 128], p.forward())
    assert torch.all(out[0] == 7) and torch.all(out[-1] == 7) and torch.all(out[:, :8] == 7) and torch.all(out[:, 136:] == 7)


def test_same_bits_in_every_call_and_stream():
    p = Problem(9, 1500, 4, 2, 64)
    y, grads = p.forward(), p.backward()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        y2, grads2 = p.forward(), p.backward()
    y3 = p.forward()
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(y, y3) and all(torch.equal(a, b) for a, b in zip(grads, grads2))


def test_captured_and_replayed():
    p = Problem(10, 200, 4, 2, 64)
    y, d, ws = p.forward(), empty16(*p.t["dy"].shape), torch.empty(mp.mp_qk_norm_rope_bwd_workspace_bytes(p.desc), dtype=torch.uint8, device="cuda")
    out = p.backward(d=d, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(y=y)
        out = p.backward(d=d, ws=ws)
    r = np.random.default_rng(0)
    for k in range(4):
        p.t["x"].copy_(torch.from_numpy(r.standard_normal(p.qkv.shape).astype(np.float16)))
        p.t["pos"].copy_(torch.from_numpy(r.integers(0, 99999, p.pos.shape).astype(np.int32)))
        graph.replay()
        got = [x.clone() for x in (y, *out)]
        want = [p.forward(), *p.backward()]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_no_rows():
    p = Problem(11, 4, 2, 1, 32)
    desc = mp.rope_desc(0, 2, 1, 32)
    dg = [torch.ones(32, dtype=torch.float16, device="cuda") for _ in range(2)]
    ws = torch.empty(64, dtype=torch.uint8, device="cuda")
    mp.mp_qk_norm_rope_fwd(desc, None, None, p.t["gq"], p.t["gk"], None, None, None, None)
    mp.mp_qk_norm_rope_bwd(desc, None, None, p.t["gq"], p.t["gk"], None, None, None, None, None, None, *dg, ws=ws)
    assert all(torch.all(g == 0) for g in dg)


def test_more_than_2_31_elements():
    rows, ld = (1 << 20) + 3, 4096
    x = torch.zeros(rows, ld, dtype=torch.float16, device="cuda")
    p = Problem(12, 5, 1, 1, 64)
    some = [0, 1, rows // 2, rows - 2, rows - 1]
    pos = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for i, s in enumerate(some):
        x[s, :128] = p.t["x"][i, :128]
        pos[s] = int(p.pos[0, i])
    desc = mp.rope_desc(rows, 1, 1, 64, eps=EPS, ld_q=ld, ld_k=ld, ld_yq=ld, ld_yk=ld)
    mp.mp_qk_norm_rope_fwd(desc, x, x[:, 64:], p.t["gq"], p.t["gk"], pos, p.t["freqs"], x, x[:, 64:])
    assert torch.equal(x[some, :128], p.forward())

"""Codes of 8-bit moments rounded without bias, on the device against the oracle: bit by bit, as the stated operations are."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1805_10387_amd as mp
from paper_1805_10387_amd import _lib as ML
import mp_inputs as I
from oracle import MIXED
from oracle import optimizer as O
from gpu_util import *
from test_gpu_adamw import SIZES, same, state, tensors8, to_device

CODES = ("m8", "v8", "ms", "vs")


def opt(kind="adamw", wd=0.1):
    return I.OptCfg(kind=kind, lr=1e-3, weight_decay=wd, state_bits=8), mp.opt_cfg(kind, 1e-3, weight_decay=wd)


@pytest.mark.parametrize("kind", ["adam", "adamw"])
@pytest.mark.parametrize("step,wd,skew", [(0, 0.0, 0), (1, 1e-2, 0), (57, 0.1, 1), (100003, 0.3, 4)])
def test_codes_match_the_oracle(kind, step, wd, skew):
    host = tensors8(SIZES, step)
    dev, before = [to_device(t, skew) for t in host], [t["w32"].copy() for t in host]
    ocfg, cfg = opt(kind, wd)
    assert O.unscale_check_update8(MIXED, host, ocfg, O.ScaleState(scale=2.0 ** 7, opt_step=step)) == 0
    mp.mp_unscale_check_update8(mp.tensor_list8(dev), len(dev), cfg, state(2.0 ** 7, step), ML.MP_UPDATE_UNBIASED8)
    for h, d, w0 in zip(host, dev, before):
        assert all(same(d[k], h[k]) for k in CODES), h["w32"].size
        assert np.all(np.abs(np32(d["w32"]).astype(np.float64) - h["w32"]) <= 2.0 ** -22 * (np.abs(h["w32"]) + np.abs(h["w32"] - w0)))


def test_many_blocks_over_steps():
    """3 million codes of each kind and step, so that those next to a border are among them."""
    host = tensors8([3000000], 6)
    dev, (ocfg, cfg) = [to_device(host[0])], opt()
    r = np.random.default_rng(2)
    for step in range(4):
        host[0]["g16"][...] = MIXED.store(r.standard_normal(3000000))
        dev[0]["g16"].copy_(h16(host[0]["g16"]))
        O.unscale_check_update8(MIXED, host, ocfg, O.ScaleState(scale=2.0 ** 7, opt_step=step))
        mp.mp_unscale_check_update8(mp.tensor_list8(dev), 1, cfg, state(2.0 ** 7, step), ML.MP_UPDATE_UNBIASED8)
        assert all(same(dev[0][k], host[0][k]) for k in CODES), step


def test_blocks_of_zeros_of_tiny_moments_and_of_single_values():
    n = 256 * 6
    g = np.zeros(n)
    g[256:512], g[512:768], g[768], g[1024:1280:2] = 6e-8, 6e4, 1.0, -1.0
    host = [dict(g16=MIXED.store(g), w32=np.ones(n, np.float32), w16=np.ones(n, np.float32), m8=np.zeros(n, np.int8), v8=np.zeros(n, np.uint8),
                 ms=np.zeros(6, np.float32), vs=np.zeros(6, np.float32))]
    dev, (ocfg, cfg) = [to_device(host[0])], opt(wd=0.0)
    for step in range(12):
        O.unscale_check_update8(MIXED, host, ocfg, O.ScaleState(scale=2.0 ** 24, opt_step=step))
        mp.mp_unscale_check_update8(mp.tensor_list8(dev), 1, cfg, state(2.0 ** 24, step), ML.MP_UPDATE_UNBIASED8)
        assert all(same(dev[0][k], host[0][k]) for k in CODES), step
        assert np.all(np.isfinite(np32(dev[0]["w32"])))


def test_the_end_of_the_iteration_and_a_graph():
    """Captured with both flags, each replay is the oracle's next step; what overflowed is skipped, codes and all."""
    host = tensors8([5000, 300], 8)
    dev, st, counters = [to_device(t) for t in host], state(2.0 ** 7, 0), mp.update_counters_alloc()
    (ocfg, cfg), ost = opt(), O.ScaleState(scale=2.0 ** 7, growth_interval=3)
    lst = mp.tensor_list8(dev)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mp.mp_unscale_check_update8_end(lst, 2, cfg, st, counters, ML.MP_UPDATE_UNBIASED8 | ML.MP_UPDATE_PRECHECKED)
    r = np.random.default_rng(1)
    for step in range(6):
        for t, d in zip(host, dev):
            t["g16"][...] = MIXED.store(r.standard_normal(t["g16"].size))
            d["g16"].copy_(h16(t["g16"]))
        if step == 2:
            host[1]["g16"][7] = np.inf
            st[7:8].fill_(1)
        graph.replay()
        O.loss_scale_update(ost, O.unscale_check_update8(MIXED, host, ocfg, ost))
        s = mp.scale_state_read(st)
        assert (s.scale, s.opt_step, s.skipped_steps) == (ost.scale, ost.opt_step, ost.skipped_steps)
        for t, d in zip(host, dev):
            assert all(same(d[k], t[k]) for k in CODES), step


def test_the_flag_is_for_moments_in_8_bits():
    t = dict(g16=h16(np.ones(8)), w32=f32(np.ones(8)), w16=h16(np.ones(8)), m=f32(np.zeros(8)), v=f32(np.zeros(8)))
    with pytest.raises(mp.MPError, match="unknown flags"):
        mp.mp_unscale_check_update(mp.tensor_list([t]), 1, opt()[1], state(1.0, 0), ML.MP_UPDATE_UNBIASED8)

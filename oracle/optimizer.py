"""Optimizer wrapper and loss-scale policy of the oracle (test infrastructure only).

Section 3.2 of the paper: the wrapper takes the fp16 gradients, converts them
to fp32, hands them to an ordinary optimizer that updates the fp32 master
weights, and converts the updated masters back to fp16 for the next
iteration.  Section 3.1, item 1: the optimizer inspects the gradients every
iteration and sets the loss scale of the next one ("Backoff" policy; the
paper gives the name only - halve on overflow, skip that step, double after
`growth_interval` consecutive clean steps is the reading taken here).
Section 3.3: a weight-decay regulariser acts on the fp32 copy, its gradient
being added to the unscaled fp32 gradient.
"""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import Dict, List, Tuple

import numpy as np

from .numerics import Policy, half_bits


@dataclass
class ScaleState:
    mode: str = "backoff"            # "static" | "backoff"
    scale: float = 2.0 ** 15
    growth_interval: int = 10
    min_scale: float = 1.0
    max_scale: float = 2.0 ** 24
    good_steps: int = 0
    opt_step: int = 0                # t of Adam: counts applied steps only
    total_steps: int = 0
    skipped_steps: int = 0
    history: List[Tuple[float, int]] = field(default_factory=list)  # (scale used, found_inf)


def has_nonfinite(P: Policy, grads) -> bool:
    """True iff any stored gradient value is inf or NaN.  Under MIXED the test
    is on the binary16 encoding: exponent field all ones."""
    for g in grads:
        if P.half_storage:
            if np.any((half_bits(g) & 0x7C00) == 0x7C00):
                return True
        elif not np.all(np.isfinite(g)):
            return True
    return False


def unscale_check_update(P: Policy, tensors: List[Dict[str, np.ndarray]], opt, st: ScaleState) -> int:
    """One optimizer-wrapper call over every parameter tensor.

    `tensors` is a list of dicts with keys g16 (stored gradient, loss-scaled),
    w32 (master), w16 (stored copy), m, v (Adam moments; absent for SGD); the
    arrays are updated in place.  If any gradient holds inf/NaN nothing is
    touched and 1 is returned.  Otherwise, per element, in the arithmetic type:
        g   = g16 * (1/S)  [+ weight_decay * w32]
        SGD : w32 -= lr * g
        Adam: m = b1 m + (1-b1) g ; v = b2 v + (1-b2) g^2 ;  t = opt_step + 1
              w32 -= lr * (m / (1-b1^t)) / (sqrt(v / (1-b2^t)) + eps)
        AdamW: g without the decay;  w32 -= (lr weight_decay) w32;  then as Adam
        w16 = store(w32)
    Scalars (1-b1, 1-b2, bias corrections) are formed in double and cast.
    """
    if has_nonfinite(P, [t["g16"] for t in tensors]):
        return 1
    A = P.scalar
    inv_s = A(1) / A(st.scale)
    lr, wd = A(opt.lr), A(opt.weight_decay)
    if opt.kind in ("adam", "adamw"):
        t = st.opt_step + 1
        b1, b2, eps = A(opt.beta1), A(opt.beta2), A(opt.eps)
        omb1, omb2 = A(1.0 - opt.beta1), A(1.0 - opt.beta2)
        bc1, bc2 = A(1.0 - float(opt.beta1) ** t), A(1.0 - float(opt.beta2) ** t)
    for tn in tensors:
        g = tn["g16"] * inv_s
        if opt.kind == "adamw":
            tn["w32"][...] = tn["w32"] - A(float(opt.lr) * float(opt.weight_decay)) * tn["w32"]
        elif opt.weight_decay != 0.0:
            g = g + wd * tn["w32"]
        if opt.kind == "sgd":
            tn["w32"][...] = tn["w32"] - lr * g
        elif opt.kind in ("adam", "adamw"):
            tn["m"][...] = b1 * tn["m"] + omb1 * g
            tn["v"][...] = b2 * tn["v"] + omb2 * (g * g)
            mhat = tn["m"] / bc1
            vhat = tn["v"] / bc2
            tn["w32"][...] = tn["w32"] - lr * mhat / (np.sqrt(vhat) + eps)
        else:
            raise ValueError(opt.kind)
        tn["w16"][...] = P.store(tn["w32"])
    return 0


STATE8_BLOCK = 256


def _blocks(x, P: Policy):
    x = np.asarray(x, P.acc).reshape(-1)
    return np.concatenate([x, np.zeros(-x.size % STATE8_BLOCK, P.acc)]).reshape(-1, STATE8_BLOCK)


def state8_decode(P: Policy, codes, scales, second):
    """Values of 8-bit codes: m = sm q |q| / 127^2, and (second) v = (sv (q / 255)^2)^2; blocks of 256 elements share a scale."""
    q, A = _blocks(codes, P), P.scalar
    if second:
        out = np.square((q * q) * (np.asarray(scales, P.acc) * A(1 / 65025.0))[:, None])
    else:
        out = (q * np.abs(q)) * (np.asarray(scales, P.acc) * A(1 / 16129.0))[:, None]
    return out.reshape(-1)[:np.asarray(codes).size]


def state8_encode(P: Policy, m, root):
    """(m8, ms, v8, vs) of moments m and sqrt(v): scales are the blocks' largest |m| and sqrt(v) (0 up to 2^-100, codes 0), codes
    rounded to nearest even in sqrt(|m|) and in the root of sqrt(v), the latter at least 1 where v > 0."""
    A, n = P.scalar, np.asarray(m).size
    mb, rb = _blocks(m, P), _blocks(root, P)

    def fit(top, k):
        ok = top > 2.0 ** -100
        return np.where(ok, top, A(0)), np.where(ok, A(k) / np.where(ok, top, A(1)), A(0))[:, None]
    ms, mf = fit(np.abs(mb).max(1), 16129.0)
    vs, vf = fit(rb.max(1), 65025.0)
    qm = np.minimum(np.rint(np.sqrt(np.abs(mb) * mf)), 127) * np.sign(mb)
    qv = np.minimum(np.rint(np.sqrt(rb * vf)), 255)
    qv = np.where((rb > 0) & (vf > 0), np.maximum(qv, 1), qv)
    return qm.reshape(-1)[:n].astype(np.int8), ms, qv.reshape(-1)[:n].astype(np.uint8), vs


def state8_uniforms(ms, vs, step):
    """Two numbers in (0, 1) for each element of each block, 16 bits and a half: for m's codes and for v's.  They come from the block's
    new scales (their fp32 bits), the step and the element's place in the block, so that a tensor's place in a list or an arena does not
    matter.  The multipliers are odd words of the fractions of sqrt 2, 3, 5, 7 and of the golden ratio."""
    u32 = lambda x: np.asarray(x, np.float32).view(np.uint32)  # noqa: E731
    word, lane = np.uint32, np.arange(STATE8_BLOCK // 4, dtype=np.uint32)
    x = (u32(ms) + u32(vs) * word(0x9E3779B9) + word(step * 0xA54FF53B & 0xFFFFFFFF))[:, None] + lane * word(0x3C6EF373)
    x = (x ^ (x >> word(16))) * word(0x6A09E667)
    x = (x ^ (x >> word(15))) * word(0xBB67AE85)
    x = x ^ (x >> word(16))
    x = x[:, :, None] * np.array([0x6A09E667, 0xBB67AE85, 0x3C6EF373, 0xA54FF53B], np.uint32)
    x = (x ^ (x >> word(15))).reshape(-1, STATE8_BLOCK)
    return [(y.astype(np.float32) + np.float32(0.5)) * np.float32(2.0 ** -16) for y in (x & word(0xFFFF), x >> word(16))]


def state8_encode_unbiased(P: Policy, m, root, step):
    """As state8_encode, but a value between two codes takes the upper one as often as it is nearer to what that stands for, so that what
    the codes stand for is m and v in the mean (v's least code apart, which a v > 0 does not go below)."""
    A, n = P.scalar, np.asarray(m).size
    _, ms, _, vs = state8_encode(P, m, root)
    mb, rb = _blocks(m, P), _blocks(root, P)
    um, uv = (P.island(u) for u in state8_uniforms(ms, vs, step))
    fit = lambda s, k: np.where(s > 0, A(k) / np.where(s > 0, s, A(1)), A(0))[:, None]  # noqa: E731
    z, y = np.abs(mb) * fit(ms, 16129.0), rb * fit(vs, 65025.0)
    q = np.minimum(np.floor(np.sqrt(z)), A(126))                        # values go with q^2 ...
    qm = (q + ((z - q * q) - um * (2 * q + 1) > 0)) * np.sign(mb)
    q = np.minimum(np.floor(np.sqrt(y)), A(254))                        # ... and with q^4
    qv = q + ((y - q * q) * (y + q * q) - uv * ((2 * q + 1) * (2 * (q * (q + 1)) + 1)) > 0)
    qv = np.where((rb > 0) & (vs > 0)[:, None], np.maximum(qv, 1), qv)
    return qm.reshape(-1)[:n].astype(np.int8), ms, qv.reshape(-1)[:n].astype(np.uint8), vs


def unscale_check_update8(P: Policy, tensors: List[Dict[str, np.ndarray]], opt, st: ScaleState) -> int:
    """unscale_check_update with moments in 8 bits (keys m8, ms, v8, vs instead of m, v; opt.kind "adam" or "adamw"):
        m = b1 decode(m8) + (1-b1) g,  v = b2 decode(v8) + (1-b2) g^2,
        w32 -= ((lr / (1-b1^t)) m) / (sqrt(v) (1 / sqrt(1-b2^t)) + eps),  then the moments are encoded.
    opt.state_bits 8, as an iteration is configured with it, rounds the codes without bias, as iterations do; else to nearest."""
    if has_nonfinite(P, [t["g16"] for t in tensors]):
        return 1
    A, t = P.scalar, st.opt_step + 1
    inv_s, b1, b2 = A(1) / A(st.scale), float(opt.beta1), float(opt.beta2)
    rate, rbc2 = A(opt.lr / (1.0 - b1 ** t)), A(1.0 / np.sqrt(1.0 - b2 ** t))
    for tn in tensors:
        g, w = tn["g16"].reshape(-1) * inv_s, tn["w32"].reshape(-1)
        if opt.kind == "adamw":
            w = w - A(float(opt.lr) * float(opt.weight_decay)) * w
        elif opt.weight_decay != 0.0:
            g = g + A(opt.weight_decay) * w
        m = A(b1) * state8_decode(P, tn["m8"], tn["ms"], False) + A(1.0 - b1) * g
        v = A(b2) * state8_decode(P, tn["v8"], tn["vs"], True) + A(1.0 - b2) * (g * g)
        root = np.sqrt(v)
        w = w - (rate * m) / (root * rbc2 + A(opt.eps))
        tn["w32"][...] = w.reshape(tn["w32"].shape)
        unbiased = getattr(opt, "state_bits", 32) == 8
        tn["m8"][...], tn["ms"][...], tn["v8"][...], tn["vs"][...] = state8_encode_unbiased(P, m, root, t) if unbiased else state8_encode(P, m, root)
        tn["w16"][...] = P.store(tn["w32"])
    return 0


def loss_scale_update(st: ScaleState, found_inf: int) -> None:
    """Record the step and set the scale of the next iteration.

    overflow : scale <- max(scale/2, min), good_steps <- 0, step counted as skipped
    clean    : opt_step += 1, good_steps += 1; when good_steps reaches
               growth_interval: scale <- min(2 scale, max), good_steps <- 0
    static   : the scale never changes; an overflowing step is still skipped.
    """
    st.history.append((float(st.scale), int(found_inf)))
    st.total_steps += 1
    if found_inf:
        st.skipped_steps += 1
        st.good_steps = 0
        if st.mode == "backoff":
            st.scale = max(st.scale / 2.0, st.min_scale)
    else:
        st.opt_step += 1
        st.good_steps += 1
        if st.mode == "backoff" and st.good_steps >= st.growth_interval:
            st.scale = min(st.scale * 2.0, st.max_scale)
            st.good_steps = 0

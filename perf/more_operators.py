"""Operators of a Transformer language model, one at a time: norms of queries and keys with the rotation by position (one axis or
several), log probabilities of given tokens with entropy and alternatives, and distillation from a teacher's top logits.

Where `own` is true the calls are the framework's, as TransformerStep and XentStep make them; elsewhere they are the plain statement of
the same arithmetic in elementary torch operations."""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
SCALE = 2.0 ** 15                # the loss scale


# ------------------------------------------------------------------------------------------------------------ cases
def _rope(name, rows, heads, kv_heads, d_head, rot=None, axes=1, order="blocks", adjacent=False, norm=True, train=True, far=0):
    return {"name": name, "kind": "rope", "rows": rows, "heads": heads, "kv_heads": kv_heads, "d_head": d_head, "rot": rot or d_head,
            "axes": axes, "order": order, "adjacent": adjacent, "norm": norm, "train": train, "far": far}


def _logprobs(name, rows, vocab, top, temperature=1.0, train=False, banned=0, pad=0):
    return {"name": name, "kind": "logprobs", "rows": rows, "vocab": vocab, "top": top, "temperature": temperature, "train": train,
            "banned": banned, "pad": pad}


def _distill(name, rows, vocab, top, temperature=1.0, tail=False, hard=0.0, short=False):
    return {"name": name, "kind": "distill", "rows": rows, "vocab": vocab, "top": top, "temperature": temperature, "tail": tail,
            "hard": hard, "short": short}


def listed():
    return [
        # one new token far into a conversation: what a call costs
        _rope("rope_1_far", 1, 16, 4, 128, train=False, far=1 << 20),
        # the tokens of an iteration of the big layer, forward and backward with the norms' weights
        _rope("rope_8192x32x64", 8192, 16, 16, 64),
        # a document of an odd length, shared kv heads
        _rope("rope_12289x10x128", 12289, 8, 2, 128),
        # the patches of a few small images, row and column; half of each head turns, neighbours are pairs, no norm
        _rope("axes_61x8x80", 61, 4, 4, 80, rot=40, axes=2, adjacent=True, norm=False),
        # a film: time, height and width, dealt to the pairs in turn
        _rope("axes_16384x20x128", 16384, 16, 4, 128, axes=3, order="turns"),
        # the next token's alternatives as a program that answers reports them
        _logprobs("logprobs_1x32768_top20", 1, 32768, 20),
        # answers that a policy's loss weighs: probabilities and entropy of all tokens of an iteration, and the logits' gradient
        _logprobs("logprobs_8192x32768_train", 8192, 32768, 0, train=True, pad=97),
        # a teacher's pass over an odd vocabulary at a temperature, some classes never allowed
        _logprobs("logprobs_1021x50021_top64", 1021, 50021, 64, temperature=2.0, banned=21),
        # a batch of answers over a large vocabulary
        _logprobs("logprobs_64x131071_top8", 64, 131071, 8),
        # a few sentences, small vocabulary, lists of differing lengths
        _distill("distill_61x1000_top8", 61, 1000, 8, short=True),
        # the tokens of an iteration, the teacher's 64 classes and all others as one
        _distill("distill_8192x32768_top64", 8192, 32768, 64, tail=True),
        # a large odd vocabulary, softened, mixed with the texts' own tokens
        _distill("distill_1021x131071_top100", 1021, 131071, 100, temperature=2.0, hard=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "axes", "logprobs", "logprobs", "distill", "distill"])
    if kind in ("rope", "axes"):
        d = rng.choice([32, 64, 64, 80, 96, 128, 128])
        kv = rng.choice([1, 2, 4])
        c = _rope("", _log(rng, 1, 16384), kv * rng.choice([1, 2, 4]), kv, d, rot=rng.choice([d, d, d // 2, d // 4 * 3 // 4 * 4]),
                  axes=1 if kind == "rope" else rng.choice([2, 3]), order=rng.choice(["blocks", "turns"]), adjacent=rng.random() < 0.3,
                  norm=rng.random() < 0.75, train=rng.random() < 0.7, far=rng.choice([0, 0, _log(rng, 1, 1 << 21)]))
    else:
        vocab = _log(rng, 500, 131071)
        if rng.random() < 0.6:
            vocab = vocab // 8 * 8
        rows = max(1, min(_log(rng, 1, 8192), 8192 * 32768 // vocab))
        if kind == "logprobs":
            c = _logprobs("", rows, vocab, rng.choice([0, 1, _log(rng, 2, 100)]), temperature=rng.choice([1.0, 1.0, 0.7, 2.0]),
                          train=rng.random() < 0.4, banned=rng.choice([0, 0, rng.randint(1, vocab // 4)]), pad=rng.choice([0, rng.randint(0, rows // 8)]))
        else:
            c = _distill("", rows, vocab, _log(rng, 1, 100), temperature=rng.choice([1.0, 1.0, 2.0, 4.0]), tail=rng.random() < 0.5,
                         hard=rng.choice([0.0, 0.0, 0.25, 1.0]), short=rng.random() < 0.5)
            if c["temperature"] != 1.0 and c["hard"]:                      # both softmaxes: within the largest listed work
                c["rows"] = max(1, min(rows, 1021 * 131071 // vocab))
    del c["name"]
    return c


# ----------------------------------------------------------------------------------------------------------- inputs
def _axis_of_pairs(case):
    n, a = case["rot"] // 2, case["axes"]
    if case["order"] == "turns":
        return [i % a for i in range(n)]
    return [min(i * a // n, a - 1) for i in range(n)]


def _positions(case, seed):
    """[axes, rows]: one axis: packed documents, or a long way into one; several: a grid's coordinates, its text ahead on the diagonal."""
    T, a = case["rows"], case["axes"]
    r = np.random.RandomState(int(seed) % (1 << 31))
    if a == 1:
        if case["far"]:
            return (case["far"] + r.randint(0, 1000) + np.arange(T))[None]
        cuts = np.sort(r.randint(0, T + 1, max(1, T // 700)))
        start = np.concatenate([[0], cuts])
        return (np.arange(T) - start[np.searchsorted(start, np.arange(T), side="right") - 1])[None]
    text = r.randint(0, T // 8 + 1)
    n = T - text
    side = max(1, int(round(n ** (1.0 / a))))
    i = np.arange(n)
    grid = [i // side ** (a - 1 - k) if k == 0 else i // side ** (a - 1 - k) % side for k in range(a)]
    return np.stack([np.concatenate([np.arange(text), text + g]) for g in grid]) + case["far"]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    normal = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    if case["kind"] == "rope":
        T, H, G, D, R = case["rows"], case["heads"], case["kv_heads"], case["d_head"], case["rot"]
        s = {"qkv": normal(T, (H + 2 * G) * D).half(),                     # one projection's output, [q | k | v]
             "dy": (normal(T, (H + G) * D) * 0.25).half(),                 # loss-scaled, [dq | dk] behind the rotation
             "gq": (1 + 0.1 * normal(D)).half(), "gk": (1 + 0.1 * normal(D)).half(),
             "positions": torch.from_numpy(_positions(case, seed).astype(np.int32)).cuda(),
             "freqs": torch.from_numpy(10000.0 ** (-2.0 * np.arange(R // 2) / R)).cuda()}
    else:
        T, V, k = case["rows"], case["vocab"], case["top"]
        x = normal(T, V).mul_(2.0)
        # every other row knows what comes next: one class far ahead
        known = torch.randint(0, V, (T,), generator=g, device="cuda")
        x[torch.arange(T, device="cuda"), known] += torch.where(torch.arange(T, device="cuda") % 2 == 0, 14.0, 0.0)
        targets = torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, known, torch.randint(0, V, (T,), generator=g, device="cuda")).int()
        if case["kind"] == "logprobs":
            targets[T - case["pad"]:] = -1
            if case["banned"]:
                x[:, V - case["banned"]:] = -math.inf
                targets %= V - case["banned"]
            s = {"logits": x.half(), "targets": targets, "dlogp": normal(T) / T, "dentropy": torch.full((T,), -0.01 / T, device="cuda")}
        else:
            teacher = x.half()
            t = teacher.float().div_(case["temperature"])
            top, ids = torch.topk(t, k, dim=1)
            top = top - torch.logsumexp(t, 1, keepdim=True)
            del t
            if case["short"]:                                              # lists that end early, or hold nothing
                n = torch.randint(0, k + 1, (T, 1), generator=g, device="cuda")
                ids = torch.where(torch.arange(k, device="cuda")[None] < n, ids, -1)
            s = {"logits": (0.8 * teacher.float() + normal(T, V)).half(), "ids": ids.int().contiguous(), "top": top.contiguous(),
                 "targets": targets}
    s["case"] = case
    return s


# ----------------------------------------------------------------------------------------------------- plain forms
def _turn(n, cos, sin, adjacent, rot):
    """Pairs of the first `rot` columns turned; n [rows, heads, d], cos and sin [rows, 1, rot / 2]."""
    if adjacent:
        a, b = n[..., 0:rot:2], n[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = n[..., :rot // 2], n[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, n[..., rot:]], -1)


def _plain_rope(s):
    c = s["case"]
    T, H, G, D, R = c["rows"], c["heads"], c["kv_heads"], c["d_head"], c["rot"]
    axis = torch.tensor(_axis_of_pairs(c), device="cuda")
    angle = s["positions"][axis].double().t() * s["freqs"]                 # 32 bits lose the angles of far positions
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x = s["qkv"][:, :(H + G) * D].float().reshape(T, H + G, D)
    if c["norm"]:
        w = torch.cat([s["gq"].float().expand(H, D), s["gk"].float().expand(G, D)])
        r = torch.rsqrt(x.square().mean(2, keepdim=True) + EPS)
        hat = x * r
        n = hat * w
    else:
        n = x
    out = {"y": _turn(n, cos, sin, c["adjacent"], R).reshape(T, -1).half()}
    if c["train"]:
        u = _turn(s["dy"].float().reshape(T, H + G, D), cos, -sin, c["adjacent"], R)
        if c["norm"]:
            out["dgq"] = (u * hat)[:, :H].sum((0, 1)).half()
            out["dgk"] = (u * hat)[:, H:].sum((0, 1)).half()
            v = u * w
            u = r * (v - hat * (v * hat).mean(2, keepdim=True))
        out["d"] = u.reshape(T, -1).half()
    return out


def _plain_top(z, x, lse, k):
    """The k largest of each row of x in descending order, ties to the lowest index."""
    V = x.shape[1]
    i = (x + 0.0).view(torch.int32)
    key = (i ^ ((i >> 31) & 0x7fffffff)).long() * (1 << 32) + (V - 1 - torch.arange(V, device="cuda"))
    best = torch.topk(key, k, dim=1).values
    ids = V - 1 - (best & 0xffffffff)
    return ids.int(), z.gather(1, ids) - lse[:, None]


def _log_sum(z):
    top = z.amax(1, keepdim=True)
    safe = torch.where(top == -math.inf, 0.0, top)
    return safe[:, 0] + torch.log(torch.exp(z - safe).sum(1))


def _plain_logprobs(s):
    c = s["case"]
    V, ct = c["vocab"], 1.0 / c["temperature"]
    x = s["logits"].float()
    z = x * ct
    lse = _log_sum(z)
    t = s["targets"].long()
    there = (t >= 0) & (t < V)
    safe = torch.where(there, t, 0)
    logp = torch.where(there, z.gather(1, safe[:, None])[:, 0] - lse, 0.0)
    lp = z - lse[:, None]
    p = torch.exp(lp)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    out = {"logp": logp, "entropy": entropy, "lse": lse}
    if c["top"]:
        out["top_ids"], out["top_logp"] = _plain_top(z, x, lse, c["top"])
    if c["train"]:
        g = torch.where(there, s["dlogp"], 0.0)[:, None]
        d = -p * g - s["dentropy"][:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), 0.0)
        d.scatter_add_(1, safe[:, None], g)
        out["dlogits"] = (d * (SCALE * ct)).half()
    return out


def _plain_distill(s):
    c = s["case"]
    T, V, ct = c["rows"], c["vocab"], 1.0 / c["temperature"]
    w = c["temperature"] ** 2
    x = s["logits"].float()
    z = x * ct
    lse = _log_sum(z)
    ids, there = s["ids"].long(), (s["ids"] >= 0) & (s["ids"] < V)
    safe = torch.where(there, ids, 0)
    t = torch.where(there, s["top"], -math.inf).double()                   # 1 - sum of probabilities next to 1: 64 bits
    if c["tail"]:
        q = torch.exp(t)
        r = (1 - q.sum(1)).clamp_(min=0)
    else:
        top = t.amax(1, keepdim=True)
        q = torch.exp(t - torch.where(top == -math.inf, 0.0, top))
        total = q.sum(1, keepdim=True)
        q, r = q / torch.where(total == 0, 1.0, total), torch.zeros(T, dtype=torch.float64, device="cuda")
    some = there.any(1)
    r = torch.where(some, r, 0.0).float()
    q = torch.zeros(T, V, device="cuda").scatter_add_(1, safe, q.float())  # a class that is listed twice counts with the sum
    listed_ = torch.zeros(T, V, dtype=torch.int32, device="cuda").scatter_add_(1, safe, there.int()) > 0
    lp = z - lse[:, None]
    loss = torch.where(q > 0, q * (torch.log(q) - lp), 0.0).sum(1)
    p = torch.exp(lp)
    d = p * (q.sum(1) + r)[:, None] - q
    if c["tail"]:
        rest = z.masked_fill(listed_, -math.inf)
        rest_lse = _log_sum(rest)
        r = torch.where(rest_lse == -math.inf, 0.0, r)
        loss = loss + torch.where(r > 0, r * (torch.log(r) - (rest_lse - lse)), 0.0)
        d = d - r[:, None] * torch.exp(rest - rest_lse[:, None])
    loss = torch.where(some, loss, 0.0) * w
    d = torch.where(some[:, None], d, 0.0) * (w * ct)
    if c["hard"]:
        y = s["targets"].long()
        real = (y >= 0) & (y < V)
        y = torch.where(real, y, 0)
        lse1 = _log_sum(x)
        loss = loss + c["hard"] * torch.where(real, lse1 - x.gather(1, y[:, None])[:, 0], 0.0)
        h = torch.where(real, c["hard"], 0.0)[:, None]
        d = d + torch.exp(x - lse1[:, None]) * h
        d.scatter_add_(1, y[:, None], -h)
    return {"loss": loss.sum() / T, "dlogits": (d * (SCALE / T)).half()}


# ------------------------------------------------------------------------------------------------ the framework's
def _own_rope(s):
    import paper_1805_10387_amd as mp
    c = s["case"]
    T, H, G, D = c["rows"], c["heads"], c["kv_heads"], c["d_head"]
    if "own" not in s:                                                      # a program's buffers, from its first iteration on
        e16 = lambda *n: torch.empty(n, dtype=torch.float16, device="cuda")  # noqa: E731
        ld = (H + 2 * G) * D
        desc = mp.rope_desc(T, H, G, D, rot=c["rot"], n_axes=c["axes"], axis=_axis_of_pairs(c), adjacent=c["adjacent"], eps=EPS, ld_q=ld, ld_k=ld,
                            ld_yq=(H + G) * D, ld_yk=(H + G) * D, ld_dq=(H + G) * D, ld_dk=(H + G) * D)
        train = c["train"]
        s["own"] = {"desc": desc, "y": e16(T, (H + G) * D), "d": e16(T, (H + G) * D) if train else None, "dgq": e16(D), "dgk": e16(D),
                    "ws": torch.empty(mp.mp_qk_norm_rope_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda") if train else None}
    b, x, dy, kq = s["own"], s["qkv"], s["dy"], H * D
    gq, gk = (s["gq"], s["gk"]) if c["norm"] else (None, None)
    mp.mp_qk_norm_rope_fwd(b["desc"], x, x[:, kq:], gq, gk, s["positions"], s["freqs"], b["y"], b["y"][:, kq:])
    out = {"y": b["y"]}
    if c["train"]:
        dgq, dgk = (b["dgq"], b["dgk"]) if c["norm"] else (None, None)
        mp.mp_qk_norm_rope_bwd(b["desc"], x, x[:, kq:], gq, gk, s["positions"], s["freqs"], dy, dy[:, kq:], b["d"], b["d"][:, kq:], dgq, dgk,
                               ws=b["ws"])
        if c["norm"]:
            out["dgq"], out["dgk"] = dgq, dgk
        out["d"] = b["d"]
    return out


def _own_state():
    import paper_1805_10387_amd as mp
    from paper_1805_10387_amd import _lib as ML
    st = mp.scale_state_alloc()
    mp.mp_scale_state_init(st, ML.MP_SCALE_STATIC, SCALE, 1)
    return st


def _own_logprobs(s):
    import paper_1805_10387_amd as mp
    c = s["case"]
    T, V, k, ct = c["rows"], c["vocab"], c["top"], 1.0 / c["temperature"]
    if "own" not in s:
        e32 = lambda *n: torch.empty(n, dtype=torch.float32, device="cuda")  # noqa: E731
        s["own"] = {"logp": e32(T), "entropy": e32(T), "lse": e32(T), "top_ids": torch.empty(T, k, dtype=torch.int32, device="cuda") if k else None,
                    "top_logp": e32(T, k) if k else None, "dlogits": torch.empty_like(s["logits"]) if c["train"] else None,
                    "ws": torch.empty(mp.mp_token_logprobs_workspace_bytes(T, V, k), dtype=torch.uint8, device="cuda"), "st": _own_state()}
    b = s["own"]
    mp.mp_token_logprobs(T, V, k, s["logits"], V, s["targets"], ct, b["logp"], b["entropy"], b["lse"], b["top_ids"], b["top_logp"], b["ws"])
    out = {"logp": b["logp"], "entropy": b["entropy"], "lse": b["lse"]}
    if k:
        out["top_ids"], out["top_logp"] = b["top_ids"], b["top_logp"]
    if c["train"]:
        mp.mp_token_logprobs_bwd(T, V, s["logits"], V, s["targets"], ct, b["entropy"], b["lse"], s["dlogp"], s["dentropy"], b["st"], b["dlogits"])
        out["dlogits"] = b["dlogits"]
    return out


def _own_distill(s):
    import paper_1805_10387_amd as mp
    c = s["case"]
    T, V = c["rows"], c["vocab"]
    if "own" not in s:
        desc = mp.distill_desc(T, V, c["top"], inv_temperature=1.0 / c["temperature"], weight=c["temperature"] ** 2, hard_weight=c["hard"],
                               tail=c["tail"])
        s["own"] = {"desc": desc, "loss": torch.empty(1, dtype=torch.float32, device="cuda"), "dlogits": torch.empty_like(s["logits"]),
                    "ws": torch.empty(mp.mp_distill_workspace_bytes(desc), dtype=torch.uint8, device="cuda"), "st": _own_state()}
    b = s["own"]
    mp.mp_distill_scaled(b["desc"], s["logits"], s["ids"], s["top"], s["targets"] if c["hard"] else None, b["st"], b["loss"], b["dlogits"], b["ws"])
    return {"loss": b["loss"][0], "dlogits": b["dlogits"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rope": _own_rope, "logprobs": _own_logprobs, "distill": _own_distill}[kind](state)
    return {"rope": _plain_rope, "logprobs": _plain_logprobs, "distill": _plain_distill}[kind](state)


# ------------------------------------------------------------------------------------------------------ 64 bits
def _exact_rope(s):
    """Head by head, with complex numbers for the pairs."""
    c = s["case"]
    T, H, G, D, R = c["rows"], c["heads"], c["kv_heads"], c["d_head"], c["rot"]
    at = torch.arange(R, device="cuda").reshape(-1, 2) if c["adjacent"] else torch.arange(R, device="cuda").reshape(2, -1).t()
    pos = torch.stack([s["positions"][a].double() for a in _axis_of_pairs(c)], 1)
    spin = torch.exp(1j * (pos * s["freqs"]))                              # [rows, pairs]

    def turned(v, by):
        v = v.clone()
        w = torch.complex(v[:, at[:, 0]], v[:, at[:, 1]]) * by
        v[:, at[:, 0]], v[:, at[:, 1]] = w.real, w.imag
        return v

    y, d, dg = [], [], [torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(2)]
    for h in range(H + G):
        x = s["qkv"][:, h * D:h * D + D].double()
        g = s["gq" if h < H else "gk"].double()
        norm = ((x ** 2).sum(1, keepdim=True) / D + EPS) ** 0.5
        y.append(turned(g * x / norm if c["norm"] else x, spin))
        u = turned(s["dy"][:, h * D:h * D + D].double(), spin.conj())
        if c["norm"]:
            dg[int(h >= H)] += (u * x / norm).sum(0)
            u = u * g / norm - x * ((u * g * x).sum(1, keepdim=True) / (D * norm ** 3))
        d.append(u)
    out = {"y": torch.cat(y, 1)}
    if c["train"]:
        if c["norm"]:
            out["dgq"], out["dgk"] = dg
        out["d"] = torch.cat(d, 1)
    return out


def _exact_logprobs(s):
    c = s["case"]
    V, out = c["vocab"], {"logp": [], "entropy": [], "lse": []}
    if c["top"]:
        out.update(top_ids=[], top_logp=[])
    if c["train"]:
        out.update(dlogits=[])
    step = max(1, (1 << 26) // V)
    for a in range(0, c["rows"], step):
        z = s["logits"][a:a + step].double() / c["temperature"]
        t, g, h = s["targets"][a:a + step].tolist(), s["dlogp"][a:a + step].double(), s["dentropy"][a:a + step].double()
        lp = torch.log_softmax(z, 1)
        e = torch.special.entr(torch.exp(lp)).sum(1)
        out["lse"].append(torch.logsumexp(z, 1))
        out["entropy"].append(e)
        out["logp"].append(torch.stack([lp[i, j] if 0 <= j < V else lp.new_zeros(()) for i, j in enumerate(t)]))
        if c["top"]:
            order = torch.sort(s["logits"][a:a + step].double(), dim=1, descending=True, stable=True).indices[:, :c["top"]]
            out["top_ids"].append(order.int())
            out["top_logp"].append(lp.gather(1, order))
        if c["train"]:
            real = torch.tensor([float(0 <= j < V) for j in t], dtype=torch.float64, device="cuda")
            one = torch.zeros_like(lp)
            one[torch.arange(len(t)), [j if 0 <= j < V else 0 for j in t]] = real
            p = torch.exp(lp)
            d = (g * real)[:, None] * (one - p) - h[:, None] * (e[:, None] * p - torch.special.entr(p))
            out["dlogits"].append(d * SCALE / c["temperature"])
    return {k: torch.cat(v) for k, v in out.items()}


def _exact_distill(s):
    """Some rows at a time; the derivative of a sum of logarithms of probabilities, term by term."""
    c = s["case"]
    T, V, w = c["rows"], c["vocab"], c["temperature"] ** 2
    total, out, step = 0.0, [], max(1, (1 << 26) // V)
    for a in range(0, T, step):
        x = s["logits"][a:a + step].double()
        n = x.shape[0]
        lp = torch.log_softmax(x / c["temperature"], 1)
        p = torch.exp(lp)
        teach = torch.zeros(n, V + 1, dtype=torch.float64, device="cuda")  # one more class for what is not there
        ids = s["ids"][a:a + step].long()
        ids = torch.where((ids >= 0) & (ids < V), ids, V)
        teach.scatter_add_(1, ids, torch.exp(s["top"][a:a + step].double()))
        named = torch.zeros(n, V + 1, dtype=torch.bool, device="cuda")
        named.scatter_(1, ids, torch.ones_like(ids, dtype=torch.bool))
        teach, named = teach[:, :V], named[:, :V]
        mass = teach.sum(1)
        some = (mass > 0).double()
        if c["tail"]:
            rest = torch.where(some > 0, (1 - mass).clamp(min=0), 0.0)
        else:
            teach, rest = teach / torch.where(mass > 0, mass, 1.0)[:, None], torch.zeros_like(mass)
        kl = (torch.xlogy(teach, teach) - torch.where(teach > 0, teach * lp, 0.0)).sum(1)
        d = teach.sum(1, keepdim=True) * p - teach
        if c["tail"]:
            others = torch.where(named, 0.0, p).sum(1)
            kl += torch.xlogy(rest, rest) - rest * torch.log(others)
            d += rest[:, None] * (p - torch.where(named, 0.0, p) / others[:, None])
        total = total + (kl * some).sum() * w
        d = d * some[:, None] * (w / c["temperature"])
        if c["hard"]:
            lp1 = torch.log_softmax(x, 1)
            t = s["targets"][a:a + step].long()
            total = total - c["hard"] * lp1.gather(1, t[:, None]).sum()
            d += c["hard"] * torch.exp(lp1)
            d.scatter_add_(1, t[:, None], torch.full((n, 1), -c["hard"], dtype=torch.float64, device="cuda"))
        out.append(d * (SCALE / T))
    return {"loss": total / T, "dlogits": torch.cat(out)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "logprobs": _exact_logprobs, "distill": _exact_distill}[case["kind"]](s)


# ------------------------------------------------------------------------------------------------------ least work
def work(case):
    """Rotation: queries and keys read and written, positions and weights read; backward the two and their gradients read, gradients
    written.  Log probabilities: the logits once, and for a gradient (whose coefficients a program has only after the forward pass) once
    more, and it written.  Distillation: the logits once, their gradient, the teacher's lists."""
    if case["kind"] == "rope":
        n = float(case["rows"]) * (case["heads"] + case["kv_heads"]) * case["d_head"]
        small = 4.0 * case["rows"] * case["axes"] + 4.0 * case["rot"] + (4.0 * case["d_head"] if case["norm"] else 0)
        fwd = {"bytes": 4 * n + small, "flops": n * (8 if case["norm"] else 3)}
        if not case["train"]:
            return fwd
        return {"bytes": fwd["bytes"] + n * (6 if case["norm"] else 4) + small + (4.0 * case["d_head"] if case["norm"] else 0),
                "flops": fwd["flops"] + n * (14 if case["norm"] else 3)}
    n = float(case["rows"]) * case["vocab"]
    if case["kind"] == "logprobs":
        small = case["rows"] * (16.0 + 8.0 * case["top"])
        return {"bytes": n * (6 if case["train"] else 2) + small, "flops": n * (12 if case["train"] else 6)}
    return {"bytes": 4 * n + case["rows"] * (8.0 * case["top"] + 8.0), "flops": n * (14 if case["hard"] else 9)}

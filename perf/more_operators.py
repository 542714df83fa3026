"""Performance cases of what a training step runs beside the expert layer and the
losses: embedding, layer norm, the gradients' norm and the AdamW update.

  embed   the embedding of a batch's tokens and its weight gradient;
  norm    layer norm, of a residual sum or of one tensor, and its gradients;
  gnorm   the sum of squares of many tensors' gradients;
  adamw   an AdamW step over many tensors, its states in 32 bits or in 8 (then
          also read back as the values they stand for, as a checkpoint does).

`run` computes them in elementary torch operations, or through the Python
binding (paper_2607_01844_amd.moe) where `own` is true.  Sizes are those of
workloads.py, of the tests, and generic ones beside them.
"""
from __future__ import annotations

import math

import torch

own = False

W_STD = 0.02
BLOCK = 128  # values of one scale of an 8-bit state
EPS_NORM = 1e-5
LR, BETA1, BETA2, EPS, DECAY, STEP = 3e-4, 0.9, 0.95, 1e-8, 0.1, 100
MAX_NORM = 1.0
SEED = 20


# ------------------------------------------------------------------- cases
def _embed(name, N, H, V, shard=False, pad=0.0):
    return {"name": name, "kind": "embed", "N": N, "H": H, "V": V, "shard": shard, "pad": pad}


def _norm(name, T, d, residual, backward=True):
    return {"name": name, "kind": "norm", "T": T, "d": d, "residual": residual,
            "backward": backward}


def _gnorm(name, layers, d, E, f, V):
    return {"name": name, "kind": "gnorm", "layers": layers, "d": d, "E": E, "f": f, "V": V}


def _adamw(name, layers, d, E, f, V, bits, master, clip=True):
    return {"name": name, "kind": "adamw", "layers": layers, "d": d, "E": E, "f": f, "V": V,
            "bits": bits, "master": master, "clip": clip}


def listed():
    return [
        # the smallest vocabulary of the tests: launches and little else
        _embed("embed_tiny", 256, 128, 1000),
        # a rank's half of an odd vocabulary, some padding, width no multiple of 64
        _embed("embed_ragged", 1100, 520, 32003, shard=True, pad=0.05),
        # the long-context chunk over a vocabulary of 200,000
        _embed("embed_long", 65536, 4096, 200000),
        # generation: a handful of tokens, forward alone, with the residual sum
        _norm("norm_decode", 16, 4096, True, backward=False),
        # odd sizes: rows that end inside a wave's reach, no residual
        _norm("norm_ragged", 1100, 520, False),
        # the long-context chunk between attention and the expert layer
        _norm("norm_long", 65536, 4096, True),
        # two of the smallest layers: small tensors, launches
        _gnorm("gnorm_tiny", 2, 128, 8, 256, 1000),
        # a mid-sized layer and its vocabulary
        _gnorm("gnorm_mid", 1, 2048, 64, 1408, 32000),
        # two of the smallest layers, states in 32 bits
        _adamw("adamw_tiny", 2, 128, 8, 256, 1000, 32, True),
        # a mid-sized layer: fp32 weights with a bf16 copy, states in 32 bits
        _adamw("adamw_mid", 1, 2048, 64, 1408, 32000, 32, True),
        # odd sizes, weights in bf16 alone, states in 8 bits, no clipping
        _adamw("adamw8_ragged", 3, 520, 12, 328, 32003, 8, False, clip=False),
        # the mid-sized layer with states in 8 bits
        _adamw("adamw8_mid", 1, 2048, 64, 1408, 32000, 8, True),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """One more case of the listed ranges, at most the largest listed one's
    work."""
    kind = rng.choice(["embed", "embed", "norm", "norm", "gnorm", "adamw", "adamw"])
    while True:
        if kind == "embed":
            c = _embed("", _log_int(rng, 1, 65536), _log_int(rng, 64, 8192, 8),
                       _log_int(rng, 100, 262144), rng.random() < 0.3, rng.choice([0.0, 0.0, 0.1]))
            if c["N"] * c["H"] <= 2.7e8 and c["V"] * c["H"] <= 8.2e8:
                break
        elif kind == "norm":
            c = _norm("", _log_int(rng, 1, 65536), _log_int(rng, 64, 16384, 8),
                      rng.random() < 0.6, rng.random() < 0.7)
            if c["T"] * c["d"] <= 2.7e8:
                break
        else:
            a = (rng.randint(1, 24), _log_int(rng, 64, 4096, 8), rng.choice([4, 8, 12, 16, 32, 64]),
                 _log_int(rng, 64, 2048, 8), _log_int(rng, 1000, 200000))
            if a[0] * 3 * a[1] * a[2] * a[3] + a[1] * a[4] > 6.1e8:
                continue
            if kind == "gnorm":
                c = _gnorm("", *a)
            else:
                c = _adamw("", *a, rng.choice([8, 8, 32]), rng.random() < 0.6, rng.random() < 0.7)
            break
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _normal(shape, std, gen, dtype):
    """N(0, std) of `dtype`, drawn a slice of the first axis at a time."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 27) // max(1, out[:1].numel()))
    for i in range(0, shape[0], step):
        part = out[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(std))
    return out


def _sizes(case):
    """Elements of the tensors of a model: (matrices, the small fp32 ones)."""
    L, d, E, f, V = (case[n] for n in ("layers", "d", "E", "f", "V"))
    return [V * d] + [E * d * f] * (3 * L), [d * E, d, d] * L + [d, d]


def _starts(sizes):
    """Places of the tensors in one buffer, each at a multiple of 128 elements,
    and the buffer's length."""
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // BLOCK) * BLOCK)
    return at


def _inside(sizes, at, dev="cuda"):
    """Which elements of such a buffer belong to a tensor."""
    t = torch.zeros(at[-1], dtype=torch.bool, device=dev)
    for n, a in zip(sizes, at):
        t[a:a + n] = True
    return t


def _magnitudes(case, n, gen):
    """States of a model that has trained a while: spread over some octaves."""
    return torch.exp(_normal((n,), 1.5, gen, torch.float32)).mul_(1e-4)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    bf, f32, dev = torch.bfloat16, torch.float32, "cuda"
    s = {"case": case}
    if case["kind"] == "embed":
        N, H, V = (case[n] for n in ("N", "H", "V"))
        # the words of a text: the n-th most frequent one as often as 1 / n
        u = torch.rand((N,), generator=gen, device=dev, dtype=torch.float64)
        ids = (torch.exp(u * math.log(V + 1)) - 1).long().clamp(max=V - 1)
        order = torch.randperm(V, generator=gen, device=dev)
        ids = order[ids]
        ids[torch.rand((N,), generator=gen, device=dev) < case["pad"]] = -1
        s["ids"] = ids.to(torch.int32)
        s["begin"], s["rows"] = (V // 4, V // 2) if case["shard"] else (0, V)
        s["w"] = _normal((s["rows"], H), W_STD, gen, bf)
        s["dy"] = _normal((N, H), 1.0, gen, bf)
        s["scale"] = math.sqrt(H)
        return s
    if case["kind"] == "norm":
        T, d = case["T"], case["d"]
        s["x"] = _normal((T, d), 1.0, gen, bf)
        s["x"] += _normal((1, d), 0.5, gen, bf)  # channels with an offset of their own
        s["residual"] = _normal((T, d), 2.0, gen, bf) if case["residual"] else None
        s["gamma"] = 1 + _normal((d,), 0.1, gen, f32)
        s["beta"] = _normal((d,), 0.1, gen, f32)
        if case["backward"]:
            s["dy"] = _normal((T, d), 1.0, gen, bf)
            s["dh"] = _normal((T, d), 1.0, gen, bf) if case["residual"] else None
        return s
    s["groups"] = []
    for i, sizes in enumerate(_sizes(case)):
        at = _starts(sizes)
        ok = _inside(sizes, at)
        g = {"sizes": sizes, "at": at, "g": _normal((at[-1],), 1e-4, gen, f32 if i else bf) * ok}
        s["groups"].append(g)
        if case["kind"] == "gnorm":
            continue
        w = _normal((at[-1],), W_STD, gen, f32) * ok
        g["w"] = w if i or case["master"] else w.to(bf)
        g["copy"] = w.to(bf) if case["master"] and not i else None
        m = _magnitudes(case, at[-1], gen) * torch.randn((at[-1],), generator=gen, device=dev) * ok
        v = _magnitudes(case, at[-1], gen).square_() * ok
        if case["bits"] == 32:
            g["m"], g["v"] = m, v
        else:
            zero = torch.full((1,), 1 << 15, dtype=torch.int64, device=dev)  # to the nearest
            g["m"], g["v"] = _encode(m, True, zero), _encode(v, False, zero)
    # of all ranks' gradients, as the caller has summed it: twice the norm allowed
    s["sumsq"] = torch.full((1,), 4.0 * MAX_NORM, device=dev) if case.get("clip") else None
    return s


# ------------------------------------------------- states held in 8 bits
def _bits(x):
    return x.view(torch.int32).long()


def _from_bits(b):
    return b.to(torch.int32).view(torch.float32)


def _encode(x, signed, r):
    """(codes, scales) of a state, blocks of 128: |x| + u, u a power of two below
    the block's largest, keeps its exponent and three bits of mantissa; the
    rest, r / 65536 of a step added, is cut off."""
    b = x.view(-1, BLOCK)
    top = _bits(b.abs().amax(1)) >> 23
    scale = (top - (14 if signed else 30)).clamp(min=1)
    scale = torch.where(top == 255, 255, scale)
    y = _bits(b.abs() + _from_bits(scale << 23)[:, None])
    c = ((y + (r.expand(x.shape).reshape(b.shape) << 4) + 8) >> 20) - (scale << 3)[:, None]
    if signed:
        c = c | ((b < 0).long() << 7)
    else:
        c = torch.maximum(c, (b > 0).long())
    c = torch.where(scale[:, None] == 255, 0, c)
    return c.to(torch.uint8).view(-1), scale.to(torch.uint8)


def _decode(codes, scales, signed):
    c = codes.view(-1, BLOCK).long()
    e = scales.long()[:, None] << 23
    mag = _from_bits(((c & 127 if signed else c) << 20) + e) - _from_bits(e)
    return (torch.where(c > 127, -mag, mag) if signed else mag).view(-1)


def _mix(x, k):
    x = x ^ (x >> 16)
    x = (x * k) & 0xFFFFFFFF
    return x ^ (x >> 15)


def _random(group, first):
    """Two times 16 bits for each element of a group's tensors (numbered from
    `first`): of the element's place in its tensor, the tensor's number, the step
    and the seed."""
    dev = group["g"].device
    at = torch.tensor(group["at"], device=dev)
    n = at[1:] - at[:-1]
    j = torch.arange(first, first + n.numel(), device=dev)
    key = (SEED + STEP * 0x85A308D3 + j * 0x9E3779B9) & 0xFFFFFFFF
    key = _mix(_mix(key, 0x6A09E667), 0xBB67AE85)
    x = torch.arange(group["at"][-1], device=dev) - at[:-1].repeat_interleave(n)
    x = (x * 0x9E3779B9 + key.repeat_interleave(n)) & 0xFFFFFFFF
    return _mix(x, 0x6A09E667)


# ------------------------------------------------------- elementary forms
def _run_embed(s):
    ids = s["ids"].long() - s["begin"]
    there = (ids >= 0) & (ids < s["rows"])
    row = torch.where(there, ids, 0)
    y = torch.where(there[:, None], s["w"][row].float() * s["scale"], 0.0)
    dw = torch.zeros(s["w"].shape, dtype=torch.float32, device=row.device)
    dw.index_add_(0, row, torch.where(there[:, None], s["dy"].float(), 0.0))
    return {"y": y.bfloat16(), "dw": (dw * s["scale"]).bfloat16()}


def _run_norm(s):
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).bfloat16()
    x = h.float()
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1 / torch.sqrt((c * c).mean(1) + EPS_NORM)
    xh = c * rstd[:, None]
    out = {"y": (xh * s["gamma"] + s["beta"]).bfloat16(), "h": h, "mean": mean, "rstd": rstd}
    if s["case"]["backward"]:
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)
        dx *= rstd[:, None]
        if s["dh"] is not None:
            dx += s["dh"].float()
        out |= {"dx": dx.bfloat16(), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    return out


def _run_gnorm(s):
    return {"sumsq": sum(g["g"].float().square().sum(dtype=torch.float64)
                         for g in s["groups"]).float().view(1)}


def _clip(s):
    """What the gradients are multiplied by: 32 bits of a factor found in 64."""
    if s["sumsq"] is None:
        return 1.0
    return (MAX_NORM / s["sumsq"].double().sqrt().clamp(min=MAX_NORM)).float()


def _run_group(s, group, first):
    bits = s["case"]["bits"]
    g = group["g"].float() * _clip(s)
    m, v = group["m"], group["v"]
    if bits == 8:
        m, v = _decode(*m, True), _decode(*v, False)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    u = m / (torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS)
    w = group["w"].float() * (1 - LR * DECAY) - u * (LR / (1 - BETA1 ** STEP))
    if bits == 8 or group["w"].dtype is torch.bfloat16:
        r = _random(group, first)
    if group["w"].dtype is torch.bfloat16:
        # up or down at random: a step is a small part of a bf16 weight's last bit
        rw = ((r * 0xBB67AE85) & 0xFFFFFFFF) >> 16
        w = _from_bits((_bits(w) + rw) & ~0xFFFF)
    group["w"].copy_(w)
    if group["copy"] is not None:
        group["copy"].copy_(w)
    if bits == 32:
        group["m"].copy_(m)
        group["v"].copy_(v)
    else:
        for name, x, q, signed in (("m", m, r & 0xFFFF, True), ("v", v, r >> 16, False)):
            for held, new in zip(group[name], _encode(x, signed, q)):
                held.copy_(new)
        m, v = _decode(*group["m"], True), _decode(*group["v"], False)
    return {"w": group["w"], "copy": group["copy"], "m": m, "v": v}


def _run_adamw(s):
    mats, small = s["groups"]
    return [_run_group(s, mats, 0), _run_group(s, small, len(mats["sizes"]))]


# --------------------------------------------------------- framework calls
def _cut(group, flat):
    return [flat[a:a + n] for a, n in zip(group["at"], group["sizes"])]


def _states(group, name):
    """The tensors' states: fp32 values, or (codes, scales)."""
    if not isinstance(group[name], tuple):
        return _cut(group, group[name])
    codes, scales = group[name]
    return [(codes[a:a + n], scales[a // BLOCK:a // BLOCK + -(-n // BLOCK)])
            for a, n in zip(group["at"], group["sizes"])]


def _plan(s, moe):
    """The list of tensors that a program makes once and keeps."""
    if "params" not in s:
        both = s["groups"]
        w = [t for g in both for t in _cut(g, g["w"])]
        copy = [t for g in both for t in
                (_cut(g, g["copy"]) if g["copy"] is not None else [None] * len(g["sizes"]))]
        s["params"] = moe.Params(w, [t for g in both for t in _cut(g, g["g"])],
                                 [t for g in both for t in _states(g, "m")],
                                 [t for g in both for t in _states(g, "v")], copy)
        if s["case"]["bits"] == 8:
            s["read"] = [[torch.zeros(g["at"][-1], device="cuda") for g in both] for _ in "mv"]
            s["read_cut"] = [[t for g, x in zip(both, flat) for t in _cut(g, x)]
                             for flat in s["read"]]
    return s["params"]


def _own_embed(s, moe):
    y = moe.moe_embedding_fwd(s["ids"], s["w"], s["scale"], s["begin"])
    return {"y": y, "dw": moe.moe_embedding_bwd(s["ids"], s["dy"], s["rows"], s["scale"],
                                                s["begin"])}


def _own_norm(s, moe):
    y, h, mean, rstd = moe.moe_layer_norm_fwd(s["x"], s["gamma"], s["beta"], EPS_NORM,
                                              s["residual"])
    out = {"y": y, "h": h, "mean": mean, "rstd": rstd}
    if s["case"]["backward"]:
        dx, dgamma, dbeta = moe.moe_layer_norm_bwd(s["dy"], h, s["gamma"], mean, rstd, s["dh"])
        out |= {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    return out


def _own_gnorm(s, moe):
    if "grads" not in s:
        s["grads"] = moe.Params(None, [t for g in s["groups"] for t in _cut(g, g["g"])])
    return {"sumsq": moe.moe_grad_sumsq(s["grads"])}


def _own_adamw(s, moe):
    params = _plan(s, moe)
    moe.moe_adamw_step(params, LR, STEP, BETA1, BETA2, EPS, DECAY, grad_sumsq=s["sumsq"],
                       max_norm=MAX_NORM, seed=SEED)
    if s["case"]["bits"] == 8:
        moe.moe_adamw_states(params, *s["read_cut"])
        m, v = s["read"]
    else:
        m, v = ([g[n] for g in s["groups"]] for n in "mv")
    return [{"w": g["w"], "copy": g["copy"], "m": m[i], "v": v[i]}
            for i, g in enumerate(s["groups"])]


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2607_01844_amd import moe
        return {"embed": _own_embed, "norm": _own_norm, "gnorm": _own_gnorm,
                "adamw": _own_adamw}[kind](state, moe)
    return {"embed": _run_embed, "norm": _run_norm, "gnorm": _run_gnorm,
            "adamw": _run_adamw}[kind](state)


# ------------------------------------------------------------------- floors
def work(case):
    """Bytes: every input read once, every output written once (embedding rows
    that the tokens are expected to name)."""
    if case["kind"] == "embed":
        N, H, V = (case[n] for n in ("N", "H", "V"))
        p = torch.log1p(1 / torch.arange(1, V + 1, dtype=torch.float64)) / math.log(V + 1)
        p *= 1 - case["pad"]
        share = 0.5 if case["shard"] else 1.0
        used = share * float((1 - (1 - p) ** N).sum())
        n = N * (1 - case["pad"]) * share  # tokens of this rank
        return {"bytes": int(2 * H * (used + N + n + share * V) + 8 * N),
                "flops": int(2 * n * H + share * V * H)}
    if case["kind"] == "norm":
        n = case["T"] * case["d"]
        b = 8 if case["residual"] else 4
        if case["backward"]:
            b += 8 if case["residual"] else 6
        return {"bytes": b * n, "flops": (20 if case["backward"] else 8) * n}
    mats, small = (sum(x) for x in _sizes(case))
    if case["kind"] == "gnorm":
        return {"bytes": 2 * mats + 4 * small, "flops": 2 * (mats + small)}
    state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK
    if case["bits"] == 8:
        state += 2 + 2 / BLOCK + 8  # read back as values
    return {"bytes": int((2 + (10 if case["master"] else 4) + state) * mats + (12 + state) * small),
            "flops": 20 * (mats + small)}


# ------------------------------------------------------- 64-bit reference
def _exact_embed(s):
    H, rows = s["case"]["H"], s["rows"]
    lo = s["begin"]
    order = torch.argsort(s["ids"], stable=True)
    ids = s["ids"][order].long()
    order = order[(ids >= lo) & (ids < lo + rows)]
    ids = s["ids"][order].long() - lo
    y = torch.zeros((s["case"]["N"], H), dtype=torch.float64, device=ids.device)
    y[order] = s["w"][ids].double() * s["scale"]
    found, n = torch.unique_consecutive(ids, return_counts=True)
    # sums of runs as differences of running sums, some columns at a time
    dw = torch.zeros((rows, H), dtype=torch.float64, device=ids.device)
    if found.numel():
        for c in range(0, H, 512):
            run_sum = s["dy"][order, c:c + 512].double().cumsum(0)[n.cumsum(0) - 1]
            run_sum[1:] -= run_sum[:-1].clone()
            dw[found, c:c + 512] = run_sum * s["scale"]
    return {"y": y, "dw": dw}


def _exact_norm(s):
    h = s["x"]
    if s["residual"] is not None:
        h = (s["x"].double() + s["residual"].double()).bfloat16()
    x = h.double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    r = (var + EPS_NORM).rsqrt()
    n = (x - mean).mul_(r)
    out = {"y": n * s["gamma"].double() + s["beta"].double(), "h": h, "mean": mean[:, 0],
           "rstd": r[:, 0]}
    if s["case"]["backward"]:
        dy = s["dy"].double()
        out["dbeta"] = dy.sum(0)
        out["dgamma"] = (dy * n).sum(0)
        dy *= s["gamma"].double()
        along = (dy * n).mean(1, keepdim=True)
        dx = (dy - dy.mean(1, keepdim=True) - n * along) * r
        out["dx"] = dx if s["dh"] is None else dx + s["dh"].double()
    return out


def _exact_adamw(s):
    out = []
    for g in s["groups"]:
        grad = g["g"].double()
        if s["sumsq"] is not None:
            grad *= min(1.0, MAX_NORM / math.sqrt(s["sumsq"].item()))
        if s["case"]["bits"] == 32:
            m, v = g["m"].double(), g["v"].double()
        else:
            m, v = (_values64(*g[n], n == "m") for n in "mv")
        m.mul_(BETA1).add_(grad, alpha=1 - BETA1)
        v.mul_(BETA2).addcmul_(grad, grad, value=1 - BETA2)
        w = g["w"].double()
        w -= LR * DECAY * w
        step = torch.sqrt(v / (1 - BETA2 ** STEP)).add_(EPS)
        w -= LR * (m / (1 - BETA1 ** STEP)) / step
        # 8-bit states are rounded at random: no value in 64 bits
        held = s["case"]["bits"] == 32
        out.append({"w": w, "copy": w if g["copy"] is not None else None,
                    "m": m if held else None, "v": v if held else None})
    return out


def _values64(codes, scales, signed):
    """The values of an 8-bit state by its definition: u (2^k (1 + j / 8) - 1)."""
    c = codes.double()
    neg = (c > 127) if signed else torch.zeros_like(c, dtype=torch.bool)
    c = torch.where(neg, c - 128, c)
    k = torch.floor(c / 8)
    u = torch.exp2(scales.double() - 127).repeat_interleave(BLOCK)
    mag = u * (torch.exp2(k) * (1 + (c - 8 * k) / 8) - 1)
    return torch.where(neg, -mag, mag)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "gnorm":
        return {"sumsq": sum(torch.dot(t, t) for t in (g["g"].double() for g in s["groups"])).view(1)}
    return {"embed": _exact_embed, "norm": _exact_norm, "adamw": _exact_adamw}[case["kind"]](s)

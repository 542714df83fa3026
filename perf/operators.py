"""Performance cases of the operators beside the expert layer's own: the router's
balance loss, distillation through the blockwise vocabulary projection, and the
expert layer's forward in MXFP4 (4-bit values, one 8-bit scale per 32).

  balance  the balance loss, z-loss and per-expert counts of a batch of
           sequences, and the gradient of the router's logits;
  distill  the loss of a student's vocabulary projection against a teacher's
           top logits, and its gradients;
  mxfp4    the expert layer's forward (given the routing) on MXFP4 weights;
  quant    MXFP4 quantisation of a matrix, along its rows (activations) or its
           columns (expert weights), and back to the values it stands for.

`run` computes them in elementary torch operations, or through the Python
binding (paper_2607_01844_amd.moe) where `own` is true.  Sizes are those of
workloads.py, of the tests, and generic ones beside them.
"""
from __future__ import annotations

import math

import torch

own = False

W_STD = 0.02
MXB = 32  # values of one MXFP4 block


# ------------------------------------------------------------------- cases
def _balance(name, T, E, k, groups=1, masked=False):
    return {"name": name, "kind": "balance", "T": T, "E": E, "k": k, "groups": groups,
            "masked": masked}


def _distill(name, N, H, V, K, vblock, tau=1.0, absolute=False):
    return {"name": name, "kind": "distill", "N": N, "H": H, "V": V, "K": K, "vblock": vblock,
            "tau": tau, "absolute": absolute}


def _mxfp4(name, T, d, E, k, f, local=0, skew=0.0):
    return {"name": name, "kind": "mxfp4", "T": T, "d": d, "E": E, "k": k, "f": f,
            "local": local or E, "skew": skew}


def _quant(name, B, R, C, transpose):
    return {"name": name, "kind": "quant", "B": B, "R": R, "C": C, "transpose": transpose}


def listed():
    return [
        # the smallest layer's router: launches and little else
        _balance("balance_tiny", 256, 8, 2),
        # an expert-parallel rank's tokens: ragged packed sequences with padding
        _balance("balance_ep_share", 16384, 384, 8, groups=13, masked=True),
        # the long-context chunk, one sequence
        _balance("balance_long", 65536, 128, 8),
        # the smallest vocabulary of the tests
        _distill("distill_tiny", 256, 128, 1000, 8, 256),
        # odd sizes: vocabulary rows not 16-byte aligned, ragged blocks, softened
        # distributions, teacher probabilities that do not sum to one
        _distill("distill_ragged", 1000, 520, 32003, 20, 4096, tau=2.0, absolute=True),
        # the mid layer's width, a vocabulary of 200,000, 64 teacher logits a token
        _distill("distill_mid", 4096, 2048, 200000, 64, 16384),
        # generation: a handful of tokens against all of a layer's weights
        _mxfp4("mxfp4_decode", 16, 2048, 64, 6, 1408),
        # odd sizes: no dimension a multiple of a block or tile, uneven experts
        _mxfp4("mxfp4_ragged", 1100, 520, 12, 3, 328, skew=1.0),
        # a mid-sized layer: a few hundred rows per expert
        _mxfp4("mxfp4_mid", 4096, 2048, 64, 6, 1408),
        # a large layer's prompt: 512 rows per expert
        _mxfp4("mxfp4_large", 8192, 4096, 128, 8, 1536),
        # activations of odd width, along the rows
        _quant("quant_rows", 1, 1100, 520, False),
        # one weight of every expert of the mid layer, along the contraction
        _quant("quant_weights", 64, 2048, 1408, True),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    """One more case of the listed ranges, at most the largest listed one's
    work."""
    kind = rng.choice(["balance", "balance", "distill", "distill", "mxfp4", "mxfp4", "mxfp4",
                       "quant"])
    while True:
        if kind == "balance":
            E = _log_int(rng, 4, 1024)
            c = _balance("", _log_int(rng, 1, 65536), E, rng.randint(1, min(16, E)),
                         rng.choice([1, 1, 2, 5, 16, 64]), rng.random() < 0.5)
            if c["T"] * E <= 8_400_000:
                break
        elif kind == "distill":
            V = _log_int(rng, 1000, 200000)
            c = _distill("", _log_int(rng, 1, 8192), _log_int(rng, 64, 4096, 8), V,
                         _log_int(rng, 1, 128), _log_int(rng, 256, 32768, 8),
                         rng.choice([1.0, 1.0, 2.0, 0.7]), rng.random() < 0.4)
            if c["N"] * c["H"] * V <= 4e11 and c["H"] * V <= 5e8:
                break
        elif kind == "mxfp4":
            E = rng.choice([8, 12, 16, 32, 64, 96, 128, 384])
            c = _mxfp4("", _log_int(rng, 1, 16384), _log_int(rng, 64, 7168, 8), E,
                       rng.choice([1, 2, 3, 4, 6, 8]), _log_int(rng, 64, 2048, 8),
                       rng.choice([E, E, E // 4]), rng.choice([0.0, 0.0, 1.0]))
            df = c["d"] * c["f"]
            if c["T"] * c["k"] * df <= 2e11 and c["local"] * df <= 6e8:
                break
        else:
            c = _quant("", rng.choice([1, 1, 4, 16]), _log_int(rng, 8, 16384, 8),
                       _log_int(rng, 8, 7168, 8), rng.random() < 0.5)
            if c["B"] * c["R"] * c["C"] <= 180_000_000:
                break
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _normal(shape, std, gen, dtype):
    """N(0, std) of `dtype`, drawn a slice of the first axis at a time."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 28) // max(1, out[:1].numel()))
    for i in range(0, shape[0], step):
        part = out[i:i + step]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(std))
    return out


def _pack(values):
    """(codes, scales) of float32 values [..., rows, K], in the library's layout:
    the codes of an even and the next k in one byte, low half first, rows padded
    with zeros to a multiple of 32; the scales of 256 k together, [..., groups,
    rows, 8], the four of even blocks first."""
    K = values.shape[-1]
    v = torch.nn.functional.pad(values, (0, -K % MXB))
    v = v.reshape(*v.shape[:-1], -1, MXB)
    e = _scale_exponent(v)
    m = _round_e2m1(v * torch.exp2(-e)[..., None])
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=v.device)
    code = torch.searchsorted(grid, m.abs().contiguous()).to(torch.uint8)
    code = (code | (torch.signbit(m).to(torch.uint8) << 3)).flatten(-2)
    q = code[..., 0::2] | (code[..., 1::2] << 4)
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[-1] % 8))
    s = s.reshape(*s.shape[:-1], -1, 4, 2).transpose(-1, -2).flatten(-2)
    return q, s.transpose(-2, -3).contiguous()


def _pack_weights(B, rows, K, gen):
    """MXFP4 weights [B][rows][K] with values ~ N(0, 0.02), a few at a time."""
    step = max(1, (1 << 26) // (rows * K))
    parts = [_pack(_normal((min(step, B - b), rows, K), W_STD, gen, torch.bfloat16).float())
             for b in range(0, B, step)]
    return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    bf = torch.bfloat16
    s = {"case": case}
    dev = "cuda"
    if case["kind"] == "balance":
        T, E, k, G = (case[n] for n in ("T", "E", "k", "groups"))
        # logits spread as those of a trained router, some experts liked more
        s["logits"] = _normal((T, E), 1.3, gen, torch.float32)
        s["logits"] += _normal((1, E), 0.5, gen, torch.float32)
        s["topk_idx"] = s["logits"].topk(k, dim=1).indices.to(torch.int32)
        # packed sequences of any length, none among them
        cuts = torch.randint(0, T + 1, (G - 1,), generator=gen, device=dev).sort().values
        ends = torch.tensor([0, T], device=dev)
        s["seq_offsets"] = torch.cat([ends[:1], cuts, ends[1:]]).to(torch.int32)
        s["token_mask"] = None
        if case["masked"]:
            s["token_mask"] = torch.rand((T,), generator=gen, device=dev) < 0.9
        s["dbalance"] = torch.full((G,), 0.01 / G, device=dev)
        s["dzloss"] = torch.full((G,), 0.001 / G, device=dev)
        return s
    if case["kind"] == "distill":
        N, H, V, K = (case[n] for n in ("N", "H", "V", "K"))
        s["x"] = _normal((N, H), 1.0, gen, bf)
        s["w_voc"] = _normal((H, V), W_STD, gen, bf)
        # distinct vocabulary entries a token, low ones (frequent words) more often
        u = torch.rand((N, K), generator=gen, device=dev)
        ids = (u.pow(3) * (V - K)).to(torch.int64).sort(1).values + torch.arange(K, device=dev)
        order = torch.rand((N, K), generator=gen, device=dev).argsort(1)
        ids = ids.gather(1, order).to(torch.int32)
        t = _normal((N, K), 2.0, gen, torch.float32).sort(1, descending=True).values
        # a teacher that keeps a share of its probability gives few logits; some
        # tokens (padding) have none
        have = torch.randint(1, K + 1, (N, 1), generator=gen, device=dev)
        have *= torch.rand((N, 1), generator=gen, device=dev) > 0.06
        s["topk_idx"] = torch.where(torch.arange(K, device=dev) < have, ids, -1).contiguous()
        s["topk_logit"] = t.contiguous()
        s["teacher_lse"] = None
        if case["absolute"]:
            s["teacher_lse"] = (t / case["tau"]).logsumexp(1) + \
                torch.rand((N,), generator=gen, device=dev)
        s["dloss"] = torch.full((N,), 1.0 / N, device=dev)  # of a mean over the tokens
        return s
    if case["kind"] == "quant":
        shape = (case["B"], case["R"], case["C"])
        s["src"] = _normal(shape, W_STD if case["transpose"] else 1.0, gen, bf)
        return s
    T, d, E, k, f, local = (case[n] for n in ("T", "d", "E", "k", "f", "local"))
    s["x"] = _normal((T, d), 1.0, gen, bf)
    score = torch.randn((T, E), generator=gen, device=dev)
    score -= case["skew"] * torch.rand((E,), generator=gen, device=dev)
    top = score.topk(k, dim=1)
    s["topk_idx"] = top.indices.to(torch.int32)
    s["topk_gate"] = torch.softmax(top.values, dim=1)
    s["w_gate"] = _pack_weights(local, f, d, gen)
    s["w_up"] = _pack_weights(local, f, d, gen)
    s["w_down"] = _pack_weights(local, d, f, gen)
    # the rows of the fullest local expert: what a padded batch is sized by
    s["most"] = int(torch.bincount(top.indices.flatten(), minlength=E)[:local].max())
    return s


# ------------------------------------------------------- elementary forms
def _scale_exponent(v):
    """floor(log2(max |v|)) - 2 over the last axis, in [-127, 127] (floats)."""
    e = torch.frexp(v.abs().amax(-1)).exponent - 3
    return e.clamp(-127, 127).to(v.dtype)


def _round_e2m1(v):
    """To the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (ties to the even code)."""
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).to(v.dtype)
    return torch.copysign((torch.round(a / step) * step).clamp(max=6.0), v)


def _mx_values(v):
    """What the MXFP4 form of `v` [..., K] stands for."""
    K = v.shape[-1]
    b = torch.nn.functional.pad(v, (0, -K % MXB)).reshape(*v.shape[:-1], -1, MXB)
    sc = torch.exp2(_scale_exponent(b))[..., None]
    return (_round_e2m1(b / sc) * sc).flatten(-2)[..., :K]


def _unpack(w, K, dtype=torch.float32):
    """The values of MXFP4 codes and scales (see _pack)."""
    q, s = w
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=dtype, device=q.device)
    grid = torch.cat([grid, -grid])
    v = grid[torch.stack([q & 15, q >> 4], -1).flatten(-2).int()]
    e = s.transpose(-2, -3).to(dtype) - 127
    e = e.reshape(*e.shape[:-1], 2, 4).transpose(-1, -2).flatten(-3)[..., :v.shape[-1] // MXB]
    v = v.reshape(*v.shape[:-1], -1, MXB) * torch.exp2(e)[..., None]
    return v.flatten(-2)[..., :K]


def _run_balance(s):
    case, logits, idx = s["case"], s["logits"], s["topk_idx"].long()
    T, E, k, G = (case[n] for n in ("T", "E", "k", "groups"))
    off = s["seq_offsets"].long()
    tok = torch.arange(T, device=logits.device)
    member = (tok >= off[:-1, None]) & (tok < off[1:, None])  # [G, T]
    if s["token_mask"] is not None:
        member &= s["token_mask"]
    mf = member.float()
    n = member.sum(1)
    group = torch.searchsorted(off[1:], tok, right=True).clamp(max=G - 1)
    valid = mf.sum(0)
    counts = torch.zeros(G * E, dtype=torch.int64, device=logits.device)
    counts.scatter_add_(0, (group[:, None] * E + idx).flatten(),
                        valid.long()[:, None].expand(-1, k).flatten())
    counts = counts.view(G, E)
    m = logits.amax(1, keepdim=True)
    ex = torch.exp(logits - m)
    den = ex.sum(1, keepdim=True)
    p = ex / den
    lse = (m + torch.log(den))[:, 0]
    prob_sum = mf @ p
    nf = n.clamp(min=1).float()
    a = counts * (E / k) / nf[:, None]
    balance = (a * prob_sum).sum(1) / nf
    zloss = (mf @ (lse * lse)[:, None])[:, 0] / nf
    at = a[group]
    db, dz = (s["dbalance"] / nf)[group] * valid, (s["dzloss"] / nf)[group] * valid
    inner = (at * p).sum(1, keepdim=True)
    dlogits = p * (db[:, None] * (at - inner) + 2 * (dz * lse)[:, None])
    return {"balance": balance, "zloss": zloss, "counts": counts.int(), "prob_sum": prob_sum,
            "n_tokens": n.int(), "dlogits": dlogits}


def _teacher(s):
    """Teacher probabilities [N, K] (0 where a slot is absent) and their logs."""
    there = s["topk_idx"] >= 0
    t = torch.where(there, s["topk_logit"] / s["case"]["tau"], -math.inf)
    if s["teacher_lse"] is not None:
        logp = t - s["teacher_lse"][:, None]
    else:
        m = torch.where(there.any(1), t.amax(1), 0.0)[:, None]
        logp = t - m - torch.log(torch.exp(t - m).sum(1, keepdim=True))
    logp = torch.where(there, logp, 0.0)
    return torch.where(there, torch.exp(logp), 0.0), logp


def _run_distill(s):
    tau = s["case"]["tau"]
    x, w = s["x"].float(), s["w_voc"].float()
    p, logp = _teacher(s)
    ids = s["topk_idx"].long().clamp(min=0)
    there = s["topk_idx"] >= 0
    y = x @ w
    y_topk = torch.where(there, y.gather(1, ids), 0.0)
    y /= tau
    m = y.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(y - m).sum(1, keepdim=True)))[:, 0]
    loss = (p * (logp - y_topk / tau + lse[:, None])).sum(1)
    dl = s["dloss"] / tau
    G = torch.exp(y - lse[:, None]) * (dl * p.sum(1))[:, None]
    G.scatter_add_(1, ids, -p * dl[:, None])
    return {"loss": loss, "lse": lse, "y_topk": y_topk, "dx": (G @ w.t()).bfloat16(),
            "dw_voc": (x.t() @ G).bfloat16()}


def _run_mxfp4(s):
    T, d, E, k, f, local = (s["case"][n] for n in ("T", "d", "E", "k", "f", "local"))
    most = s["most"]
    flat = s["topk_idx"].flatten().long()
    order = torch.argsort(flat, stable=True)
    counts = torch.zeros(E, dtype=torch.int64, device=flat.device)
    counts.scatter_add_(0, flat, torch.ones_like(flat))
    start = counts.cumsum(0) - counts
    # [local, most] assignments, the experts' rows padded to the fullest one's
    pos = torch.arange(most, device=flat.device)
    there = pos < counts[:local, None]
    a = order[(start[:local, None] + pos).clamp(max=T * k - 1)]
    xe = torch.where(there[..., None], _mx_values(s["x"].float())[a // k], 0.0)
    g = torch.bmm(xe, _unpack(s["w_gate"], d).transpose(1, 2).contiguous())
    u = torch.bmm(xe, _unpack(s["w_up"], d).transpose(1, 2).contiguous())
    act = _mx_values(g / (1 + torch.exp(-g)) * u)
    y = torch.bmm(act, _unpack(s["w_down"], f).transpose(1, 2).contiguous())
    gate = torch.where(there, s["topk_gate"].flatten()[a], 0.0)
    out = torch.zeros((T, d), device=flat.device)
    out.index_add_(0, (a // k).flatten(), (y * gate[..., None]).flatten(0, 1))
    return {"y": out.bfloat16()}


def _run_quant(s):
    v = s["src"].float()
    if s["case"]["transpose"]:
        v = v.transpose(1, 2).contiguous()
    return {"values": _mx_values(v).bfloat16()}


# --------------------------------------------------------- framework calls
def _own_balance(s, moe):
    seq, mask = s["seq_offsets"], s["token_mask"]
    bal, z, counts, prob_sum, n = moe.moe_balance_loss_fwd(s["logits"], s["topk_idx"], seq, mask)
    dl = moe.moe_balance_loss_bwd(s["logits"], counts, n, s["dbalance"], s["dzloss"],
                                  s["case"]["k"], seq, mask)
    return {"balance": bal, "zloss": z, "counts": counts, "prob_sum": prob_sum, "n_tokens": n,
            "dlogits": dl}


def _own_distill(s, moe):
    a = (s["x"], s["w_voc"], s["topk_idx"], s["topk_logit"])
    vb, tau, tl = s["case"]["vblock"], s["case"]["tau"], s["teacher_lse"]
    loss, lse, y_topk = moe.moe_vocab_distill_fwd(*a, vb, tau, tl)
    dx, dw = moe.moe_vocab_distill_bwd(*a, lse, y_topk, s["dloss"], vb, tau, tl)
    return {"loss": loss, "lse": lse, "y_topk": y_topk, "dx": dx, "dw_voc": dw}


def _own_mxfp4(s, moe):
    return {"y": moe.moe_ffn_fwd_mxfp4(s["x"], s["topk_idx"], s["topk_gate"], s["case"]["E"],
                                       s["w_gate"], s["w_up"], s["w_down"])}


def _own_quant(s, moe):
    q, sc = moe.moe_mxfp4_quantize(s["src"], transpose=s["case"]["transpose"])
    K = s["case"]["R"] if s["case"]["transpose"] else s["case"]["C"]
    return {"values": moe.moe_mxfp4_dequantize(q, sc, K)}


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2607_01844_amd import moe
        return {"balance": _own_balance, "distill": _own_distill, "mxfp4": _own_mxfp4,
                "quant": _own_quant}[kind](state, moe)
    return {"balance": _run_balance, "distill": _run_distill, "mxfp4": _run_mxfp4,
            "quant": _run_quant}[kind](state)


# ------------------------------------------------------------------- floors
def work(case):
    """Bytes: every input read once, every output written once (weights of
    experts that get a row); flops: the products, and of the vocabulary logits
    one recomputation, which a backward that is not given them needs."""
    if case["kind"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": 12 * T * E + 4 * T * k, "flops": 20 * T * E}
    if case["kind"] == "distill":
        N, H, V, K = (case[n] for n in ("N", "H", "V", "K"))
        return {"bytes": 2 * (2 * N * H + 2 * H * V) + 12 * N * K + 16 * N,
                "flops": 8 * N * H * V}
    if case["kind"] == "quant":
        n = case["B"] * case["R"] * case["C"]
        # in, codes and scales out and in again, values out
        return {"bytes": int(2 * n + 2 * n * 17 / 32 + 2 * n), "flops": 4 * n}
    T, d, E, k, f, local = (case[n] for n in ("T", "d", "E", "k", "f", "local"))
    used = local * (1 - (1 - k / E) ** T)  # experts expected to have rows
    return {"bytes": int(3 * used * d * f * 17 / 32 + 4 * T * d + 8 * T * k),
            "flops": int(6 * T * k * local / E * d * f)}


# ------------------------------------------------------- 64-bit reference
def _q64(v):
    """MXFP4 values of float64 [..., K], by comparison with the midpoints."""
    out = torch.zeros_like(v)
    for b in range(0, v.shape[-1], MXB):
        x = v[..., b:b + MXB]
        top = x.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140)))
        e = torch.where(torch.exp2(e) > top, e - 1, torch.where(torch.exp2(e + 1) <= top, e + 1, e))
        sc = torch.exp2((e - 2).clamp(-127, 127))
        m = x.abs() / sc
        r = torch.zeros_like(m)
        # upper neighbour taken above the midpoint, at it where its code is even
        for up, mid, even in ((0.5, 0.25, False), (1.0, 0.75, True), (1.5, 1.25, False),
                              (2.0, 1.75, True), (3.0, 2.5, False), (4.0, 3.5, True),
                              (6.0, 5.0, False)):
            r = torch.where(m >= mid if even else m > mid, up, r)
        out[..., b:b + MXB] = torch.copysign(r * sc, x)
    return out


def _exact_balance(s):
    case, E, k = s["case"], s["case"]["E"], s["case"]["k"]
    y = s["logits"].double()
    lse = torch.logsumexp(y, 1)
    p = torch.softmax(y, 1)
    off = s["seq_offsets"].tolist()
    ok = torch.ones(case["T"], dtype=torch.bool, device=y.device)
    if s["token_mask"] is not None:
        ok = s["token_mask"]
    out = {"balance": [], "zloss": [], "prob_sum": []}
    dl = torch.zeros_like(y)
    for g in range(case["groups"]):
        rows = torch.arange(off[g], off[g + 1], device=y.device)
        rows = rows[ok[rows]]
        n = max(1, rows.numel())
        f = torch.bincount(s["topk_idx"][rows].flatten().long(), minlength=E).double() * E / (k * n)
        out["prob_sum"].append(p[rows].sum(0))
        out["balance"].append((f * p[rows]).sum() / n)
        out["zloss"].append(lse[rows].square().sum() / n)
        up = f * s["dbalance"][g].double() / n
        dl[rows] = p[rows] * (up - (p[rows] @ up)[:, None]
                              + 2 * s["dzloss"][g].double() / n * lse[rows, None])
    return {n: torch.stack(v) for n, v in out.items()} | {"counts": None, "n_tokens": None,
                                                          "dlogits": dl}


def _exact_distill(s):
    case, tau = s["case"], s["case"]["tau"]
    x, w = s["x"].double(), s["w_voc"].double()
    ids = s["topk_idx"].long()
    t = s["topk_logit"].double() / tau
    t[ids < 0] = -math.inf
    if s["teacher_lse"] is None:
        p = torch.nan_to_num(torch.softmax(t, 1))
    else:
        p = torch.exp(t - s["teacher_lse"].double()[:, None])
    y = x @ w
    rows = torch.arange(case["N"], device=y.device)[:, None]
    y_topk = torch.where(ids < 0, 0.0, y[rows, ids])
    y /= tau
    lse = torch.logsumexp(y, 1)
    loss = (torch.xlogy(p, p) - p * (y_topk / tau - lse[:, None])).sum(1)
    dl = s["dloss"].double()[:, None] / tau
    G = y.sub_(lse[:, None]).exp_().mul_(dl * p.sum(1, keepdim=True))
    G.index_put_((rows.expand_as(ids), ids.clamp(min=0)), -dl * p, accumulate=True)
    return {"loss": loss, "lse": lse, "y_topk": y_topk, "dx": G @ w.t(), "dw_voc": x.t() @ G}


def _exact_mxfp4(s):
    T, d, k, f, local = (s["case"][n] for n in ("T", "d", "k", "f", "local"))
    x = _q64(s["x"].double())
    idx, gate = s["topk_idx"].long(), s["topk_gate"].double()
    y = torch.zeros((T, d), dtype=torch.float64, device=x.device)
    w = [s[n] for n in ("w_gate", "w_up", "w_down")]
    for e in range(local):
        t, i = torch.nonzero(idx == e, as_tuple=True)
        if t.numel() == 0:
            continue
        wg, wu, wd = (_unpack((q[e], sc[e]), n, torch.float64)
                      for (q, sc), n in zip(w, (d, d, f)))
        hg, hu = x[t] @ wg.t(), x[t] @ wu.t()
        y.index_add_(0, t, (_q64(hg * torch.sigmoid(hg) * hu) @ wd.t()) * gate[t, i][:, None])
    return {"y": y}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quant":
        v = s["src"].double()
        return {"values": _q64(v.transpose(1, 2).contiguous() if case["transpose"] else v)}
    return {"balance": _exact_balance, "distill": _exact_distill,
            "mxfp4": _exact_mxfp4}[case["kind"]](s)

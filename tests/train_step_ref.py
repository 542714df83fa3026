"""Plain references of the embedding, the layer norm and the AdamW update, in
64 bits on the CPU (torch), and the 8-bit states' format in 32-bit arithmetic
(numpy, which rounds every operation), from their definitions in moe.h."""
import numpy as np
import torch

U = 2.0 ** -24   # half a step of fp32, relative to the value
UB = 2.0 ** -8   # of bf16


def f64(t):
    return t.detach().to("cpu", torch.float64)


# --------------------------------------------------------------- embedding
def embed(ids, w, scale, begin):
    """y of the embedding; ids, w on the CPU."""
    rows = w.shape[0]
    y = torch.zeros((ids.numel(), w.shape[1]), dtype=w.dtype)
    for t, i in enumerate(ids.tolist()):
        if begin <= i < begin + rows:
            y[t] = w[i - begin] * scale
    return y


def embed_bwd(ids, dy, rows, scale, begin):
    """(dw, sum of |dy| of each element, tokens of each row), scaled."""
    dw = torch.zeros((rows, dy.shape[1]), dtype=torch.float64)
    mass, n = torch.zeros_like(dw), torch.zeros(rows, 1, dtype=torch.float64)
    for t, i in enumerate(ids.tolist()):
        if begin <= i < begin + rows:
            dw[i - begin] += dy[t]
            mass[i - begin] += dy[t].abs()
            n[i - begin] += 1
    return dw * scale, mass * abs(scale), n


# -------------------------------------------------------------- layer norm
def norm(h, gamma, beta, eps):
    """(y, mean, rstd) of rows h."""
    mean = h.mean(1, keepdim=True)
    var = ((h - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    return (h - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def norm_bwd(dy, h, gamma, mean, rstd, dh):
    """(dx, dgamma, dbeta) given the forward's statistics."""
    xh = (h - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx + dh, (dy * xh).sum(0), dy.sum(0)


# ------------------------------------------------------------------- AdamW
def adamw(w, g, m, v, lr, t, b1, b2, eps, wd, clip=1.0):
    """(w', m', v')."""
    g = g * clip
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    u = m / (1 - b1 ** t) / (torch.sqrt(v / (1 - b2 ** t)) + eps)
    return w - lr * wd * w - lr * u, m, v


# ----------------------------------------------------- states held in 8 bits
BLOCK = 128
SPAN = {"m": 14, "v": 30}


def mix(x, q):
    x = np.asarray(x, dtype=np.uint64) & 0xFFFFFFFF
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(q)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(15))


def random_bits(n, seed, t, j):
    """r of the elements 0 .. n - 1 of tensor j of a list, at step t."""
    key = (seed + 0x85A308D3 * t + 0x9E3779B9 * j) & 0xFFFFFFFF
    key = mix(mix(key, 0x6A09E667), 0xBB67AE85)
    i = np.arange(n, dtype=np.uint64) & np.uint64(0xFFFFFFFF)
    return mix(i * np.uint64(0x9E3779B9) + key, 0x6A09E667)


def decode(codes, scales, kind):
    """fp32 values of codes [n] and scales [ceil(n / 128)] (uint8 arrays)."""
    c = codes.astype(np.uint32)
    s = np.repeat(scales.astype(np.uint32), BLOCK)[:c.size] << np.uint32(23)
    u = s.view(np.float32)
    mag = c & np.uint32(127) if kind == "m" else c
    with np.errstate(invalid="ignore"):
        x = ((mag << np.uint32(20)) + s).view(np.float32) - u
    return np.where(c > 127, -x, x).astype(np.float32) if kind == "m" else x


def encode(x, kind, r16):
    """(codes, scales) of fp32 x [n] with random bits r16 [n]."""
    n = x.size
    pad = np.zeros(-(-n // BLOCK) * BLOCK, dtype=np.float32)
    pad[:n] = x
    top = (np.abs(pad).view(np.uint32).reshape(-1, BLOCK).max(1) >> np.uint32(23)).astype(np.int64)
    s = np.where(top == 255, 255, np.maximum(top - SPAN[kind], 1))
    se = np.repeat(s, BLOCK)[:n].astype(np.uint32)
    u = (se << np.uint32(23)).view(np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        y = (np.abs(x) + u).view(np.uint32).astype(np.int64)
        c = ((y + (r16.astype(np.int64) << 4) + 8) >> 20) - (se.astype(np.int64) << 3)
        c = c | ((x.view(np.uint32) >> 31).astype(np.int64) << 7) if kind == "m" else \
            np.maximum(c, x > 0)
    c = np.where(se == 255, 0, c)
    return c.astype(np.uint8), s.astype(np.uint8)


def states32(m, v, g, b1, b2, clip=np.float32(1)):
    """m', v' in fp32, every operation rounded (all arrays fp32)."""
    f = np.float32
    x = g * f(clip)
    return f(b1) * m + f(1 - b1) * x, f(b2) * v + f(1 - b2) * (x * x)

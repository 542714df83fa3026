"""MXFP4 in plain torch on the CPU, 64 bits (the tests' reference): the format's
packing and unpacking, quantisation by comparison with the midpoints between
code values, and the grouped SwiGLU forward with bounds on its error."""
import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
U = 2.0 ** -24


def blocks(v):
    """[..., K] -> [..., ceil(K/32), 32], zeros at the end."""
    K = v.shape[-1]
    v = torch.nn.functional.pad(v, (0, -K % 32))
    return v.reshape(*v.shape[:-1], -1, 32)


def scale_byte(b):
    """Scale byte of each block [..., 32] of finite or non-finite float64."""
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    e = torch.frexp(torch.where(bad, 1.0, top)).exponent - 1  # floor(log2)
    e = torch.where(top == 0, -127, (e - 2).clamp(-127, 127)).to(torch.int64)
    return torch.where(bad, 255, e + 127)


def encode(v, byte):
    """Codes of blocks [..., 32] at a scale byte each (NaN blocks: code 0)."""
    a = v.abs() / torch.exp2(byte.double() - 127)[..., None]
    c = torch.zeros(a.shape, dtype=torch.int64)
    # code c + 1 from the midpoint above code c: at it where c + 1 is even
    for lo in range(7):
        mid = (GRID[lo] + GRID[lo + 1]) / 2
        c += (a >= mid) if lo % 2 == 1 else (a > mid)
    c |= torch.signbit(v).to(torch.int64) << 3
    return torch.where((byte == 255)[..., None], 0, c)


def decode(codes, byte):
    v = GRID[codes & 7] * torch.where(codes >= 8, -1.0, 1.0)
    v = v * torch.exp2(byte.double() - 127)[..., None]
    return torch.where((byte == 255)[..., None], torch.nan, v)


def pack(codes, byte):
    """(q, s) of codes [B][rows][nb][32] and scale bytes [B][rows][nb]."""
    c = codes.flatten(-2)
    q = (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)
    nb = byte.shape[-1]
    s = torch.zeros((*byte.shape[:-1], -(-nb // 8) * 8), dtype=torch.uint8)
    for b in range(nb):
        s[..., b // 8 * 8 + b % 2 * 4 + b % 8 // 2] = byte[..., b].to(torch.uint8)
    s = s.reshape(*byte.shape[:-1], -1, 8).transpose(-2, -3).contiguous()
    return q, s


def quantize(v):
    """(q, s, values) of float64 [B][rows][K]."""
    K = v.shape[-1]
    b = blocks(v)
    byte = scale_byte(b)
    codes = encode(b, byte)
    q, s = pack(codes, byte)
    return q, s, decode(codes, byte).flatten(-2)[..., :K]


def values(v):
    return quantize(v)[2]


def act_bounds(a, ea):
    """(values of a [rows][f] after quantisation, how far each may be off when a
    is known to +- ea only): the block's scale from its magnitude less or more
    the error, each value from a less or more its own."""
    f = a.shape[-1]
    b, e = blocks(a), blocks(ea)
    byte = scale_byte(b)
    mid = decode(encode(b, byte), byte)
    off = torch.zeros_like(mid)
    for sb in (scale_byte((b.abs() - e).clamp(min=0)), scale_byte(b.abs() + e)):
        for v in (b - e, b, b + e):
            off = torch.maximum(off, (decode(encode(v, sb), sb) - mid).abs())
    return mid.flatten(-2)[..., :f], off.flatten(-2)[..., :f]


def swiglu(x, wg, wu, wd):
    """(y, bound) of rows x [n][d] (values) against wg, wu [f][d], wd [d][f]
    (values): the result before its rounding to bf16, and how far a kernel of
    fp32 sums may be from it before its own."""
    d, f = x.shape[1], wd.shape[1]
    g, u = x @ wg.t(), x @ wu.t()
    eg = d * U * (x.abs() @ wg.abs().t())
    eu = d * U * (x.abs() @ wu.abs().t())
    sg = torch.sigmoid(g)
    a = g * sg * u
    # |silu'| <= 1.1; sigmoid by a hardware exponential and reciprocal, 2^-20
    ea = 1.1 * eg * (u.abs() + eu) + (g * sg).abs() * eu + a.abs() * 2.0 ** -20 + 2.0 ** -140
    av, off = act_bounds(a, ea)
    y = av @ wd.t()
    return y, off @ wd.abs().t() + f * U * ((av.abs() + off) @ wd.abs().t())


def close(got, ref, bound):
    """A bf16 result within `bound` of ref before its rounding (half a step)."""
    got = got.double()
    return ((got - ref).abs() <= bound + 2.0 ** -8 * (ref.abs() + bound) + 2.0 ** -134).all()

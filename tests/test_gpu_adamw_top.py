"""8-bit states at the upper end of fp32: what is finite stays finite when it is
held, bit for bit against 32-bit arithmetic."""
import numpy as np
import pytest
import torch

from tests import train_step_ref as R

pytestmark = pytest.mark.gpu

TOP = float(np.finfo(np.float32).max)
EDGE = 1.875 * 2.0 ** 127  # from here on the nearest code would stand for 2^128


def encode(x, kind, r16):
    """(codes, scales) of fp32 x: as in 32-bit arithmetic, but no code above the last
    that stands for a finite value, 8 (255 - s) - 1."""
    codes, scales = R.encode(x, kind, r16)
    last = 8 * (255 - np.repeat(scales.astype(np.int64), R.BLOCK)[:x.size]) - 1
    sign = codes & 128 if kind == "m" else 0
    mag = (codes & 127 if kind == "m" else codes).astype(np.int64)
    mag = np.where(last < 0, mag, np.minimum(mag, last))
    return (mag | sign).astype(np.uint8), scales


def by_definition(codes, scales, kind):
    c = codes.astype(np.int64)
    mag = c & 127 if kind == "m" else c
    u = 2.0 ** (np.repeat(scales.astype(float), R.BLOCK)[:c.size] - 127)
    x = u * (2.0 ** (mag // 8) * (1 + mag % 8 / 8.0) - 1)
    # 2^k (1 + j / 8) - 1, k < 31, has 31 bits at most: exact in 64 bits, and the fp32
    # difference that reads a code rounds that value once
    return (np.where(c > 127, -x, x) if kind == "m" else x).astype(np.float32)


def values(seed):
    """Blocks whose largest lies beyond, at and below EDGE, in the octave below, and
    far below; ends inside a block."""
    rng = np.random.default_rng(seed)
    x = rng.random(6 * 128 + 77) * 2.0 ** rng.integers(-20, 1, 6 * 128 + 77)
    for i, top in enumerate((TOP, EDGE, np.nextafter(np.float32(EDGE), np.float32(0)), 2.0 ** 127,
                             np.nextafter(np.float32(2.0 ** 127), np.float32(0)), 1.0, TOP)):
        x[128 * i:128 * (i + 1)] *= float(top) * 0.99
        x[128 * i + 5:128 * i + 25] = float(top)
    return x


@pytest.mark.parametrize("kind", ["m", "v"])
@pytest.mark.parametrize("seed", range(3))
def test_finite_states_are_held_as_finite(kind, seed):
    from paper_2607_01844_amd import moe
    x = values(seed)
    if kind == "m":  # m' is the gradient itself
        x[::3] *= -1
        g, beta1, beta2 = x.astype(np.float32), 0.0, 0.95
    else:            # v' its square, below 2^128
        g, beta1, beta2 = np.minimum(np.sqrt(x), np.sqrt(TOP) * (1 - 1e-7)).astype(np.float32), 0.9, 0.0
    n = g.size
    p = moe.Params([torch.zeros(n, device="cuda")], [torch.from_numpy(g).cuda()], bits=8)
    z = np.zeros(n, dtype=np.float32)
    held = {"m": z, "v": z}
    for step in (1, 2, 3):
        with np.errstate(over="ignore", invalid="ignore"):
            m32, v32 = R.states32(held["m"], held["v"], g, beta1, beta2)
        now = m32 if kind == "m" else v32
        assert np.isfinite(now).all()
        r = R.random_bits(n, seed, step, 0)
        codes, scales = encode(now, kind, r & np.uint64(0xFFFF) if kind == "m" else r >> np.uint64(16))
        moe.moe_adamw_step(p, 0.0, step, beta1, beta2, 1e-8, 0.0, seed=seed)
        got = [t.cpu().numpy() for t in getattr(p, kind)[0]]
        assert np.array_equal(got[1], scales), step
        assert np.array_equal(got[0], codes), step
        value = moe.moe_adamw_states(p)["mv".index(kind)][0].cpu().numpy()
        assert np.isfinite(value).all() and np.array_equal(value, by_definition(codes, scales, kind))
        # a step of a segment is an eighth of |x| + u at most; beyond the last code 2^124
        # of 1.875 * 2^127 are lost, less than that
        u = 2.0 ** (np.repeat(scales.astype(float), 128)[:n] - 127)
        assert (np.abs(value.astype(float) - now) <= (np.abs(now.astype(float)) + u) / 8 * (1 + 1e-6)).all()
        held[kind] = value
        if kind == "m":
            beta1 = 0.5
        else:
            beta2 = 0.5

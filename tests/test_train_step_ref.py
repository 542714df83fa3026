"""The references themselves: gradients against differences, the update against
its textbook form, the 8-bit format's steps, range and mean."""
import numpy as np
import pytest
import torch

from tests import train_step_ref as R


def test_embedding_gradient_is_the_forwards_transpose():
    g = torch.Generator().manual_seed(0)
    ids = torch.tensor([3, 5, 3, -1, 9, 4, 3])
    w = torch.randn((4, 6), generator=g, dtype=torch.float64)
    dy = torch.randn((7, 6), generator=g, dtype=torch.float64)
    dw, mass, n = R.embed_bwd(ids, dy, 4, 1.5, 3)
    assert torch.allclose((R.embed(ids, w, 1.5, 3) * dy).sum(), (w * dw).sum())
    assert n[:, 0].tolist() == [3, 1, 1, 0] and (mass >= dw.abs() - 1e-12).all()


def test_norm_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    h, gamma, beta, dy, dh = n(3, 8), n(8), n(8), n(3, 8), n(3, 8)

    def loss(h, gamma, beta):
        return (R.norm(h, gamma, beta, 1e-3)[0] * dy).sum() + (h * dh).sum()
    y, mean, rstd = R.norm(h, gamma, beta, 1e-3)
    dx, dgamma, dbeta = R.norm_bwd(dy, h, gamma, mean, rstd, dh)
    d = 1e-6
    for x, dxx, at in ((h, dx, 0), (gamma, dgamma, 1), (beta, dbeta, 2)):
        for i in range(x.numel()):
            a = [h.clone(), gamma.clone(), beta.clone()]
            b = [h.clone(), gamma.clone(), beta.clone()]
            a[at].view(-1)[i] += d
            b[at].view(-1)[i] -= d
            # central differences: an error of d^2 and of rounding over 2 d
            assert abs((loss(*a) - loss(*b)) / (2 * d) - dxx.view(-1)[i]) < 1e-7


def test_adamw_first_step_moves_by_the_learning_rate():
    w, g = torch.zeros(3, dtype=torch.float64), torch.tensor([2.0, -0.1, 0.0], dtype=torch.float64)
    w1, m, v = R.adamw(w, g, 0 * w, 0 * w, 0.01, 1, 0.9, 0.99, 1e-12, 0.1)
    assert torch.allclose(w1, -0.01 * torch.sign(g), atol=1e-10)
    assert torch.allclose(m, 0.1 * g) and torch.allclose(v, 0.01 * g * g)


@pytest.mark.parametrize("kind", ["m", "v"])
def test_every_code_decodes_and_encodes_to_itself(kind):
    # 2^k (1 + j / 8) - 1 units, exact in fp32 while it needs 24 bits at most
    codes = np.arange(128 if kind == "m" else 176, dtype=np.uint8)
    scale = np.array([100], dtype=np.uint8)
    k, j = codes // 8, codes % 8
    x = np.concatenate([R.decode(codes[i:i + 128], scale, kind) for i in (0, 128)])
    assert np.array_equal(x, (2.0 ** k * (1 + j / 8.0) - 1) * 2.0 ** (100 - 127))
    # alone with the block's largest value, whatever the random bits are
    top = np.float32(2.0 ** (100 - 127 + R.SPAN[kind]))
    for c, v in zip(codes[:8 * 15], x):
        for r in (0, 1, 0xFFFF):
            got, s = R.encode(np.array([v, top], dtype=np.float32), kind, np.full(2, r))
            assert s[0] == 100 and got[0] == c


@pytest.mark.parametrize("kind", ["m", "v"])
def test_encoding_is_right_in_the_mean_and_within_a_step(kind):
    rng = np.random.default_rng(2)
    n = 1 << 16
    x = (rng.standard_normal(n) * np.exp(2 * rng.standard_normal(n))).astype(np.float32)
    if kind == "v":
        x = x * x
    r = R.random_bits(n, 7, 11, 3)
    c, s = R.encode(x, kind, (r & np.uint64(0xFFFF)) if kind == "m" else r >> np.uint64(16))
    got = R.decode(c, s, kind).astype(np.float64)
    u = 2.0 ** (np.repeat(s, 128).astype(float) - 127)
    # a step is an eighth of the segment's width, at most (|x| + u) / 8
    step = (np.abs(x) + u) / 8
    assert (np.abs(got - x) <= step * (1 + 1e-6)).all()
    # errors over steps have mean 0 and variance at most 1 / 4: six sigma
    e = (got - x) / step
    if kind == "v":
        e = e[c > 1]  # the smallest values are held as the first code
    assert abs(e.mean()) < 6 * 0.5 / np.sqrt(e.size)


def test_special_blocks():
    z = np.zeros(3, dtype=np.float32)
    for kind in "mv":
        c, s = R.encode(z, kind, np.full(3, 0xFFFF))
        assert not R.decode(c, s, kind).any()
        assert not R.decode(np.zeros(3, np.uint8), np.zeros(1, np.uint8), kind).any()
        for bad in (np.inf, np.nan):
            c, s = R.encode(np.array([1, bad, 2], dtype=np.float32), kind, np.zeros(3))
            assert s[0] == 255 and np.isnan(R.decode(c, s, kind)).all()
    # a v above 0 is never held as 0
    c, s = R.encode(np.array([1e-30, 1.0], dtype=np.float32), "v", np.zeros(2))
    assert c[0] == 1


def test_random_bits_are_even_and_apart():
    n = 1 << 18
    for seed, t, j in ((0, 1, 0), (0, 2, 0), (5, 1, 9)):
        r = R.random_bits(n, seed, t, j)
        m, v = (r & np.uint64(0xFFFF)).astype(float), (r >> np.uint64(16)).astype(float)
        w = ((r * np.uint64(0xBB67AE85) & np.uint64(0xFFFFFFFF)) >> np.uint64(16)).astype(float)
        cols = [m, v, w, np.roll(m, 1), np.roll(v, 1)]
        cols += [x for s in (1, 2) for x in
                 [(R.random_bits(n, seed, t + s, j) & np.uint64(0xFFFF)).astype(float)]]
        z = np.stack([(x - 32767.5) / 18918.6 for x in cols])
        # means and correlations of n even values: six sigma
        assert np.abs(z.mean(1)).max() < 6 / np.sqrt(n)
        c = z @ z.T / n - np.eye(len(cols))
        assert np.abs(c - np.diag(np.diag(c))).max() < 6 / np.sqrt(n)

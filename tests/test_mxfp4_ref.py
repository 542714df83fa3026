"""The MXFP4 reference against the format's definition (CPU)."""
import torch

from tests import mxfp4_ref as R


def test_every_code_is_its_own_nearest():
    for byte in (0, 1, 100, 127, 200, 252):
        v = R.decode(torch.arange(16)[None], torch.tensor([byte]))
        c = R.encode(v, torch.tensor([byte]))
        assert torch.equal(c[0], torch.arange(16))


def test_nearest_and_ties_to_even():
    g = R.GRID
    for lo in range(7):
        mid = (g[lo] + g[lo + 1]) / 2
        v = torch.stack([mid * (1 - 1e-12), mid, mid * (1 + 1e-12)])[None]
        c = R.encode(v, torch.tensor([127]))[0].tolist()
        assert c == [lo, lo if lo % 2 == 0 else lo + 1, lo + 1]
    assert R.encode(torch.tensor([[7.9, -100.0]]).double(), torch.tensor([127])).tolist() == [[7, 15]]


def test_scales():
    b = torch.zeros((6, 32), dtype=torch.float64)
    b[0, 3] = -1.0
    b[1, 0] = 7.99
    b[2, 1] = 8.0
    b[3, 5] = 2.0 ** -133
    b[4, 31] = torch.inf
    assert R.scale_byte(b).tolist() == [125, 127, 128, 0, 255, 0]


def test_layout():
    v = torch.zeros((1, 3, 300), dtype=torch.float64)
    v[0, 1, 33] = 3.0   # block 1: scale 2^-1, value 6
    v[0, 2, 256] = -4.0  # block 8: first of the second eight
    q, s, val = R.quantize(v)
    assert q.shape == (1, 3, 160) and s.shape == (1, 2, 3, 8)
    assert q[0, 1, 16] == 7 << 4 and q[0, 2, 128] == 6 | 8
    assert s[0, 0, 1].tolist() == [0, 0, 0, 0, 126, 0, 0, 0]
    assert s[0, 1, 2].tolist() == [127, 0, 0, 0, 0, 0, 0, 0]
    assert torch.equal(val, v)


def test_bounds_cover_a_shifted_activation():
    g = torch.Generator().manual_seed(0)
    a = torch.randn(50, 96, generator=g).double()
    ea = torch.full_like(a, 1e-3)
    mid, off = R.act_bounds(a, ea)
    for k in range(5):
        b = a + ea * (2 * torch.rand(a.shape, generator=g).double() - 1)
        assert ((R.values(b[None])[0] - mid).abs() <= off).all()

"""Distillation where a row of W is longer than a tile's loads reach (the block
goes through a copy), at every alignment of the rows, and where blocks are cut;
against the dense formula in double precision."""
import pytest
import torch

from tests import distill_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("V,vblock", [(34_100_000, 1 << 26), (35_000_003, 1 << 22)])
def test_long_rows(V, vblock):
    from paper_2607_01844_amd import moe
    N, H, K = 3, 32, 5
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((N, H), generator=g, device="cuda").bfloat16()
    w = (torch.randn((H, V), generator=g, device="cuda") * 0.3).bfloat16()
    ids = torch.tensor([[0, V - 1, V // 2, -1, 7], [V - 1, V - 2, V - 3, V - 64, V - 65],
                        [1 << 22, (1 << 22) - 1, 33_554_432, 33_554_431, 63]], dtype=torch.int32, device="cuda")
    t = torch.randn((N, K), generator=g, device="cuda") * 2
    dl = torch.randn((N,), generator=g, device="cuda")
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, vblock)
    dx, dw = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, vblock)
    y = torch.cat([x.double() @ w[:, a:a + (1 << 21)].double() for a in range(0, V, 1 << 21)], 1)
    p, logp = R.teacher(ids, t, V, 1.0)
    there = ids >= 0
    ryk = torch.where(there, y.gather(1, torch.where(there, ids, 0).long()), 0.0)
    rlse = torch.logsumexp(y, 1)
    mag = x.double().abs().sum(1, keepdim=True) * w.abs().max().double()
    assert ((yk.double() - ryk).abs() <= H * U * mag).all()
    # sums of exp: each rounding is relative to a sum of positive terms, pairs of 64
    # columns merged in a chain of at most V / 64 / 256 a lane and 300 more
    el = H * U * mag[:, 0] + (V / 64 / 256 + 300) * U + 4 * U * rlse.abs()
    assert ((lse.double() - rlse).abs() <= el).all()
    rloss = (p * (logp - ryk + rlse[:, None])).sum(1)
    assert ((loss.double() - rloss).abs() <= 2 * el + 200 * U * rloss.abs()).all()
    G = torch.softmax(y, 1) * dl.double()[:, None]
    G.scatter_add_(1, torch.where(there, ids, 0).long(), -torch.where(there, p, 0.0) * dl.double()[:, None])
    eG = G.abs() * 2.0 ** -8 + dl.double().abs()[:, None] * (torch.softmax(y, 1) * (4 * el[:, None]) + 100 * U * p.max())
    for a in (0, V // 2 - 100, (1 << 22) - 500, 33_554_432 - 500, V - 1000):
        c = slice(a, a + 1000)
        rw = x.double().t() @ G[:, c]
        ew = x.double().abs().t() @ eG[:, c]
        assert ((dw[:, c].double() - rw).abs() <= ew + 2.0 ** -8 * (rw.abs() + ew) + 2.0 ** -133).all()
    rx, ex = 0, 0
    for a in range(0, V, 1 << 21):
        c = slice(a, a + (1 << 21))
        wt = w[:, c].double().t().contiguous()
        rx, ex = rx + G[:, c] @ wt, ex + (G[:, c].abs() * (2.0 ** -8 + 0.3)) @ wt.abs()
    # a chain of at most 2^22 fp32 sums: 2^22 U = 0.25 of the sum of magnitudes
    assert ((dx.double() - rx).abs() <= ex + 2.0 ** -8 * rx.abs()).all()

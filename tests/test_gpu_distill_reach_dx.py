"""dx of distillation over blocks that are cut or go through copies, where every
block's share of dx stands well above the tolerance: a block left out or taken
twice does not pass.

Block b's columns of W lean along direction b (its logits follow x[:, b], and
its part of dx, mass_b dl, lies along b).  Tolerance (U = 2^-24): G is rounded to
bf16 (2^-8 of itself) and its softmax part moves by 4 el, el the bound of lse
(products of H terms; pairs of 64 columns merged in chains of V / 64 / 256 a lane
and 300 more); dx adds up at most ceil(block / 170) + 64 columns in one chain
(few rows take 170 ranges of a block), one term a block and the 170 ranges, each
rounding at most U of the sum of magnitudes, and is rounded to bf16 once."""
import pytest
import torch

from tests import distill_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
CUT = (0x7ffffff0 // (2 * 32)) // 64 * 64  # columns of a copy of 32 rows that 2^31 bytes hold
STEP = 1 << 21


@pytest.mark.parametrize("V,vblock,starts,lean", [
    (34_100_000, 1 << 26, (0, CUT), (0.0, 3.0)),
    (35_000_003, 1 << 22, tuple(range(0, 35_000_003, 1 << 22)), (1.0,) * 9)])
def test_every_block_counts(V, vblock, starts, lean):
    from paper_2607_01844_amd import moe
    N, H, K = 3, 32, 4
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((N, H), generator=g, device="cuda").clamp(-1, 1).bfloat16()
    x[:, 1] = 1.5
    w = (torch.randn((H, V), generator=g, device="cuda") * 0.3).bfloat16()
    ends = starts[1:] + (V,)
    for b, (lo, hi) in enumerate(zip(starts, ends)):
        w[b, lo:hi] += lean[b]
    ids = torch.tensor([[0, V - 1, V // 2, -1], [CUT, CUT - 1, 1 << 22, (1 << 22) - 1], [-1, -1, 5, 6]],
                       dtype=torch.int32, device="cuda")
    t = torch.randn((N, K), generator=g, device="cuda")
    dl = torch.tensor([1.0, -0.5, 2.0], device="cuda")
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, vblock)
    dx, _ = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, vblock)

    xd, dld = x.double(), dl.double()[:, None]
    y = torch.cat([xd @ w[:, a:a + STEP].double() for a in range(0, V, STEP)], 1)
    rlse = torch.logsumexp(y, 1, keepdim=True)
    el = (H * U * xd.abs().sum(1, keepdim=True) * w.abs().max().double()
          + (V / 64 / 256 + 300) * U + 4 * U * rlse.abs())
    p, _ = R.teacher(ids, t, V, 1.0)
    parts, mags = [], 0.0
    for lo, hi in zip(starts, ends):
        part = torch.zeros((N, H), dtype=torch.float64, device="cuda")
        for a in range(lo, hi, STEP):
            c = slice(a, min(a + STEP, hi))
            wt = w[:, c].double().t().contiguous()
            q = torch.exp(y[:, c] - rlse)
            part += dld * (q @ wt)
            mags = mags + dld.abs() * (q @ wt.abs())
        parts.append(part)
    slots, smag = torch.zeros_like(parts[0]), torch.zeros_like(parts[0])
    for n in range(N):
        for s in range(K):
            if ids[n, s] >= 0:
                col = w[:, ids[n, s].item()].double()
                slots[n] -= dld[n] * p[n, s] * col
                smag[n] += dld[n].abs() * p[n, s] * col.abs()
    rx = sum(parts) + slots
    block = max(hi - lo for lo, hi in zip(starts, ends))
    chain = -(-block // 170) + 64 + len(starts) + 170
    err = (2.0 ** -8 + 4 * el + chain * U) * mags + (2.0 ** -8 + 100 * U + chain * U) * smag
    tol = err + 2.0 ** -8 * (rx.abs() + err)
    assert ((dx.double() - rx).abs() <= tol).all()
    for part in parts:  # dx without it, or with it twice, is off by |part| - tol > tol in some element
        assert (part.abs() > 2 * tol).any()

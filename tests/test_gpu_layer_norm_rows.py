"""The layer norm over many rows at every width class: each wave's and workgroup's second
row and further ones, both ways of loading (kept by the caches or streamed past them), and
rows beyond the registers' reach in many groups.  Against 64 bits, some rows at a time;
dy holds small whole numbers, so that dbeta is exact in any order and shows every row
counted once."""
import pytest
import torch

from tests import train_step_ref as R
from tests.test_gpu_layer_norm import depth

pytestmark = pytest.mark.gpu

# T, d, residual.  Rows of one wave up to 2048 columns, of eight and sixteen beyond.
# The forward streams from 768 MiB (8 bytes an element with the residual, else 4), the
# backward from 384 MiB (8 and 6)
CASES = [
    (3001, 64, True), (9001, 512, True), (5003, 1024, False), (5003, 2048, True), (1500, 2056, True),
    (1500, 4096, True), (2001, 4096, False), (1500, 8192, True), (1100, 8200, True), (1500, 16384, True),
    (1100, 16384, False), (1100, 16392, True), (5000, 16392, False), (700, 65544, True), (63, 16392, True),
    (129, 24576, False), (70001, 16392, False),
    # streamed: backward alone, then both
    (66001, 1024, False), (140001, 512, True),
    (197001, 512, True), (99001, 1024, True), (49500, 2048, True), (24701, 4096, True), (12401, 8192, True),
    (6203, 16384, True), (396001, 512, False), (49301, 4096, False), (24703, 8192, False), (12401, 16384, False),
]


def rows_of_a_sum(T, d):
    """Additions that a row's share of dgamma passes: the rows of its team or group, the
    workgroup's teams, the parts of all (768 at most, in 16 places)."""
    own = max(128, -(-T // 64)) if d > 16384 else max(16, -(-T // 256))
    return own + 4 + 48 + 16


@pytest.mark.parametrize("T,d,residual", CASES, ids=lambda c: str(c))
def test_many_rows(T, d, residual):
    from paper_2607_01844_amd import moe
    print(T, d, residual, flush=True)
    eps, k = 1e-5, depth(d)
    g = torch.Generator(device="cuda").manual_seed(T + d)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = (n(T, d) + n(1, d)).bfloat16()
    res, dh = (n(T, d).mul_(2).bfloat16() if residual else None for _ in range(2))
    gamma, beta = 1 + 0.2 * n(d), 0.3 * n(d)
    dy = torch.randint(-3, 4, (T, d), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    y, h, mean, rstd = moe.moe_layer_norm_fwd(x, gamma, beta, eps, res)
    dx, dgamma, dbeta = moe.moe_layer_norm_bwd(dy, h, gamma, mean, rstd, dh)
    G, B = gamma.double(), beta.double()
    sums, mass, whole = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(3))
    step = max(1, (1 << 24) // d)
    for i in range(0, T, step):
        at = slice(i, i + step)
        if residual:
            assert torch.equal(h[at], (x[at].float() + res[at].float()).bfloat16())
        H, DY, M, S = h[at].double(), dy[at].double(), mean[at].double(), rstd[at].double()
        ry, rm, rr = R.norm(H, G, B, eps)
        # as for single rows: the statistics' errors, and what they make of y
        dm = (k + 2) * R.U * H.abs().mean(1)
        rel = 0.5 * ((k + 6) * R.U + dm ** 2 * rr ** 2) + 3 * R.U
        assert ((M - rm).abs() <= dm).all(), i
        assert ((S - rr).abs() <= 1.01 * rel * rr).all(), i
        xh = ((H - rm[:, None]) * rr[:, None]).abs()
        tol = G.abs() * (dm[:, None] * rr[:, None] + xh * (rel[:, None] + 4 * R.U)) + \
            2 * R.U * (G.abs() * xh + B.abs())
        assert ((y[at].double() - ry).abs() <= 1.01 * (tol + R.UB * ry.abs())).all(), i
        DH = dh[at].double() if residual else torch.zeros_like(DY)
        rx, rg, rb = R.norm_bwd(DY, H, G, M, S, DH)
        xh = (H - M[:, None]) * S[:, None]
        gr = DY * G
        part = gr.abs() + gr.abs().mean(1, keepdim=True) + \
            xh.abs() * (gr * xh).abs().mean(1, keepdim=True)
        tol = S[:, None] * (k + 8) * R.U * part + 2 * R.U * (DH.abs() + rx.abs())
        assert ((dx[at].double() - rx).abs() <= 1.01 * (tol + R.UB * rx.abs())).all(), i
        sums += rg
        whole += rb
        mass += (DY * xh).abs().sum(0)
    # a difference, two products, then the additions
    assert ((dgamma.double() - sums).abs() <= 1.01 * (rows_of_a_sum(T, d) + 3) * R.U * mass).all()
    assert torch.equal(dbeta.double(), whole)

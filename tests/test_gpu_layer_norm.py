"""Layer norm and its gradients on the GPU against 64 bits."""
import pytest
import torch

from tests import train_step_ref as R

pytestmark = pytest.mark.gpu


def depth(d):
    """Additions that one value passes in a row's sum: the lane's own, six steps
    of the wave, the waves (at most 16)."""
    return 8 * max(4, -(-d // 8192)) + 6 + 16


def make(T, d, residual, beta, seed, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    x = (n(T, d) + offset + n(1, d)).bfloat16()
    res = (2 * n(T, d)).bfloat16() if residual else None
    return (x, res, 1 + 0.2 * n(d), 0.3 * n(d) if beta else None, n(T, d).bfloat16(),
            n(T, d).bfloat16() if residual else None)


def check_fwd(x, res, gamma, beta, eps, y, h, mean, rstd):
    T, d = x.shape
    ref_h = x if res is None else (x.float() + res.float()).bfloat16()
    assert torch.equal(h.cpu().view(torch.int16), ref_h.view(torch.int16))
    H, G = R.f64(ref_h), R.f64(gamma)
    B = torch.zeros(d, dtype=torch.float64) if beta is None else R.f64(beta)
    ry, rm, rr = R.norm(H, G, B, eps)
    k = depth(d)
    dm = (k + 2) * R.U * H.abs().mean(1)
    var = 1 / rr ** 2
    # (h - mean)^2 about a mean that is dm off, k additions, a division, the sum
    # with eps, a root and a reciprocal
    rel = 0.5 * ((k + 6) * R.U + dm ** 2 / var) + 3 * R.U
    assert ((R.f64(mean) - rm).abs() <= dm).all()
    assert ((R.f64(rstd) - rr).abs() <= 1.01 * rel * rr).all()
    xh = ((H - rm[:, None]) * rr[:, None]).abs()
    tol = G.abs() * (dm[:, None] * rr[:, None] + xh * (rel[:, None] + 4 * R.U)) + \
        2 * R.U * (G.abs() * xh + B.abs())
    tol = 1.01 * (tol + R.UB * ry.abs())
    assert ((R.f64(y) - ry).abs() <= tol).all()


# T, d, residual, beta: one row and one chunk, the ends of every width's reach,
# rows that end inside a wave's reach, rows beyond the registers'
FWD = [(1, 8, False, True), (1, 64, True, True), (3, 512, True, False), (5, 520, False, True),
       (9, 1024, True, True), (4, 1032, True, True), (2, 2048, False, False), (7, 2056, True, True),
       (16, 4096, True, True), (3, 4104, False, True), (2, 8192, True, True), (3, 8200, True, True),
       (2, 16384, False, True), (3, 16392, True, True), (2, 65544, False, False), (1, 262144, True, True),
       (1100, 520, False, True), (300, 128, True, True), (5000, 64, True, True)]


@pytest.mark.parametrize("case", FWD, ids=lambda c: "-".join(map(str, c)))
def test_forward_and_backward(case):
    from paper_2607_01844_amd import moe
    T, d, residual, has_beta = case
    print(case, flush=True)
    eps = 1e-5
    x, res, gamma, beta, dy, dh = make(T, d, residual, has_beta, T + d)
    c = lambda t: None if t is None else t.cuda()  # noqa: E731
    y, h, mean, rstd = moe.moe_layer_norm_fwd(c(x), c(gamma), c(beta), eps, c(res))
    check_fwd(x, res, gamma, beta, eps, y, h, mean, rstd)
    dx, dgamma, dbeta = moe.moe_layer_norm_bwd(c(dy), h, c(gamma), mean, rstd, c(dh),
                                               with_dbeta=has_beta)
    again = moe.moe_layer_norm_bwd(c(dy), h, c(gamma), mean, rstd, c(dh))
    DY, H, G, M, S = (R.f64(t) for t in (dy, h, gamma, mean, rstd))
    DH = torch.zeros_like(DY) if dh is None else R.f64(dh)
    rx, rg, rb = R.norm_bwd(DY, H, G, M, S, DH)
    k = depth(d)
    xh = (H - M[:, None]) * S[:, None]
    g = DY * G
    part = g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)
    # each of the three terms: k additions and some six products and differences
    tol = S[:, None] * (k + 8) * R.U * part + 2 * R.U * (DH.abs() + rx.abs())
    assert ((R.f64(dx) - rx).abs() <= 1.01 * (tol + R.UB * rx.abs())).all()
    # at most T additions over rows and parts, beside the products
    n = (T + 8) * R.U * 1.01
    assert ((R.f64(dgamma) - rg).abs() <= n * (DY * xh).abs().sum(0)).all()
    if has_beta:
        assert ((R.f64(dbeta) - rb).abs() <= n * DY.abs().sum(0)).all()
        assert torch.equal(dbeta, again[2])
    else:
        assert dbeta is None
    assert torch.equal(dx.view(torch.int16), again[0].view(torch.int16))
    assert torch.equal(dgamma, again[1])


@pytest.mark.parametrize("offset", [100.0, -3000.0])
def test_rows_far_from_zero(offset):
    # bf16 rows around a large mean: squares minus the squared mean would keep
    # nothing of the variance
    from paper_2607_01844_amd import moe
    x, res, gamma, beta, _, _ = make(6, 1000, False, True, 5, offset)
    y, h, mean, rstd = moe.moe_layer_norm_fwd(x.cuda(), gamma.cuda(), beta.cuda(), 1e-6)
    check_fwd(x, None, gamma, beta, 1e-6, y, h, mean, rstd)


def test_constant_rows_and_special_values():
    from paper_2607_01844_amd import moe
    d = 72
    x = torch.ones((4, d), device="cuda", dtype=torch.bfloat16)
    x[1, 3], x[2, 0] = float("nan"), float("inf")
    x[3] = 0
    gamma, beta = torch.full((d,), 2.0, device="cuda"), torch.full((d,), 0.5, device="cuda")
    y, h, mean, rstd = moe.moe_layer_norm_fwd(x, gamma, beta, 1e-4)
    assert h.data_ptr() == x.data_ptr()
    assert (y[[0, 3]] == 0.5).all() and y[1].isnan().all() and y[2].isnan().all()
    # sqrt and the reciprocal of 1e-4 in 32 bits
    assert ((rstd[[0, 3]] - 100).abs() <= 4 * R.U * 100).all()
    dx, dgamma, dbeta = moe.moe_layer_norm_bwd(torch.ones_like(x), h, gamma, mean, rstd)
    assert not dx[[0, 3]].any() and dx[1].isnan().all() and (dbeta == 4).all()
    assert dgamma.isnan().any()


def test_without_rows_or_statistics():
    from paper_2607_01844_amd import moe
    d = 136
    gamma = torch.ones((d,), device="cuda")
    none = torch.empty((0, d), dtype=torch.bfloat16, device="cuda")
    y, h, mean, rstd = moe.moe_layer_norm_fwd(none, gamma)
    dx, dgamma, dbeta = moe.moe_layer_norm_bwd(none, none, gamma, mean, rstd)
    assert y.shape == dx.shape == (0, d) and not dgamma.any() and not dbeta.any()
    x = torch.randn((3, d), device="cuda").bfloat16()
    full = moe.moe_layer_norm_fwd(x, gamma, residual=x)
    bare = moe.moe_layer_norm_fwd(x, gamma, residual=x, stats=False)
    assert bare[2] is None and bare[3] is None
    assert torch.equal(full[0], bare[0]) and torch.equal(full[1], bare[1])


def test_gradients_against_differences():
    # of the loss sum(y dy) + sum(h dh), by the 64-bit reference about the same h
    from paper_2607_01844_amd import moe
    x, res, gamma, beta, dy, dh = make(3, 40, True, True, 9)
    y, h, mean, rstd = moe.moe_layer_norm_fwd(x.cuda(), gamma.cuda(), beta.cuda(), 1e-3, res.cuda())
    dx, dgamma, dbeta = moe.moe_layer_norm_bwd(dy.cuda(), h, gamma.cuda(), mean, rstd, dh.cuda())
    H, G, B = R.f64(h), R.f64(gamma), R.f64(beta)

    def loss(H, G, B):
        return (R.norm(H, G, B, 1e-3)[0] * R.f64(dy)).sum() + (H * R.f64(dh)).sum()
    step = 1e-5
    for at, got in enumerate((dx, dgamma, dbeta)):
        args = [H, G, B]
        flat, ref = R.f64(got).view(-1), []
        for i in range(flat.numel()):
            side = []
            for s in (step, -step):
                a = [t.clone() for t in args]
                a[at].view(-1)[i] += s
                side.append(loss(*a))
            ref.append((side[0] - side[1]) / (2 * step))
        ref = torch.stack(ref)
        # bf16 of dx; 32-bit sums of some tens of terms; the differences' own 1e-9
        big = ref.abs().max()
        tol = (R.UB if at == 0 else 0) * ref.abs() + 200 * R.U * big + 1e-7
        assert ((flat - ref).abs() <= 1.01 * tol).all()


def test_refusals():
    from paper_2607_01844_amd import moe
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    g = torch.ones((64,), device="cuda")
    s = torch.ones((4,), device="cuda")
    for bad in (lambda: moe.moe_layer_norm_fwd(x.float(), g), lambda: moe.moe_layer_norm_fwd(x, g.bfloat16()),
                lambda: moe.moe_layer_norm_fwd(x.cpu(), g), lambda: moe.moe_layer_norm_bwd(x, x, g, s.double(), s)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: moe.moe_layer_norm_fwd(x, g[:60]), lambda: moe.moe_layer_norm_fwd(x.t(), g),
                lambda: moe.moe_layer_norm_fwd(x, g, residual=x[:3]),
                lambda: moe.moe_layer_norm_fwd(x, g, h=torch.empty_like(x)),
                lambda: moe.moe_layer_norm_bwd(x, x, g, s[:3], s),
                lambda: moe.moe_layer_norm_bwd(x, x, g, s, s, dh=x[:2])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(moe.MoEError):
        moe.moe_layer_norm_fwd(x, g, eps=0.0)
    with pytest.raises(moe.MoEError):
        moe.moe_layer_norm_fwd(x[:, :60].contiguous(), g[:60])

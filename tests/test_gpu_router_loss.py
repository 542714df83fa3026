"""Balance loss, z-loss, counts and their gradient on the GPU against the
64-bit reference.

Tolerances.  A probability is an fp32 exponential (hardware, argument y - m
within 20 here: relative error up to 20 * 2^-24 + 2^-22) over an fp32 sum of E
of them (1024 at most: a lane adds 16 and six tree levels, 22 roundings): under
60 * 2^-24 relative in all.  Sums over T <= 5000 tokens add a chain of at most
5000 / 8 terms (a chunk's per wave) and 60 more, each rounding 2^-24 of a
partial sum of positive terms: under 700 * 2^-24.  Of the gradient, two terms
of opposite sign each carry the errors of a p and a sum over E (22): bounded
against the row's largest term by 200 * 2^-24."""
import numpy as np
import pytest
import torch

from tests import router_loss_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def make(T, E, k, seed=0, spread=1.5):
    rng = np.random.default_rng(seed)
    y = (spread * rng.standard_normal((T, E)) + rng.standard_normal((1, E))).astype(np.float32)
    idx = np.argsort(-y, 1, kind="stable")[:, :k].astype(np.int32)
    return y, np.ascontiguousarray(idx)


def dev(a, dtype=None):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def check(y, idx, off=None, mask=None, seed=1):
    from paper_2607_01844_amd import moe
    T, E = y.shape
    k = idx.shape[1]
    off32 = None if off is None else np.asarray(off, dtype=np.int32)
    args = (dev(off32), dev(mask))
    bal, z, counts, ps, n = moe.moe_balance_loss_fwd(dev(y), dev(idx), *args)
    rb, rz, rc, rp, rn = R.forward(y, idx, off, mask)
    assert np.array_equal(counts.cpu().numpy(), rc) and np.array_equal(n.cpu().numpy(), rn)
    rel = 760 * U
    np.testing.assert_allclose(ps.cpu().numpy(), rp, rtol=rel, atol=1e-30)
    np.testing.assert_allclose(bal.cpu().numpy(), rb, rtol=2 * rel, atol=1e-30)
    # lse: an absolute error of 60 U and of the rounding of values up to 20
    np.testing.assert_allclose(z.cpu().numpy(), rz, rtol=rel, atol=2 * 20 * 100 * U)
    G = rb.shape[0]
    rng = np.random.default_rng(seed)
    db, dz = (rng.standard_normal(G).astype(np.float32) for _ in range(2))
    ref = R.backward(y, rc, rn, db, dz, k, off, mask)
    dl = moe.moe_balance_loss_bwd(dev(y), counts, n, dev(db), dev(dz), k, *args)
    a = np.zeros((T, 1))  # the row's largest term before cancellation
    o = [0, T] if off is None else off
    for g in range(G):
        m = max(1, rn[g])
        a[o[g]:o[g + 1]] = abs(db[g]) / m * (E * rc[g].max() / (k * m)) + 2 * abs(dz[g]) / m * 20
    got = dl.cpu().numpy()
    assert (np.abs(got - ref) <= 200 * U * a + 1e-30).all()
    # added to what is there, and rows without a part left bit for bit
    base = rng.standard_normal((T, E)).astype(np.float32)
    acc = dev(base)
    out = moe.moe_balance_loss_bwd(dev(y), counts, n, dev(db), dev(dz), k, *args, dlogits=acc,
                                   accumulate=True)
    assert out is acc
    assert np.array_equal(acc.cpu().numpy(), base + got)
    return got


@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (3, 1), (4, 2), (7, 3), (8, 2), (12, 3), (16, 16),
                                 (31, 4), (64, 6), (100, 8), (128, 8), (130, 2), (255, 4), (257, 5),
                                 (384, 8), (385, 8), (500, 7), (512, 8), (700, 2), (768, 9),
                                 (1023, 16), (1024, 16)])
@pytest.mark.parametrize("T", [1, 67])
def test_experts(E, k, T):
    check(*make(T, E, k, seed=E))


@pytest.mark.parametrize("T", [2, 63, 64, 65, 257, 1100, 5000])
def test_tokens(T):
    check(*make(T, 24, 3, seed=T))


@pytest.mark.parametrize("off", [[0, 0, 5, 5, 300], [0, 64, 128, 300], [7, 9, 9, 200],
                                 list(range(0, 301, 3)) + [300], [0, 0], [300, 300], [0, 1]])
@pytest.mark.parametrize("masked", [False, True])
def test_sequences(off, masked):
    T = 300
    y, idx = make(T, 12, 3, seed=len(off))
    mask = np.random.default_rng(5).random(T) < 0.8 if masked else None
    got = check(y, idx, off, mask)
    out = np.ones(T, dtype=bool)
    out[off[0]:off[-1]] = False
    assert (got[out] == 0).all()
    if masked:
        assert (got[~mask] == 0).all()


def test_masked_tokens_may_hold_anything():
    y, idx = make(200, 20, 2)
    mask = np.random.default_rng(2).random(200) < 0.5
    clean = check(y, idx, None, mask)
    for bad in (np.nan, np.inf, -np.inf, -3.4e38):
        z = y.copy()
        z[~mask] = bad
        from paper_2607_01844_amd import moe
        bal, zl, counts, ps, n = moe.moe_balance_loss_fwd(dev(z), dev(idx), None, dev(mask))
        one = torch.ones(1, device="cuda")
        assert torch.isfinite(bal).all() and torch.isfinite(zl).all() and torch.isfinite(ps).all()
        dl = moe.moe_balance_loss_bwd(dev(z), counts, n, one, one, 2, None, dev(mask)).cpu().numpy()
        assert np.isfinite(dl).all() and (dl[~mask] == 0).all()
    assert np.isfinite(clean).all()


def test_all_masked_and_no_tokens():
    from paper_2607_01844_amd import moe
    y, idx = make(50, 8, 2)
    mask = torch.zeros(50, dtype=torch.uint8, device="cuda")
    r = moe.moe_balance_loss_fwd(dev(y), dev(idx), None, mask)
    assert all((t == 0).all() for t in r)
    one = torch.ones(1, device="cuda")
    assert (moe.moe_balance_loss_bwd(dev(y), r[2], r[4], one, one, 2, None, mask) == 0).all()
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    r = moe.moe_balance_loss_fwd(torch.empty((0, 8), device="cuda"),
                                 torch.empty((0, 2), dtype=torch.int32, device="cuda"), off)
    assert r[2].shape == (3, 8) and all((t == 0).all() for t in r)


def test_masked_experts_and_an_empty_row():
    y, idx = make(90, 16, 2)
    y[:, 5] = -np.inf
    y[3] = -np.inf  # no expert left
    y[4, 1:] = -3.4028235e38
    idx[10] = [-1, 16]  # no expert: not counted
    check(y, idx)


def test_nan_stays_in_its_group():
    from paper_2607_01844_amd import moe
    y, idx = make(120, 8, 2)
    y[70, 3] = np.nan
    off = dev(np.array([0, 60, 120], dtype=np.int32))
    bal, z, counts, ps, n = moe.moe_balance_loss_fwd(dev(y), dev(idx), off)
    assert torch.isfinite(bal[0]) and torch.isnan(bal[1]) and torch.isnan(z[1])
    assert torch.isfinite(ps[0]).all()


def test_counts_agree_with_the_permutation():
    from paper_2607_01844_amd import moe
    import workloads as W
    wl = W.WORKLOADS["tiny"]
    inp = W.make_inputs(wl, seed=1, device="cuda")
    lg = torch.empty((wl.T, wl.E), device="cuda")
    idx, _ = moe.moe_route(inp["x"], inp["w_router"], None, wl.k, logits=lg)
    pm = moe.moe_permute(inp["x"], idx, wl.E)
    counts = moe.moe_balance_loss_fwd(lg, idx)[2]
    assert torch.equal(counts[0], pm["counts_global"])


def test_same_bits_again_and_on_another_stream():
    from paper_2607_01844_amd import moe
    y, idx = make(5000, 96, 4)
    y, idx = dev(y), dev(idx)
    a = moe.moe_balance_loss_fwd(y, idx)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = moe.moe_balance_loss_fwd(y, idx)
    torch.cuda.current_stream().wait_stream(s)
    c = moe.moe_balance_loss_fwd(y, idx)
    for u, v, w in zip(a, b, c):
        assert torch.equal(u, v) and torch.equal(u, w)


@pytest.mark.parametrize("T,d,E", [(200, 64, 12), (4096, 1024, 64)])
def test_aux_joins_the_router_backward(T, d, E):
    """dlogits of the sum are the sum of the dlogits; dw_router, dbias and dx
    come from it on both of the router backward's paths."""
    from paper_2607_01844_amd import moe
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((T, d), generator=g, device="cuda").bfloat16()
    w = torch.randn((d, E), generator=g, device="cuda") * 0.02
    lg = torch.empty((T, E), device="cuda")
    idx, gate = moe.moe_route(x, w, None, 2, logits=lg)
    dg = torch.randn((T, 2), generator=g, device="cuda") * 1e-2
    aux = torch.randn((T, E), generator=g, device="cuda") * 1e-2
    plain, both = torch.empty((T, E), device="cuda"), torch.empty((T, E), device="cuda")
    moe.moe_route_bwd(x, w, lg, idx, gate, dg, dlogits=plain)
    dw, db, dx = moe.moe_route_bwd(x, w, lg, idx, gate, dg, dlogits=both, with_dbias=True,
                                   dx=torch.empty_like(x), dx_accumulate=False, dlogits_aux=aux)
    assert torch.equal(both, plain + aux)
    dl = both.double().cpu()
    rw, rx = x.double().cpu().t() @ dl, dl @ w.double().cpu().t()
    # dw: operands split in two bf16 parts (2^-17) and fp32 sums over T tokens
    # in chunks of at most 512: under 600 roundings of the sum of magnitudes
    mag = x.double().cpu().abs().t() @ dl.abs()
    assert ((dw.double().cpu() - rw).abs() <= (2.0 ** -17 + 600 * U) * mag).all()
    assert ((db.double().cpu() - dl.sum(0)).abs() <= 600 * U * dl.abs().sum(0)).all()
    mag = dl.abs() @ w.double().cpu().abs().t()
    assert ((dx.double().cpu() - rx).abs() <= (2.0 ** -16 + 600 * U) * mag + 2.0 ** -8 * rx.abs()).all()


def test_layer_step_with_router_losses():
    """The layer's step with the router's losses: the loss parts of dw_router
    come out as the difference of two steps', and a captured step replays."""
    import workloads as W
    from paper_2607_01844_amd import moe
    wl = W.WORKLOADS["tiny"]
    inp = W.make_inputs(wl, seed=2, device="cuda")
    on = moe.layer_fwd_bwd(inp, wl.k, keep=False, router_loss=(0.5, 0.25))
    off = moe.layer_fwd_bwd(inp, wl.k, keep=False, router_loss=(0.0, 0.0))
    plain = moe.layer_fwd_bwd(inp, wl.k, keep=False)
    for key in ("topk_idx", "topk_gate", "y", "dgate", "dw_gate", "dw_up", "dw_down"):
        assert torch.equal(on[key], plain[key]), key
    x = inp["x"].double().cpu()
    y = (x @ inp["w_router"].double().cpu()).numpy()
    idx = on["topk_idx"].cpu().numpy()
    rb, rz, rc, _, rn = R.forward(y, idx)
    np.testing.assert_allclose(on["balance"].cpu().numpy(), rb, rtol=1e-5)
    np.testing.assert_allclose(on["zloss"].cpu().numpy(), rz, rtol=1e-5)
    aux = R.backward(y, rc, rn, [0.5], [0.25], wl.k)
    want = x.numpy().T @ aux
    got = (on["dw_router"].double() - off["dw_router"].double()).cpu().numpy()
    # both sides' fp32 sums (300 roundings at the sum of magnitudes) cancel
    mag = np.abs(x.numpy()).T @ np.abs(aux) + np.abs(off["dw_router"].cpu().numpy()).max()
    assert (np.abs(got - want) <= 1000 * U * mag + 1e-5 * np.abs(want).max()).all()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        moe.layer_fwd_bwd(inp, wl.k, keep=False, router_loss=(0.5, 0.25))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = moe.layer_fwd_bwd(inp, wl.k, keep=False, router_loss=(0.5, 0.25))
    for _ in range(3):
        for v in out.values():
            v.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        for key in on:
            assert torch.equal(out[key], on[key]), key
        again = moe.layer_fwd_bwd(inp, wl.k, keep=False, router_loss=(0.5, 0.25))
        assert torch.equal(again["dx"], on["dx"])


def test_binding_refuses():
    from paper_2607_01844_amd import moe
    y, idx = make(10, 8, 2)
    y, idx = dev(y), dev(idx)
    off = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    one = torch.ones(1, device="cuda")
    c, n = torch.zeros((1, 8), dtype=torch.int32, device="cuda"), off[:1]
    for call, err in [
            (lambda: moe.moe_balance_loss_fwd(y.double(), idx), TypeError),
            (lambda: moe.moe_balance_loss_fwd(y.cpu(), idx), TypeError),
            (lambda: moe.moe_balance_loss_fwd(y.t(), idx), ValueError),
            (lambda: moe.moe_balance_loss_fwd(y, idx[:9]), ValueError),
            (lambda: moe.moe_balance_loss_fwd(y, idx.long()), TypeError),
            (lambda: moe.moe_balance_loss_fwd(y, idx, off[:1]), ValueError),
            (lambda: moe.moe_balance_loss_fwd(y, idx, off, torch.ones(10, device="cuda")), TypeError),
            (lambda: moe.moe_balance_loss_fwd(y, idx, off, torch.ones(9, dtype=torch.bool,
                                                                      device="cuda")), ValueError),
            (lambda: moe.moe_balance_loss_bwd(y, c[:, :7].contiguous(), n, one, one, 2), ValueError),
            (lambda: moe.moe_balance_loss_bwd(y, c, n, one, one.double(), 2), TypeError),
            (lambda: moe.moe_balance_loss_bwd(y, c, n, one, one, 2, accumulate=True), ValueError),
            (lambda: moe.moe_balance_loss_bwd(y, c, n, one, one, 9), moe.MoEError)]:
        with pytest.raises(err):
            call()

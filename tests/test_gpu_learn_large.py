"""Router losses, MXFP4 and distillation beyond 2^31 elements, and two streams
at once."""
import pytest
import torch

from tests import mxfp4_ref as M
from tests.test_gpu_mxfp4 import values, weights

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def gen(seed=0):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_router_losses():
    from paper_2607_01844_amd import moe
    T, E, k = (1 << 22) + 5, 520, 2
    assert T * E > 1 << 31
    y = torch.randn((T, E), generator=gen(), device="cuda")
    idx = torch.randint(0, E, (T, k), generator=gen(1), device="cuda", dtype=torch.int32)
    bal, z, counts, ps, n = moe.moe_balance_loss_fwd(y, idx)
    assert n.item() == T
    rc = torch.bincount(idx.flatten().long(), minlength=E)
    assert torch.equal(counts[0].long(), rc)
    rp, rz = torch.zeros(E, dtype=torch.float64, device="cuda"), 0.0
    for a in range(0, T, 1 << 19):
        v = y[a:a + (1 << 19)].double()
        lse = torch.logsumexp(v, 1)
        rp += torch.exp(v - lse[:, None]).sum(0)
        rz += (lse ** 2).sum()
    # a wave adds at most 512 tokens' terms, a group 4 chunks a lane and 20 more
    assert ((ps[0].double() - rp).abs() <= 760 * U * rp).all()
    rb = E / (k * float(T) ** 2) * (rc.double() * rp).sum()
    assert abs(bal.item() - rb.item()) <= 2 * 760 * U * rb.item()
    assert abs(z.item() - rz.item() / T) <= 760 * U * rz.item() / T + 2 * 20 * 100 * U
    db, dz = torch.full((1,), 3.0, device="cuda"), torch.full((1,), -2.0, device="cuda")
    dl = moe.moe_balance_loss_bwd(y, counts, n, db, dz, k)
    a = E * rc.double() / (k * T)
    bound = 200 * U * (3.0 / T * a.max().item() + 2 * 2.0 / T * 20)
    for rows in (slice(0, 1000), slice(T // 2, T // 2 + 1000), slice(T - 1000, T)):
        v = y[rows].double()
        lse = torch.logsumexp(v, 1, keepdim=True)
        p = torch.exp(v - lse)
        ref = p * (3.0 / T * (a - (a * p).sum(1, keepdim=True)) + 2 * -2.0 / T * lse)
        assert ((dl[rows].double() - ref).abs() <= bound).all()


def test_quantise():
    from paper_2607_01844_amd import moe
    P, n, K = 1000, 20_000, 136
    assert P * n * K > 1 << 31
    base = torch.randn((P, K), generator=gen(2), device="cuda").bfloat16()
    big = base.repeat(n, 1)
    q, s = moe.moe_mxfp4_quantize(base)
    bq, bs = moe.moe_mxfp4_quantize(big)
    assert torch.equal(bq.view(n, P, -1), q.expand(n, P, -1).contiguous())
    assert torch.equal(bs.view(n, P, 8), s.view(1, P, 8).expand(n, P, 8).contiguous())
    del big
    back = moe.moe_mxfp4_dequantize(bq, bs, K).view(n, P, K)
    want = moe.moe_mxfp4_dequantize(q, s, K)
    assert torch.equal(want.double().cpu(), M.values(base.double().cpu()[None])[0])
    for a in range(0, n, 2000):
        assert torch.equal(back[a:a + 2000], want.expand(2000, P, K))


def test_grouped_forward():
    from paper_2607_01844_amd import moe
    P, n, d, f = 500, 1100, 4104, 40
    assert P * n * d > 1 << 31
    x = torch.randn((P, d), generator=gen(3), device="cuda").bfloat16()
    w = weights(1, d, f, 4)
    xq = moe.moe_mxfp4_quantize(x)
    one = torch.tensor([0, P], dtype=torch.int32, device="cuda")
    want = moe.moe_grouped_swiglu_fwd_mxfp4(xq, one, *w, d)
    ref, bound = M.swiglu(values(xq, d), *(values((a[0], b[0]), K) for (a, b), K in zip(w, (d, d, f))))
    assert M.close(want.cpu(), ref, bound)
    off = torch.tensor([0, P * n], dtype=torch.int32, device="cuda")
    src = torch.arange(P * n, dtype=torch.int32, device="cuda") % P
    y = moe.moe_grouped_swiglu_fwd_mxfp4(xq, off, *w, d, row_src=src, k=1).view(n, P, d)
    for a in range(0, n, 100):
        assert torch.equal(y[a:a + 100], want.expand(100, P, d))


def test_distillation_in_one_block():
    """Logit gradients of one block of all columns: more than 2^31 elements; and
    the same in blocks of 16384."""
    from paper_2607_01844_amd import moe
    N, H, V, K = 4096, 64, 600_000, 9
    assert N * V > 1 << 31
    x = torch.randn((N, H), generator=gen(5), device="cuda").bfloat16()
    w = (torch.randn((H, V), generator=gen(6), device="cuda") * 0.2).bfloat16()
    ids = torch.randint(0, V, (N, K), generator=gen(7), device="cuda", dtype=torch.int32)
    ids[-1, 0] = V - 1
    t = torch.randn((N, K), generator=gen(8), device="cuda") * 3
    dl = torch.randn((N,), generator=gen(9), device="cuda")
    xd, step = x.double(), 1 << 14
    chunk = lambda a: (xd @ w[:, a:a + step].double(), w[:, a:a + step].double().t().contiguous())  # noqa: E731
    lse = torch.logsumexp(torch.stack([torch.logsumexp(chunk(a)[0], 1) for a in range(0, V, step)], 1), 1)
    p = torch.softmax(t.double(), 1)
    yk = torch.stack([xd[:, h:h + 1] * w[h][ids.long()].double() for h in range(H)]).sum(0)
    ey = H * U * (xd.abs().sum(1, keepdim=True) * w.abs().max().double())
    # log-sum-exp: positive terms in pairs of 64 columns, V / 64 / 256 a lane and 300 more
    el = ey[:, 0] + (V / 64 / 256 + 300) * U + 4 * U * lse.abs()
    loss = (p * (torch.log(p) - yk + lse[:, None])).sum(1)
    rx, ex, cols = 0, 0, {}
    for a in range(0, V, step):
        y, wt = chunk(a)
        q = torch.exp(y - lse[:, None])
        G = dl.double()[:, None] * q
        eG = dl.double().abs()[:, None] * q * (2 * el[:, None] + ey + 100 * U)
        for j in range(K):
            here = ((ids[:, j] >= a) & (ids[:, j] < a + G.shape[1])).nonzero()[:, 0]
            at = ids[here, j].long() - a
            G[here, at] -= dl[here].double() * p[here, j]
            eG[here, at] += dl[here].double().abs() * p[here, j] * 200 * U
        eG += 2.0 ** -8 * G.abs()
        rx = rx + G @ wt
        ex = ex + (eG + 0.006 * G.abs()) @ wt.abs()  # chains of at most 75,000 fp32 sums and 40 more
        if a in (0, V // 2 // step * step, (V - 1) // step * step):
            cols[a] = (xd.t() @ G, xd.abs().t() @ (eG + N * U * G.abs()))
    for vb in (V, step):
        gl, gs, gy = moe.moe_vocab_distill_fwd(x, w, ids, t, vb)
        dx, dw = moe.moe_vocab_distill_bwd(x, w, ids, t, gs, gy, dl, vb)
        assert ((gy.double() - yk).abs() <= ey).all()
        assert ((gs.double() - lse).abs() <= el).all()
        assert ((gl.double() - loss).abs() <= el + ey[:, 0] + 200 * U * (loss.abs() + 1)
                + 8 * U * (p * (yk.abs() + lse.abs()[:, None] + torch.log(p).abs())).sum(1)).all()
        assert ((dx.double() - rx).abs() <= ex + 2.0 ** -8 * (rx.abs() + ex)).all()
        for a, (rw, ew) in cols.items():
            got = dw[:, a:a + step].double()
            assert ((got - rw).abs() <= ew + 2.0 ** -8 * (rw.abs() + ew) + 2.0 ** -133).all()
        del dx, dw


def test_two_streams_at_once():
    from paper_2607_01844_amd import moe

    def work(seed):
        g = gen(seed)
        T, E = 3000 + 500 * seed, 64
        y = torch.randn((T, E), generator=g, device="cuda")
        idx = torch.randint(0, E, (T, 2), generator=g, device="cuda", dtype=torch.int32)
        x = torch.randn((T // 4, 128), generator=g, device="cuda").bfloat16()
        wv = (torch.randn((128, 5000 + 8 * seed), generator=g, device="cuda") * 0.2).bfloat16()
        ids = torch.randint(0, 5000, (T // 4, 6), generator=g, device="cuda", dtype=torch.int32)
        t = torch.randn((T // 4, 6), generator=g, device="cuda")
        dl = torch.randn((T // 4,), generator=g, device="cuda")
        ti = torch.randint(0, 4, (T // 4, 1), generator=g, device="cuda", dtype=torch.int32)
        gate = torch.rand((T // 4, 1), generator=g, device="cuda")
        w = [moe.moe_mxfp4_quantize((torch.randn(s, generator=g, device="cuda") * 0.1).bfloat16(), True)
             for s in ((4, 128, 72), (4, 128, 72), (4, 72, 128))]
        one = torch.ones(1, device="cuda")

        def run():
            r = moe.moe_balance_loss_fwd(y, idx)
            d = moe.moe_balance_loss_bwd(y, r[2], r[4], one, one, 2)
            f = moe.moe_vocab_distill_fwd(x, wv, ids, t, 1024)
            b = moe.moe_vocab_distill_bwd(x, wv, ids, t, f[1], f[2], dl, 1024)
            return (*r, d, *f, *b, moe.moe_ffn_fwd_mxfp4(x, ti, gate, 4, *w))
        return run

    runs = [work(1), work(2)]
    want = [r() for r in runs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(runs[i]())
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            for a, b in zip(g, want[i]):
                assert torch.equal(a, b)

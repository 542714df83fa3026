"""The embedding, the layer norm and the updates beyond 2^31 elements and bytes,
checked at places on both sides of the limits."""
import numpy as np
import pytest
import torch

from tests import train_step_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def free_after():
    yield
    torch.cuda.empty_cache()


def fill(t, seed, scale=1.0):
    """Normal values, a stretch of them repeated."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    some = (torch.randn(1 << 22, generator=g, device="cuda") * scale).to(t.dtype)
    flat = t.view(-1)
    for i in range(0, flat.numel(), 1 << 22):
        part = flat[i:i + (1 << 22)]
        part.copy_(some[:part.numel()].roll(i >> 22))
    return t


def test_embedding_of_a_large_table_and_batch():
    from paper_2607_01844_amd import moe
    rows, N, H = 270001, 270011, 8192  # 2.2e9 elements each
    w = fill(torch.empty((rows, H), dtype=torch.bfloat16, device="cuda"), 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, rows, (N,), generator=g, device="cuda", dtype=torch.int32)
    ids[-3:] = rows - 1
    ids[:2] = rows - 1
    y = moe.moe_embedding_fwd(ids, w, 2.0)
    at = torch.tensor([0, 1, 131071, 131072, 262143, 262144, 262145, N - 1], device="cuda")
    assert torch.equal(y[at], w[ids[at].long()] * 2)
    dw = moe.moe_embedding_bwd(ids, y, rows)
    order = ids.cpu()
    for v in [0, 5, 131072, 262143, 262144, 262145, rows - 2, rows - 1]:
        t = torch.nonzero(order == v)[:, 0].cuda()
        part = y[t].double()
        ref, mass = part.sum(0), part.abs().sum(0)
        tol = (t.numel() + 1) * R.U * mass + R.UB * ref.abs()
        assert ((dw[v].double() - ref).abs() <= 1.01 * tol).all(), v


def test_layer_norm_of_many_long_rows():
    from paper_2607_01844_amd import moe
    T, d = 270001, 8192
    x = fill(torch.empty((T, d), dtype=torch.bfloat16, device="cuda"), 3)
    gamma = 1 + 0.1 * torch.randn(d, device="cuda")
    y, h, mean, rstd = moe.moe_layer_norm_fwd(x, gamma)
    dx, dgamma, dbeta = moe.moe_layer_norm_bwd(x, h, gamma, mean, rstd)
    at = torch.tensor([0, 131071, 131072, 262143, 262144, T - 1], device="cuda")
    few = moe.moe_layer_norm_fwd(x[at], gamma)
    # a row's values do not go by where it lies
    for a, b in zip((y, mean, rstd), (few[0], few[2], few[3])):
        assert torch.equal(a[at], b)
    assert torch.equal(dx[at], moe.moe_layer_norm_bwd(x[at], x[at], gamma, few[2], few[3])[0])
    ref = torch.zeros(d, dtype=torch.float64, device="cuda")
    mass = torch.zeros_like(ref)
    for i in range(0, T, 8192):
        part = x[i:i + 8192].double()
        ref += part.sum(0)
        mass += part.abs().sum(0)
    # some 528 rows of a workgroup one after another, then 512 sums in 32 places
    assert ((dbeta.double() - ref).abs() <= (528 + 64) * R.U * mass).all()
    assert dgamma.isfinite().all()


def test_update_of_more_than_2_to_32_elements():
    from paper_2607_01844_amd import moe
    n = (1 << 32) + 5001
    w = fill(torch.empty(n, dtype=torch.bfloat16, device="cuda"), 5, 0.1)
    g = fill(torch.empty(n, dtype=torch.bfloat16, device="cuda"), 6)
    p = moe.Params([w], [g], bits=8)
    places = [0, (1 << 31) - 2048, (1 << 32) - 4096, (1 << 32), n - n % 128 - 1280]
    before = {a: w[a:a + 4096 if a + 4096 < n else n].clone() for a in places}
    moe.moe_adamw_step(p, 1e-2, 1, 0.9, 0.95, 1e-8, 0.1, seed=9)
    r_all = {}
    for a, w0 in before.items():
        m = w0.numel()
        x = g[a:a + m].float().cpu().numpy()
        m32, v32 = R.states32(0 * x, 0 * x, x, 0.9, 0.95)
        i = (np.arange(m, dtype=np.uint64) + np.uint64(a)) & np.uint64(0xFFFFFFFF)
        key = R.mix(R.mix((9 + 0x85A308D3) & 0xFFFFFFFF, 0x6A09E667), 0xBB67AE85)
        r = R.mix(i * np.uint64(0x9E3779B9) + key, 0x6A09E667)
        r_all[a] = r
        for kind, val, r16 in (("m", m32, r & np.uint64(0xFFFF)), ("v", v32, r >> np.uint64(16))):
            codes, scales = R.encode(val, kind, r16)
            held = getattr(p, kind)[0]
            assert np.array_equal(held[0][a:a + m].cpu().numpy(), codes), (a, kind)
            assert np.array_equal(held[1][a // 128:a // 128 + scales.size].cpu().numpy(), scales)
        # the first step's quotient is the gradient's sign, but for eps
        want = w0.double() * (1 - 1e-3) - 1e-2 * torch.sign(g[a:a + m].double())
        got = w[a:a + m].double()
        live = g[a:a + m].abs() > 1e-3
        step = 2.0 ** -7 * want.abs() + 1e-6  # one of the two neighbours
        assert ((got - want).abs() <= step)[live].all(), a
    q = moe.moe_grad_sumsq(p)
    ref = sum(float(g[i:i + (1 << 28)].double().square().sum()) for i in range(0, n, 1 << 28))
    assert abs(float(q) - ref) <= 66 * R.U * ref

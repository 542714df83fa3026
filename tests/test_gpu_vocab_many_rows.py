"""More rows than one launch of a wave a row holds (2^32 threads, 2^26 rows): a
row's results are those of the same row in a short call, bit for bit (they come
from its own 64 columns and one step of H = 8, in the same order)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
H, V, K = 8, 64, 1


def make(N):
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((N, H), dtype=torch.bfloat16, device="cuda")
    for part in x.split(1 << 24):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    w = torch.randn((H, V), generator=g, device="cuda").bfloat16()
    ids = torch.randint(-1, V, (N, K), generator=g, device="cuda", dtype=torch.int32)
    dl = torch.randn((N,), generator=g, device="cuda")
    return x, w, ids, dl


def pieces(N):
    m = 1 << 25
    return [slice(0, 1000), slice(m - 500, m + 500), slice(N - 1000, N)] + (
        [slice(2 * m - 500, 2 * m + 3)] if N > 2 * m + 3 else [])


def test_distillation():
    from paper_2607_01844_amd import moe
    N = (1 << 26) - 1
    x, w, ids, dl = make(N)
    t = dl[:, None] * 2
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, V)
    dx, _ = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, V)
    for r in pieces(N):
        a = [v[r].clone() for v in (x, ids, t, dl)]
        want = moe.moe_vocab_distill_fwd(a[0], w, a[1], a[2], V)
        for got, ref in zip((loss, lse, yk), want):
            assert torch.equal(got[r], ref)
        assert torch.equal(dx[r], moe.moe_vocab_distill_bwd(a[0], w, a[1], a[2], want[1], want[2], a[3], V)[0])


def test_target_loss():
    from paper_2607_01844_amd import moe
    N = (1 << 26) + 5
    x, w, ids, _ = make(N)
    target = ids[:, 0].clamp(min=0)
    loss, lse = moe.moe_vocab_loss_fwd(x, w, target, V)
    for r in pieces(N):
        want = moe.moe_vocab_loss_fwd(x[r].clone(), w, target[r].clone(), V)
        assert torch.equal(loss[r], want[0]) and torch.equal(lse[r], want[1])

"""Embedding and its gradient on the GPU against plain sums in 64 bits."""
import pytest
import torch

from tests import train_step_ref as R

pytestmark = pytest.mark.gpu


def ids_of(kind, N, rows, begin, g):
    """Token ids, some of them outside [begin, begin + rows)."""
    if kind == "one":
        return torch.full((N,), begin + rows - 1, dtype=torch.int32)
    if kind == "none":
        return torch.full((N,), -1, dtype=torch.int32)
    if kind == "ascending":
        return (begin + torch.arange(N) % rows).to(torch.int32)
    u = torch.rand((N,), generator=g)
    i = begin - 2 + (u ** (4 if kind == "skewed" else 1) * (rows + 4)).long()
    if kind == "skewed":
        i = torch.where(torch.rand((N,), generator=g) < 0.3, begin, i)
    i[torch.rand((N,), generator=g) < 0.1] = -1
    return i.to(torch.int32)


# N, H, rows, begin, scale, ids.  8192 tokens are the most that one workgroup
# sorts; widths below, at and above one wave's 512 columns; rows of one, two and
# three digits of the sort
CASES = [
    (1, 8, 1, 0, 1.0, "one"), (1, 64, 5, 3, 2.0, "even"), (2, 128, 3, 0, -0.5, "one"),
    (7, 520, 33, 1000, 1.0, "even"), (64, 512, 31, 0, 3.0, "skewed"),
    (256, 128, 1000, 0, 11.3, "even"), (1000, 520, 32, 7, 1.0, "skewed"),
    (1100, 1032, 511, 0, 1.0, "ascending"), (1024, 72, 512, 5, 22.8, "even"),
    (1025, 4096, 100, 0, 1.0, "skewed"), (3000, 16, 70000, 12, 4.0, "even"),
    (4097, 64, 3, 0, 1.0, "one"), (8192, 32, 300000, 0, 1.0, "skewed"),
    (8193, 24, 600, 9, 0.125, "skewed"), (9000, 512, 64, 0, 1.0, "none"),
    (20001, 40, 270000, 1, 1.0, "even"), (30000, 8, 2, 0, 1.0, "even"),
    (70000, 16, 1500, 0, 1.0, "skewed"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_embedding(case):
    from paper_2607_01844_amd import moe
    N, H, rows, begin, scale, kind = case
    print(case, flush=True)
    g = torch.Generator().manual_seed(N + H)
    ids = ids_of(kind, N, rows, begin, g)
    w = torch.randn((rows, H), generator=g).bfloat16()
    dy = torch.randn((N, H), generator=g).bfloat16()
    y = moe.moe_embedding_fwd(ids.cuda(), w.cuda(), scale, begin)
    dw = moe.moe_embedding_bwd(ids.cuda(), dy.cuda(), rows, scale, begin, dw=torch.full(
        (rows, H), float("nan"), dtype=torch.bfloat16, device="cuda"))
    again = moe.moe_embedding_bwd(ids.cuda(), dy.cuda(), rows, scale, begin)
    torch.cuda.synchronize()
    # one product in 32 bits, rounded once: bit for bit
    there = (ids >= begin) & (ids < begin + rows)
    ref = w.float()[torch.where(there, ids - begin, 0).long()] * torch.tensor(scale)
    ref = torch.where(there[:, None], ref, torch.zeros(())).bfloat16()
    assert torch.equal(y.cpu().view(torch.int16), ref.view(torch.int16))
    # n sums in 32 bits and a product, then a rounding to bf16
    ref, mass, n = R.embed_bwd(ids, R.f64(dy), rows, scale, begin)
    tol = (n + 1) * R.U * mass * 1.01 + R.UB * 1.01 * ref.abs()
    assert ((R.f64(dw) - ref).abs() <= tol).all()
    assert torch.equal(dw.view(torch.int16), again.view(torch.int16))
    assert not dw[(n[:, 0] == 0).cuda()].any()


def test_no_tokens():
    from paper_2607_01844_amd import moe
    ids = torch.empty((0,), dtype=torch.int32, device="cuda")
    w = torch.randn((5, 64), device="cuda").bfloat16()
    assert moe.moe_embedding_fwd(ids, w).shape == (0, 64)
    dw = torch.full((70000, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    moe.moe_embedding_bwd(ids, torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), 70000,
                          dw=dw)
    assert not dw.any()


@pytest.mark.parametrize("N", [300, 9000])
def test_special_values_stay_in_their_rows(N):
    from paper_2607_01844_amd import moe
    H, rows = 136, 40
    g = torch.Generator().manual_seed(3)
    ids = torch.randint(0, rows, (N,), generator=g, dtype=torch.int32).cuda()
    w = torch.randn((rows, H), generator=g).bfloat16().cuda()
    dy = torch.randn((N, H), generator=g).bfloat16().cuda()
    clean = moe.moe_embedding_bwd(ids, dy, rows)
    dy[5, 7], dy[6, 8], w[3, 1] = float("nan"), float("inf"), float("nan")
    dw = moe.moe_embedding_bwd(ids, dy, rows)
    bad = torch.zeros((rows, H), dtype=torch.bool, device="cuda")
    bad[ids[5].long(), 7] = bad[ids[6].long(), 8] = True
    assert dw[ids[5].long(), 7].isnan() and dw[ids[6].long(), 8].isinf()
    assert torch.equal(dw[~bad], clean[~bad])
    y = moe.moe_embedding_fwd(ids, w)
    assert torch.equal(y.isnan().any(1), ids == 3)
    # what no row holds is 0, beside a NaN row and with any scale
    out = moe.moe_embedding_fwd(ids - 100, w, float(3e38))
    assert not out.any()


def test_refusals():
    from paper_2607_01844_amd import moe
    ids = torch.zeros((4,), dtype=torch.int32, device="cuda")
    w = torch.zeros((5, 64), dtype=torch.bfloat16, device="cuda")
    dy = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: moe.moe_embedding_fwd(ids.long(), w), lambda: moe.moe_embedding_fwd(ids, w.float()),
                lambda: moe.moe_embedding_fwd(ids.cpu(), w), lambda: moe.moe_embedding_bwd(ids, dy.float(), 5)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: moe.moe_embedding_fwd(ids, w.t()), lambda: moe.moe_embedding_fwd(ids[::2], w),
                lambda: moe.moe_embedding_bwd(ids[:3], dy, 5),
                lambda: moe.moe_embedding_bwd(ids, dy, 5, dw=w[:4])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: moe.moe_embedding_fwd(ids, w, float("nan")),
                lambda: moe.moe_embedding_fwd(ids, w, 1.0, -1),
                lambda: moe.moe_embedding_bwd(ids, dy, 0)):
        with pytest.raises(moe.MoEError):
            bad()

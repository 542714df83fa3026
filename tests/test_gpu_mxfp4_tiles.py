"""The 4-bit grouped forward on its 256-row tile (many rows an expert and enough
tiles for the chip) and with more tiles than a workgroup finds at once, on both
tiles; the bounds are tests/mxfp4_ref.py's."""
import pytest
import torch

import workloads as W
from tests import mxfp4_ref as R
from tests.test_gpu_mxfp4 import check_grouped, values, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,d,f", [([700, 0, 129, 1400], 264, 2056), ([1025, 1, 256, 2900], 2056, 72),
                                        ([4000, 385, 383], 1032, 1032), ([9000], 8, 648),
                                        ([255, 257, 513, 31, 1281], 520, 2184)])
def test_grouped(counts, d, f):
    check_grouped(counts, d, f, seed=d + f)


def test_nan_and_far_scales():
    from paper_2607_01844_amd import moe
    n, d, f = 3000, 136, 2184
    g = torch.Generator().manual_seed(3)
    x = (torch.randn(n, d, generator=g) * torch.exp2(torch.randint(-12, 12, (n, d // 8), generator=g).
         float()).repeat_interleave(8, 1)).bfloat16()
    x[5] = 0
    x[6, :32] = 2.0 ** -130
    xq, off, w, y = check_grouped([n - 1000, 1000], d, f, x=x)
    x[2500, 7] = float("nan")
    bad = moe.moe_grouped_swiglu_fwd_mxfp4(moe.moe_mxfp4_quantize(x.to("cuda")), off, *w, d)
    keep = torch.arange(n) != 2500
    assert torch.isnan(bad[2500]).all() and torch.equal(bad[keep], y[keep])


@pytest.mark.parametrize("T,E,k,d,f,e0,el", [(1500, 4, 3, 264, 2056, 0, 4), (5000, 8, 2, 520, 2184, 3, 2)])
def test_layer_is_its_parts(T, E, k, d, f, e0, el):
    from paper_2607_01844_amd import moe
    g = torch.Generator().manual_seed(T)
    x = torch.randn(T, d, generator=g).bfloat16().to("cuda")
    idx = torch.from_numpy(W.make_topk(T, k, E, 0.4, T)).to("cuda")
    gate = torch.softmax(torch.randn(T, k, generator=g), 1).to("cuda")
    w = weights(el, d, f, T + 1)
    y = moe.moe_ffn_fwd_mxfp4(x, idx, gate, E, *w, expert_begin=e0)
    pm = moe.moe_permute(x, idx, E, e0, el)
    off = pm["expert_offsets"]
    counts = (off[1:] - off[:-1]).tolist()
    M = sum(counts)
    rows = moe.moe_grouped_swiglu_fwd_mxfp4(moe.moe_mxfp4_quantize(pm["x_perm"]), off, *w, d)
    tok = moe.moe_grouped_swiglu_fwd_mxfp4(moe.moe_mxfp4_quantize(x), off, *w, d,
                                           row_src=pm["row_src"], k=k)
    assert torch.equal(rows[:M], tok[:M])
    assert torch.equal(y, moe.moe_combine(rows, pm["dst"], gate))
    e = max(range(el), key=lambda i: counts[i])
    a = int(off[e])
    b = min(a + 700, a + counts[e])
    vg, vu, vd = (values((q[e:e + 1], s[e:e + 1]), K)[0] for (q, s), K in zip(w, (d, d, f)))
    ref, bound = R.swiglu(R.values(pm["x_perm"][a:b].cpu().double()[None])[0], vg, vu, vd)
    assert R.close(rows[a:b].cpu(), ref, bound)


@pytest.mark.parametrize("d,f", [(8, 2056), (4104, 8)])
def test_more_tiles_than_a_workgroup_finds_at_once(d, f):
    """250,000 rows of one expert, 500 different ones over and over: every copy
    of a row has the same sums in the same order, so the same bits."""
    from paper_2607_01844_amd import moe
    P, n = 500, 250_000
    x = torch.randn(P, d, generator=torch.Generator().manual_seed(1)).bfloat16().to("cuda")
    w = weights(1, d, f, 2)
    one = torch.tensor([0, P], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    want = moe.moe_grouped_swiglu_fwd_mxfp4(moe.moe_mxfp4_quantize(x), one, *w, d)
    ref, bound = R.swiglu(values(moe.moe_mxfp4_quantize(x), d), *(values((q[0], s[0]), K) for (q, s), K in
                                                                   zip(w, (d, d, f))))
    assert R.close(want.cpu(), ref, bound)
    src = torch.arange(n, dtype=torch.int32, device="cuda") % P
    y = moe.moe_grouped_swiglu_fwd_mxfp4(moe.moe_mxfp4_quantize(x), off, *w, d, row_src=src, k=1)
    assert torch.equal(y.view(n // P, P, d), want.expand(n // P, P, d))
    del y
    big = x.repeat(n // P, 1)
    y = moe.moe_grouped_swiglu_fwd_mxfp4(moe.moe_mxfp4_quantize(big), off, *w, d)
    assert torch.equal(y.view(n // P, P, d), want.expand(n // P, P, d))


@pytest.mark.parametrize("d,f", [(8, 2056), (4104, 8)])
def test_more_small_tiles_than_a_workgroup_finds_at_once(d, f):
    check_grouped([1 + (i % 97 == 0) for i in range(1024)], d, f)

"""The layer norm's dx in the memory of dy, h or dh: the same bits as beside them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d", [(5, 520), (700, 2048), (700, 4096), (300, 16384), (3, 16392),
                                 (700, 16392)])
def test_dx_in_place_of_an_operand(T, d):
    from paper_2607_01844_amd import moe
    g = torch.Generator(device="cuda").manual_seed(T + d)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, dy, dh = (n(T, d).bfloat16() for _ in range(3))
    gamma = 1 + 0.2 * n(d)
    _, h, mean, rstd = moe.moe_layer_norm_fwd(x, gamma)
    want = moe.moe_layer_norm_bwd(dy, h, gamma, mean, rstd, dh)
    for name in ("dy", "h", "dh"):
        a = {"dy": dy.clone(), "h": h.clone(), "dh": dh.clone()}
        got = moe.moe_layer_norm_bwd(a["dy"], a["h"], gamma, mean, rstd, a["dh"], dx=a[name])
        assert got[0].data_ptr() == a[name].data_ptr()
        for u, v in zip(got, want):
            assert torch.equal(u, v), name

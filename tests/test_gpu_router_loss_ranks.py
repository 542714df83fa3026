"""The layer step with router losses on expert-parallel ranks: dx, dw_router and
dbias summed over the ranks are those of the whole layer, the losses' gradient
in them once.

Tolerance (U = 2^-24): an entry of dlogits carries 20 U of its terms' magnitudes
(dl below: the softmax terms, the chosen slots' and the losses'); dw_router and
dbias are fp32 sums over T = 256 tokens of them, on every rank and for the whole
layer: under 600 U of the sum of magnitudes a side.  dx is rounded to bf16
(2^-8 of itself at most) once by the experts and once with the router's share."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("cuts", [(0, 4, 8), (0, 1, 3, 8)])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("renorm", [0, 1])
def test_sums_over_ranks(cuts, packed, renorm):
    import workloads as W
    from paper_2607_01844_amd import moe
    wl = W.WORKLOADS["tiny"]
    inp = W.make_inputs(wl, seed=2, device="cuda")
    inp["router_bias"] = torch.linspace(-0.1, 0.1, wl.E, device="cuda")
    inp["dy"] = inp["dy"] * 0.01  # the losses' gradient is a good part of dlogits
    if packed:
        inp["seq_offsets"] = torch.tensor([0, 70, 70, 200], dtype=torch.int32, device="cuda")
        inp["token_mask"] = torch.arange(wl.T, device="cuda") % 5 != 0
    loss = (0.5, 0.25)
    whole = moe.layer_fwd_bwd(inp, wl.k, keep=False, renorm=renorm, router_loss=loss)
    ranks = []
    for a, b in zip(cuts, cuts[1:]):
        part = dict(inp, **{n: inp[n][a:b].contiguous() for n in ("w_gate", "w_up", "w_down")})
        ranks.append(moe.layer_fwd_bwd(part, wl.k, a, b - a, renorm, keep=False, router_loss=loss))
    for r in ranks:
        for key in ("balance", "zloss", "expert_counts"):
            assert torch.equal(r[key], whole[key])
    x, w = inp["x"].double(), inp["w_router"].double()
    lg = torch.empty((wl.T, wl.E), device="cuda")
    idx, gate = moe.moe_route(inp["x"], inp["w_router"], inp["router_bias"], wl.k, renorm, logits=lg)
    seq, mask = inp.get("seq_offsets"), inp.get("token_mask")
    _, _, counts, _, n = moe.moe_balance_loss_fwd(lg, idx, seq, mask)
    G = n.shape[0]
    aux = moe.moe_balance_loss_bwd(lg, counts, n, *(torch.full((G,), c / G, device="cuda") for c in loss),
                                   wl.k, seq, mask)
    t = whole["dgate"].double().abs() * gate.double()
    dl = torch.softmax(lg.double(), 1) * t.sum(1, keepdim=True) + aux.double().abs()
    dl.scatter_add_(1, idx.long(), t + gate.double() * t.sum(1, keepdim=True))
    summed = lambda key: sum(r[key].double() for r in ranks)  # noqa: E731
    mag = x.abs().t() @ dl
    assert ((summed("dw_router") - whole["dw_router"].double()).abs() <= 2 * 620 * U * mag).all()
    assert ((summed("dbias") - whole["dbias"].double()).abs() <= 2 * 620 * U * dl.sum(0)).all()
    share = dl @ w.abs().t()
    tol = 2.0 ** -8 * (sum(2 * r["dx"].double().abs() for r in ranks)
                       + 2 * whole["dx"].double().abs() + (len(ranks) + 1) * share)
    assert ((summed("dx") - whole["dx"].double()).abs() <= tol).all()
    # the losses' gradient is well above the bound: held twice it would not pass
    twice = x.t() @ aux.double()
    assert (twice.abs() > 2 * 620 * U * mag).any()

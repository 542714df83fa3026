"""A training step as it is used: embedding, a pre-norm expert layer, the last norm
with the residual, the vocabulary loss, every gradient, the gradients' norm and the
AdamW update.  Against a dense double-precision autograd of the whole step, and
captured and replayed.

Tolerance of the gradients (Frobenius norm, relative): between the embedding's row and
a gradient at most 20 values are rounded to bf16 (the row, the normed row, two hidden
activations, their product, the rows' outputs, the layer's output, the residual sum,
the last normed row; the logits' gradient, that of the last norm's output and input, of
the rows' outputs, of two hidden activations, of the rows, of the layer's input with
and without the router's share, of the norm's input, and the result), each by at most
2^-8 of the value."""
import math

import pytest
import torch

import workloads as W

pytestmark = pytest.mark.gpu
V, VB, CB, CZ, EPS = 1000, 384, 0.05, 0.02, 1e-5
NAMES = ("emb", "w_router", "w_gate", "w_up", "w_down", "norm_gamma", "norm_beta", "last_gamma",
         "last_beta", "w_voc")
HYPER = dict(beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


def setup(seed=0):
    wl = W.WORKLOADS["tiny"]
    inp = W.make_inputs(wl, seed=seed, device="cuda", with_grad=False)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    p = {k: inp[k] for k in ("w_router", "w_gate", "w_up", "w_down")}
    for k in ("w_gate", "w_up", "w_down"):
        p[k].mul_(4)
    p["emb"] = (n(V, wl.d) * 0.1).bfloat16()
    p["w_voc"] = (n(wl.d, V) * 0.1).bfloat16()
    for k in ("norm", "last"):
        p[k + "_gamma"], p[k + "_beta"] = 1 + 0.1 * n(wl.d), 0.1 * n(wl.d)
    ids = (torch.rand((wl.T,), generator=g, device="cuda") ** 3 * V).int()
    target = torch.randint(0, V, (wl.T,), generator=g, device="cuda", dtype=torch.int32)
    return wl, p, ids, target


def gradients(wl, p, ids, target):
    """One pass: the loss and every weight's gradient."""
    from paper_2607_01844_amd import moe
    scale = math.sqrt(wl.d)
    x = moe.moe_embedding_fwd(ids, p["emb"], scale)
    normed, _, _, _ = moe.moe_layer_norm_fwd(x, p["norm_gamma"], p["norm_beta"], EPS, stats=False)
    idx, gate = moe.moe_route(normed, p["w_router"], None, wl.k)
    y = moe.moe_ffn_fwd_chunked(normed, idx, gate, wl.E, p["w_gate"], p["w_up"], p["w_down"],
                                chunk=wl.T)
    z, h, mean, rstd = moe.moe_layer_norm_fwd(y, p["last_gamma"], p["last_beta"], EPS, x)
    loss, lse = moe.moe_vocab_loss_fwd(z, p["w_voc"], target, VB)
    dloss = torch.full((wl.T,), -1.0 / wl.T, device="cuda")  # of minus the mean
    dz, dvoc = moe.moe_vocab_loss_bwd(z, p["w_voc"], target, lse, dloss, VB)
    dh, dlg, dlb = moe.moe_layer_norm_bwd(dz, h, p["last_gamma"], mean, rstd)
    layer = {k: p[k] for k in ("w_router", "w_gate", "w_up", "w_down", "norm_gamma", "norm_beta")}
    out = moe.layer_fwd_bwd(dict(layer, x=x, dy=dh, norm_eps=EPS), wl.k, keep=False,
                            router_loss=(CB, CZ))
    demb = moe.moe_embedding_bwd(ids, out["dx"], V, scale)
    grad = {"emb": demb, "w_router": out["dw_router"], "w_gate": out["dw_gate"], "w_up": out["dw_up"],
            "w_down": out["dw_down"], "norm_gamma": out["dgamma"], "norm_beta": out["dbeta"],
            "last_gamma": dlg, "last_beta": dlb, "w_voc": dvoc}
    return loss, out, grad


def reference(wl, p, ids, target, idx):
    q = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    ids, target, idx = ids.long().cpu(), target.long().cpu(), idx.long().cpu()

    def norm(x, name):
        return torch.nn.functional.layer_norm(x, (wl.d,), q[name + "_gamma"], q[name + "_beta"], EPS)
    x = q["emb"][ids] * math.sqrt(wl.d)
    n = norm(x, "norm")
    logits = n @ q["w_router"]
    probs = torch.softmax(logits, 1)
    y = 0
    for e in range(wl.E):
        g = (probs[:, e] * (idx == e).any(1))[:, None]
        y = y + g * ((torch.nn.functional.silu(n @ q["w_gate"][e]) * (n @ q["w_up"][e])) @ q["w_down"][e])
    lp = torch.log_softmax(norm(x + y, "last") @ q["w_voc"], 1)[torch.arange(wl.T), target]
    count = torch.bincount(idx.flatten(), minlength=wl.E).double()
    balance = wl.E / (wl.k * wl.T ** 2) * (count * probs.sum(0)).sum()
    zloss = (torch.logsumexp(logits, 1) ** 2).mean()
    (-lp.mean() + CB * balance + CZ * zloss).backward()
    return lp.detach(), {k: v.grad for k, v in q.items()}


def test_gradients_of_the_whole_step():
    wl, p, ids, target = setup()
    loss, out, grad = gradients(wl, p, ids, target)
    lp, ref = reference(wl, p, ids, target, out["topk_idx"])
    tol = 20 * 2.0 ** -8
    # a logit's error: the last normed row's (nine roundings before it) over the row
    assert float((loss.cpu().double() - lp).norm() / lp.norm()) <= tol
    for k in NAMES:
        err = float((grad[k].cpu().double() - ref[k]).norm() / ref[k].norm())
        print(f"{k}: {err:.2e}", flush=True)
        assert err <= tol, k


def weights(p, bits):
    """Updated tensors in their own memory: fp32 masters of the bf16 weights, which
    the passes read the copies of."""
    from paper_2607_01844_amd import moe
    master = {k: p[k].float().clone() for k in NAMES}
    live = {k: p[k].clone() if p[k].dtype is torch.bfloat16 else master[k] for k in NAMES}
    copies = [live[k] if live[k].dtype is torch.bfloat16 else None for k in NAMES]
    g = [torch.zeros_like(p[k]) for k in NAMES]
    return moe.Params([master[k] for k in NAMES], g, w_copy=copies, bits=bits), live


def one_step(wl, params, live, ids, target, lr, step):
    from paper_2607_01844_amd import moe
    _, _, grad = gradients(wl, live, ids, target)
    for held, k in zip(params.g, NAMES):
        held.copy_(grad[k])
    q = moe.moe_grad_sumsq(params)
    moe.moe_adamw_step(params, lr, step, grad_sumsq=q, max_norm=0.5, seed=3, **HYPER)
    return q


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_are_the_eager_ones(bits):
    wl, p, ids, target = setup(1)
    eager, live = weights(p, bits)
    steps = [(2.0 ** -10, 1), (2.0 ** -9, 2), (2.0 ** -11, 3), (2.0 ** -11, 4)]  # exact in fp32 too
    sums = [one_step(wl, eager, live, ids, target, lr, t).clone() for lr, t in steps]
    assert float(sums[0]) > 0.25  # clipped

    params, live2 = weights(p, bits)
    lr, t = torch.zeros(1, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # the stream's workspaces, and nothing moved: lr is 0
        gradients(wl, live2, ids, target)
        from paper_2607_01844_amd import moe
        moe.moe_grad_sumsq(params)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        q = one_step(wl, params, live2, ids, target, lr, t)
    for (rate, n), want in zip(steps, sums):
        lr.fill_(rate)
        t.fill_(n)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, want), n
        gradients(wl, live, ids, target)  # eager work in between
    for a, b in zip(eager.w + eager.m + eager.v, params.w + params.m + params.v):
        for x, y in zip(a, b) if isinstance(a, tuple) else [(a, b)]:
            assert torch.equal(x, y)
    for k in NAMES:
        assert torch.equal(live[k], live2[k])


def test_blocks_norm_is_the_separate_calls():
    from paper_2607_01844_amd import moe
    wl, p, ids, target = setup(2)
    x = moe.moe_embedding_fwd(ids, p["emb"], 3.0)
    res = moe.moe_embedding_fwd(target, p["emb"], 2.0)
    dy = torch.randn(x.shape, device="cuda").bfloat16()
    layer = {k: p[k] for k in ("w_router", "w_gate", "w_up", "w_down")}
    out = moe.layer_fwd_bwd(dict(layer, x=x, dy=dy, norm_gamma=p["norm_gamma"], residual=res), wl.k,
                            router_loss=(CB, CZ))
    n, h, mean, rstd = moe.moe_layer_norm_fwd(x, p["norm_gamma"], None, 1e-5, res)
    ref = moe.layer_fwd_bwd(dict(layer, x=n, dy=dy), wl.k, router_loss=(CB, CZ))
    dx, dgamma, _ = moe.moe_layer_norm_bwd(ref["dx"], h, p["norm_gamma"], mean, rstd, dy)
    for k in ("y", "dw_gate", "dw_router"):
        assert torch.equal(out[k], ref[k])
    assert torch.equal(out["dx"], dx) and torch.equal(out["dgamma"], dgamma)
    assert torch.equal(out["h"], h) and out["dbeta"] is None
    with pytest.raises(ValueError):
        moe.layer_fwd_bwd(dict(layer, x=x, dy=dy, residual=res), wl.k)
    with pytest.raises(ValueError):
        moe.layer_fwd_bwd(dict(layer, x=x, dy=dy, norm_gamma=p["norm_gamma"]), wl.k, 0, 4)


def passes(seed):
    """Calls with workspaces, and an update, on tensors of their own."""
    from paper_2607_01844_amd import moe
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(-1, 700, (9000,), generator=g, device="cuda", dtype=torch.int32)
    few = ids[:500].clone()
    dy = torch.randn((9000, 264), generator=g, device="cuda").bfloat16()
    gamma = torch.ones(264, device="cuda")
    y, h, mean, rstd = moe.moe_layer_norm_fwd(dy, gamma)
    p = moe.Params([torch.randn(20001, generator=g, device="cuda")], [dy.view(-1)[:20001]], bits=8)

    def run():
        q = moe.moe_grad_sumsq(p)
        moe.moe_adamw_step(p, 1e-2, 1, grad_sumsq=q, max_norm=1.0)
        return [moe.moe_embedding_bwd(ids, dy, 700, 0.5), moe.moe_embedding_bwd(few, dy[:500], 700),
                *moe.moe_layer_norm_bwd(y, h, gamma, mean, rstd, dy), q, *moe.moe_adamw_states(p)[0]], p
    return run


def test_replayed_at_once():
    def start(p):
        p.w[0].fill_(1)
        for x in (*p.m[0], *p.v[0]):
            x.zero_()
    runs, want = [passes(1), passes(2)], []
    for run in runs:
        out, p = run()
        start(p)
        out, p = run()
        want.append([v.clone() for v in out + [p.w[0]]])
    streams = [torch.cuda.Stream() for _ in runs]
    graphs, outs, held = [], [], []
    for run, s in zip(runs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()  # the stream's workspaces
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out, p = run()
        outs.append(out + [p.w[0]])
        held.append(p)
        graphs.append(graph)
    for _ in range(4):
        for out, p in zip(outs, held):
            for v in out[:-1]:
                v.fill_(7)
            start(p)
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for out, ref in zip(outs, want):
            for a, b in zip(out, ref):
                assert torch.equal(a, b)

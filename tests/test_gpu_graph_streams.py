"""Two graphs captured on streams of their own work in buffers of their own:
replayed at once, each gives its eager results."""
import pytest
import torch

from tests.test_gpu_distill import make

pytestmark = pytest.mark.gpu


def passes(seed):
    """One training pass of the vocabulary losses and the router losses."""
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(700, 264, 9001, 20, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dl = torch.randn(700, generator=g, device="cuda")
    lg = torch.randn((9000, 72), generator=g, device="cuda")
    idx = torch.topk(lg, 2).indices.int()
    one = torch.ones(1, device="cuda")
    src = torch.randn((700, 264), generator=g, device="cuda").bfloat16()

    def run():
        loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 1024)
        dx, dw = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, 1024)
        bal, z, c, ps, n = moe.moe_balance_loss_fwd(lg, idx)
        return [loss, lse, dx, dw, bal, z, c, ps, moe.moe_balance_loss_bwd(lg, c, n, one, one, 2),
                *moe.moe_mxfp4_quantize(src)]
    return run


def test_replayed_at_once():
    runs = [passes(1), passes(2)]
    want = [[v.clone() for v in run()] for run in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    graphs, outs = [], []
    for run, s in zip(runs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()  # the stream's workspaces
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(run())
        graphs.append(graph)
    for _ in range(4):
        for out in outs:
            for v in out:
                v.fill_(7)
        torch.cuda.synchronize()
        for _ in range(3):
            for graph, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    graph.replay()
        torch.cuda.synchronize()
        for out, ref in zip(outs, want):
            for a, b in zip(out, ref):
                assert torch.equal(a, b)

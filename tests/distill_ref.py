"""Distillation from a teacher's top logits in 64 bits, dense (torch, CPU; the
tests' reference)."""
import math

import torch


def teacher(ids, t, V, tau, tlse=None):
    """(p [N][K], log p where p > 0 and else 0)."""
    there = (ids >= 0) & (ids < V)
    t = torch.where(there, t.double() / tau, -math.inf)
    if tlse is None:
        shift = torch.logsumexp(t, 1, keepdim=True)
        shift = torch.where(shift == -math.inf, 0.0, shift)
    else:
        shift = tlse.double()[:, None]
    logp = t - shift
    p = torch.exp(logp)
    return p, torch.where(p > 0, logp, 0.0)


def forward(x, w, ids, t, tau=1.0, tlse=None):
    """(loss [N], lse [N], y_topk [N][K]); x, w of any float type."""
    V = w.shape[1]
    y = x.double() @ w.double()
    p, logp = teacher(ids, t, V, tau, tlse)
    there = (ids >= 0) & (ids < V)
    yk = torch.where(there, y.gather(1, torch.where(there, ids, 0).long()), 0.0)
    lse = torch.logsumexp(y / tau, 1)
    return (p * (logp - yk / tau + lse[:, None])).sum(1), lse, yk


def logit_grad(x, w, ids, t, dloss, tau=1.0, tlse=None):
    """G [N][V], the gradient of the logits."""
    V = w.shape[1]
    y = x.double() @ w.double()
    p, _ = teacher(ids, t, V, tau, tlse)
    c = dloss.double()[:, None] / tau
    G = torch.softmax(y / tau, 1) * (c * p.sum(1, keepdim=True))
    there = (ids >= 0) & (ids < V)
    return G.scatter_add(1, torch.where(there, ids, 0).long(), -c * p)

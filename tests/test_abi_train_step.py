"""Host-side refusals of the embedding, the layer norm and the weight updates
(no GPU work)."""
import ctypes
import math

import pytest

from tests.abi_cases import MIS, P, Z

BIG = 1 << 40


def _no_gpu():
    import torch
    return not torch.cuda.is_available()


pytestmark = pytest.mark.skipif(not _no_gpu(), reason="dummy pointers are only safe without a GPU")


@pytest.fixture(scope="module")
def lib():
    from paper_2607_01844_amd import moe
    return moe.lib


def efwd(ids=P, w=P, N=10, H=64, begin=0, rows=100, scale=1.0, y=P):
    return lambda L: L.moe_embedding_fwd(ids, w, N, H, begin, rows, scale, y, Z)


def ebwd(ids=P, dy=P, N=10, H=64, begin=0, rows=100, scale=1.0, dw=P, ws=P, nws=BIG):
    return lambda L: L.moe_embedding_bwd(ids, dy, N, H, begin, rows, scale, dw, ws, nws, Z)


def nfwd(x=P, res=P, gamma=P, beta=P, T=10, d=64, eps=1e-5, h=P, y=P, mean=P, rstd=P):
    return lambda L: L.moe_layer_norm_fwd(x, res, gamma, beta, T, d, eps, h, y, mean, rstd, Z)


def nbwd(dy=P, h=P, gamma=P, mean=P, rstd=P, dh=P, T=10, d=64, dx=P, dg=P, db=P, ws=P, nws=BIG):
    return lambda L: L.moe_layer_norm_bwd(dy, h, gamma, mean, rstd, dh, T, d, dx, dg, db, ws, nws,
                                          Z)


def params(**k):
    from paper_2607_01844_amd import _abi
    p = dict(w=4096, w_copy=None, g=4096, m=4096, v=4096, m_scale=4097, v_scale=4099, n=10,
             w_type=0, g_type=1)
    p.update(k)
    return (_abi.Param * 1)(_abi.Param(**p))


def step(bits=32, count=1, opt=True, **k):
    from paper_2607_01844_amd import _abi
    o = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=1, lr_device=None,
             step_device=None, grad_sumsq=None, max_norm=1.0, seed=0)
    o.update({n: k.pop(n) for n in list(k) if n in o})
    o = _abi.AdamWOptions(**o)
    return lambda L: L.moe_adamw_step(params(**k), count, bits, ctypes.byref(o) if opt else Z, Z)


def sumsq(out=P, ws=P, nws=BIG, count=1, **k):
    return lambda L: L.moe_grad_sumsq(params(**k), count, out, ws, nws, Z)


def states(m=4096, v=4096, count=1, **k):
    a, b = ((ctypes.c_void_p * 1)(x) for x in (m, v))
    return lambda L: L.moe_adamw_states(params(**k), count, a, b, Z)


INVALID = [
    ("embed N<0", efwd(N=-1)), ("embed N large", efwd(N=1 << 26)), ("embed H % 8", efwd(H=60)),
    ("embed H 0", efwd(H=0)), ("embed N*H", efwd(N=1 << 21, H=1 << 17)),
    ("embed rows 0", efwd(rows=0)), ("embed rows large", efwd(rows=1 << 28)),
    ("embed begin", efwd(begin=-1)), ("embed end", efwd(begin=(1 << 31) - 99)),
    ("embed begin overflow", efwd(begin=(1 << 63) - 1)),
    ("embed scale nan", efwd(scale=math.nan)), ("embed scale inf", efwd(scale=math.inf)),
    ("embed null ids", efwd(ids=Z)), ("embed null w", efwd(w=Z)), ("embed null y", efwd(y=Z)),
    ("embed misaligned", efwd(w=MIS)),
    ("embed bwd N<0", ebwd(N=-1)), ("embed bwd H % 8", ebwd(H=4)), ("embed bwd rows", ebwd(rows=0)),
    ("embed bwd null dw", ebwd(dw=Z)), ("embed bwd null dw, no tokens", ebwd(dw=Z, N=0)),
    ("embed bwd null dy", ebwd(dy=Z)), ("embed bwd null ids", ebwd(ids=Z)),
    ("embed bwd misaligned ws", ebwd(ws=MIS)), ("embed bwd scale", ebwd(scale=math.inf)),
    ("norm T<0", nfwd(T=-1)), ("norm T large", nfwd(T=1 << 31)), ("norm d % 8", nfwd(d=12)),
    ("norm d large", nfwd(d=262152)), ("norm eps 0", nfwd(eps=0.0)), ("norm eps nan", nfwd(eps=math.nan)),
    ("norm eps<0", nfwd(eps=-1.0)), ("norm null x", nfwd(x=Z)), ("norm null gamma", nfwd(gamma=Z)),
    ("norm null y", nfwd(y=Z)), ("norm null h", nfwd(h=Z)), ("norm misaligned residual", nfwd(res=MIS)),
    ("norm misaligned mean", nfwd(mean=MIS)), ("norm misaligned beta", nfwd(beta=MIS)),
    ("norm bwd T<0", nbwd(T=-1)), ("norm bwd d", nbwd(d=0)), ("norm bwd null dy", nbwd(dy=Z)),
    ("norm bwd null h", nbwd(h=Z)), ("norm bwd null mean", nbwd(mean=Z)),
    ("norm bwd null rstd", nbwd(rstd=Z)), ("norm bwd null dx", nbwd(dx=Z)),
    ("norm bwd null dgamma", nbwd(dg=Z)), ("norm bwd misaligned dh", nbwd(dh=MIS)),
    ("norm bwd misaligned dbeta", nbwd(db=MIS)), ("norm bwd misaligned ws", nbwd(ws=MIS)),
    ("sumsq count", sumsq(count=-1)), ("sumsq null out", sumsq(out=Z)), ("sumsq null g", sumsq(g=None)),
    ("sumsq type", sumsq(g_type=2)), ("sumsq n<0", sumsq(n=-1)), ("sumsq n large", sumsq(n=1 << 40)),
    ("sumsq misaligned g", sumsq(g=4098)), ("sumsq misaligned ws", sumsq(ws=MIS)),
    ("sumsq misaligned out", sumsq(out=MIS)),
    ("adamw bits", step(bits=16)), ("adamw no options", step(opt=False)), ("adamw count", step(count=-1)),
    ("adamw lr", step(lr=math.nan)), ("adamw beta1", step(beta1=1.0)), ("adamw beta2", step(beta2=-0.1)),
    ("adamw beta nan", step(beta2=math.nan)), ("adamw eps", step(eps=0.0)), ("adamw eps small", step(eps=9e-21)),
    ("adamw decay", step(weight_decay=math.inf)), ("adamw step 0", step(step=0)),
    ("adamw step large", step(step=1 << 31)), ("adamw max_norm", step(grad_sumsq=4096, max_norm=0.0)),
    ("adamw max_norm nan", step(grad_sumsq=4096, max_norm=math.nan)),
    ("adamw misaligned sumsq", step(grad_sumsq=4098)), ("adamw misaligned lr", step(lr_device=4100)),
    ("adamw misaligned step", step(step_device=4100)),
    ("adamw null w", step(w=None)), ("adamw null m", step(m=None)), ("adamw null v", step(v=None)),
    ("adamw null g", step(g=None)), ("adamw w_type", step(w_type=3)), ("adamw g_type", step(g_type=-1)),
    ("adamw copy of bf16", step(w_type=1, w_copy=4096)), ("adamw misaligned w", step(w=4104)),
    ("adamw misaligned copy", step(w_copy=4104)), ("adamw misaligned codes", step(bits=8, m=4097)),
    ("adamw no scales", step(bits=8, m_scale=None)), ("adamw no v scales", step(bits=8, v_scale=None)),
    ("states null m", states(m=None)), ("states null v", states(v=None)), ("states count", states(count=-1)),
    ("states misaligned", states(m=4100)), ("states no scales", states(m_scale=None)),
]


@pytest.mark.parametrize("case", INVALID, ids=[c[0] for c in INVALID])
def test_invalid_arguments_rejected_on_host(lib, case):
    assert case[1](lib) == -1
    assert lib.moe_last_error()


def test_null_lists(lib):
    n = ctypes.c_size_t()
    assert lib.moe_grad_sumsq_workspace_bytes(Z, 1, ctypes.byref(n)) == -1
    assert lib.moe_grad_sumsq_workspace_bytes(params(), 1, Z) == -1
    assert lib.moe_adamw_states(params(), 1, Z, Z, Z) == -1
    assert lib.moe_adamw_states(Z, 1, Z, Z, Z) == -1


def test_workspaces(lib):
    def query(name, *a):
        n = ctypes.c_size_t()
        return getattr(lib, name)(*a, ctypes.byref(n)), n.value
    for N, H, rows in ((1, 8, 1), (1, 262144, 9), (9, 262144, 1 << 20), (8192, 128, 1000), (8193, 4096, 200000), (65536, 4096, 200000),
                       ((1 << 26) - 1, 2048, (1 << 28) - 1)):
        rc, n = query("moe_embedding_bwd_workspace_bytes", N, H, rows)
        assert rc == 0 and 0 < n <= (N + 7) * H + 24 * N + (1 << 20), (N, H, rows, n)
        assert ebwd(N=N, H=H, rows=rows, nws=n - 1)(lib) == -3
        assert ebwd(N=N, H=H, rows=rows, ws=Z)(lib) == -3
    for T, d in ((1, 8), (65536, 4096), (5, 262144), ((1 << 31) - 1, 64)):
        rc, n = query("moe_layer_norm_bwd_workspace_bytes", T, d)
        assert rc == 0 and 0 < n <= 1 << 28
        assert nbwd(T=T, d=d, nws=n - 1)(lib) == -3
    for n in (0, 1, 1 << 39):
        rc, b = query("moe_grad_sumsq_workspace_bytes", params(n=n), 1)
        assert rc == 0 and 0 < b <= 1 << 20
        assert sumsq(n=n, nws=b - 1)(lib) == -3
    assert query("moe_embedding_bwd_workspace_bytes", -1, 8, 1)[0] == -1
    assert query("moe_embedding_bwd_workspace_bytes", 0, 8, 1)[0] == 0
    assert query("moe_layer_norm_bwd_workspace_bytes", 0, 8)[0] == 0
    assert query("moe_layer_norm_bwd_workspace_bytes", 1, 7)[0] == -1


def test_empty_lists_and_tensors_are_no_work(lib):
    assert step(count=0)(lib) == 0
    assert step(n=0, w=None, g=None, m=None, v=None)(lib) == 0
    assert states(n=0, m=None, v=None)(lib) == 0
    assert efwd(N=0, ids=Z, w=Z, y=Z)(lib) == 0
    assert nfwd(T=0, x=Z, gamma=Z, y=Z)(lib) == 0

"""Host-side refusals of the distillation loss (no GPU work)."""
import ctypes

import pytest

from tests.abi_cases import MIS, P, Z

BIG = 1 << 30


def _no_gpu():
    import torch
    return not torch.cuda.is_available()


pytestmark = pytest.mark.skipif(not _no_gpu(), reason="dummy pointers are only safe without a GPU")


@pytest.fixture(scope="module")
def lib():
    from paper_2607_01844_amd import moe
    return moe.lib


def fwd(x=P, w=P, ids=P, t=P, tl=Z, tau=1.0, N=10, H=64, V=100, vb=16, K=4, loss=P, lse=P, yk=P,
        ws=P, nws=BIG):
    return lambda L: L.moe_vocab_distill_fwd(x, w, ids, t, tl, tau, N, H, V, vb, K, loss, lse, yk,
                                             ws, nws, Z)


def bwd(x=P, w=P, ids=P, t=P, tl=Z, tau=1.0, lse=P, yk=P, dl=P, N=10, H=64, V=100, vb=16, K=4, dx=P,
        dw=P, ws=P, nws=BIG):
    return lambda L: L.moe_vocab_distill_bwd(x, w, ids, t, tl, tau, lse, yk, dl, N, H, V, vb, K, dx,
                                             dw, ws, nws, Z)


BAD = [dict(N=-1), dict(N=1 << 26), dict(N=1 << 24, K=128), dict(H=60), dict(H=0), dict(V=0),
       dict(V=1 << 31), dict(vb=12), dict(vb=0), dict(K=0), dict(K=257), dict(tau=0.0),
       dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")), dict(tau=2000.0),
       dict(tau=1e-4), dict(x=Z), dict(w=Z), dict(ids=Z), dict(t=Z), dict(x=MIS), dict(ids=MIS),
       dict(tl=MIS), dict(lse=Z), dict(yk=Z), dict(yk=MIS), dict(ws=MIS)]


@pytest.mark.parametrize("kw", BAD + [dict(loss=Z), dict(loss=MIS)], ids=str)
def test_forward_refuses(lib, kw):
    assert fwd(**kw)(lib) == -1
    assert lib.moe_last_error().startswith(b"moe_vocab_distill_fwd")


@pytest.mark.parametrize("kw", BAD + [dict(dl=Z), dict(dx=Z), dict(dw=Z), dict(dx=MIS),
                                      dict(dw=MIS), dict(dw=Z, N=0)], ids=str)
def test_backward_refuses(lib, kw):
    assert bwd(**kw)(lib) == -1
    assert lib.moe_last_error().startswith(b"moe_vocab_distill_bwd")


def test_workspace(lib):
    n, v = ctypes.c_size_t(), ctypes.c_size_t()
    q = lib.moe_vocab_distill_workspace_bytes
    assert q(4096, 2048, 200000, 16384, 64, ctypes.byref(n)) == 0
    assert lib.moe_vocab_loss_workspace_bytes(4096, 2048, 200000, 16384, ctypes.byref(v)) == 0
    # beside the plain loss's: a probability and an entry of every slot and a factor a row
    assert v.value + 4 * 4096 * 129 <= n.value <= v.value + 4 * 4096 * 129 + 1024
    assert q(4096, 2048, 400000, 16384, 64, ctypes.byref(v)) == 0
    assert v.value == n.value  # independent of V
    # few rows: blocks are taken together, within 64 MiB of logit gradients
    assert q(1000, 520, 32003, 4096, 20, ctypes.byref(n)) == 0
    assert 2 * 1000 * 32003 <= n.value <= 2 * 1000 * 32008 + 8 * 4 * 1000 * 520 + 2 * 520 * 32008 + (1 << 20)
    assert q(10, 64, 100, 16, 4, ctypes.byref(n)) == 0
    assert bwd(nws=16)(lib) == fwd(nws=16)(lib) == fwd(ws=Z)(lib) == -3
    assert q(10, 64, 100, 16, 0, ctypes.byref(n)) == q(10, 64, 100, 16, 4, None) == -1
    assert q(1 << 20, 262144, (1 << 31) - 1, 1 << 19, 256, ctypes.byref(n)) == 0


def test_no_rows_need_no_pointers(lib):
    assert fwd(x=Z, w=Z, ids=Z, t=Z, loss=Z, lse=Z, yk=Z, ws=Z, nws=0, N=0)(lib) == 0

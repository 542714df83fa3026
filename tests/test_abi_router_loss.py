"""Host-side refusals of the router's losses (no GPU work)."""
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


def fwd(logits=P, idx=P, off=P, mask=P, T=10, E=8, k=2, G=3, bal=P, z=P, counts=P, ps=P, n=P, ws=P,
        nws=BIG):
    return lambda L: L.moe_balance_loss_fwd(logits, idx, off, mask, T, E, k, G, bal, z, counts, ps,
                                            n, ws, nws, Z)


def bwd(logits=P, counts=P, n=P, db=P, dz=P, off=P, mask=P, T=10, E=8, k=2, G=3, dl=P, acc=0):
    return lambda L: L.moe_balance_loss_bwd(logits, counts, n, db, dz, off, mask, T, E, k, G, dl,
                                            acc, Z)


def aux(d=P, T=10):
    return lambda L: L.moe_route_bwd_aux(P, P, P, P, P, P, d, T, 64, 8, 2, 0, P, Z, Z, 1, Z, P,
                                         BIG, Z)


INVALID = [
    ("fwd E 0", fwd(E=0)), ("fwd E > max", fwd(E=1025)), ("fwd k > E", fwd(E=2, k=3)),
    ("fwd k 0", fwd(k=0)), ("fwd T<0", fwd(T=-1)), ("fwd T*k", fwd(T=1 << 30)),
    ("fwd G 0", fwd(G=0)), ("fwd G > max", fwd(G=65536)), ("fwd no offsets", fwd(off=Z)),
    ("fwd null logits", fwd(logits=Z)), ("fwd null idx", fwd(idx=Z)),
    ("fwd null counts", fwd(counts=Z)), ("fwd null balance", fwd(bal=Z)),
    ("fwd null zloss", fwd(z=Z)), ("fwd null prob_sum", fwd(ps=Z)), ("fwd null n", fwd(n=Z)),
    ("fwd misaligned logits", fwd(logits=MIS)), ("fwd misaligned offsets", fwd(off=MIS)),
    ("fwd misaligned mask", fwd(mask=MIS)), ("fwd misaligned workspace", fwd(ws=MIS)),
    ("bwd null dlogits", bwd(dl=Z)), ("bwd null dbalance", bwd(db=Z)), ("bwd null dzloss", bwd(dz=Z)),
    ("bwd null n", bwd(n=Z)), ("bwd null counts", bwd(counts=Z)), ("bwd accumulate", bwd(acc=2)),
    ("bwd no offsets", bwd(off=Z)), ("bwd misaligned dlogits", bwd(dl=MIS)),
    ("bwd G 0", bwd(G=0)), ("bwd k > max", bwd(E=64, k=17)),
    ("aux null", aux(Z)), ("aux misaligned", aux(MIS)),
]


@pytest.mark.parametrize("case", INVALID, ids=[c[0] for c in INVALID])
def test_invalid_arguments_rejected_on_host(lib, case):
    assert case[1](lib) == -1
    assert len(lib.moe_last_error()) > 0


def test_workspace(lib):
    n = ctypes.c_size_t()
    assert lib.moe_balance_loss_workspace_bytes(65536, 128, 1, ctypes.byref(n)) == 0
    assert 0 < n.value < 1 << 20
    assert fwd(T=65536, E=128, G=1, nws=n.value - 1)(lib) == -3
    assert fwd(ws=Z)(lib) == -3
    for T in (0, 1, (1 << 31) - 1):
        assert lib.moe_balance_loss_workspace_bytes(T, 1024, 65535, ctypes.byref(n)) == 0
    for T, E, G in ((-1, 8, 1), (10, 0, 1), (10, 8, 0), (10, 8, 65536), (1 << 31, 8, 1)):
        assert lib.moe_balance_loss_workspace_bytes(T, E, G, ctypes.byref(n)) == -1
    assert lib.moe_balance_loss_workspace_bytes(10, 8, 1, None) == -1


def test_no_tokens_need_no_backward_pointers(lib):
    assert bwd(logits=Z, counts=Z, n=Z, db=Z, dz=Z, dl=Z, T=0)(lib) == 0

"""Host-side refusals of the MXFP4 calls (no GPU work)."""
import ctypes

import pytest

from tests.abi_cases import MIS, P, Z

BIG = 1 << 34


def _no_gpu():
    import torch
    return not torch.cuda.is_available()


pytestmark = pytest.mark.skipif(not _no_gpu(), reason="dummy pointers are only safe without a GPU")


@pytest.fixture(scope="module")
def lib():
    from paper_2607_01844_amd import moe
    return moe.lib


def quant(src=P, B=2, R=64, C=64, tr=0, q=P, s=P):
    return lambda L: L.moe_mxfp4_quantize(src, B, R, C, tr, q, s, Z)


def dequant(q=P, s=P, B=2, rows=64, K=64, dst=P):
    return lambda L: L.moe_mxfp4_dequantize(q, s, B, rows, K, dst, Z)


def ffn(xq=P, xs=P, xr=100, src=P, k=2, off=P, E=4, cap=100, d=64, f=32, wgq=P, wgs=P, wuq=P, wus=P,
        wdq=P, wds=P, y=P, ws=P, nws=BIG):
    return lambda L: L.moe_grouped_swiglu_fwd_mxfp4(xq, xs, xr, src, k, off, E, cap, d, f, wgq, wgs,
                                                    wuq, wus, wdq, wds, y, ws, nws, Z)


def layer(x=P, idx=P, gate=P, T=10, d=64, E=8, k=2, eb=0, el=8, f=32, wgq=P, wgs=P, wuq=P, wus=P,
          wdq=P, wds=P, y=P, ws=P, nws=BIG):
    return lambda L: L.moe_ffn_fwd_mxfp4(x, idx, gate, T, d, E, k, eb, el, f, wgq, wgs, wuq, wus, wdq,
                                         wds, y, ws, nws, Z)


QUANT = [dict(B=-1), dict(B=65536), dict(R=-1), dict(R=1 << 25), dict(B=1024, R=1 << 15), dict(C=0),
         dict(C=12), dict(C=262152), dict(tr=2), dict(tr=1, R=60), dict(tr=1, R=262152),
         dict(tr=1, B=60000, R=8, C=1024), dict(src=Z), dict(q=Z), dict(s=Z), dict(src=MIS), dict(q=MIS),
         dict(s=MIS)]
DEQUANT = [dict(B=-1), dict(rows=1 << 25), dict(K=12), dict(K=0), dict(q=Z), dict(s=Z), dict(dst=Z),
           dict(q=MIS), dict(s=MIS), dict(dst=MIS)]
WEIGHTS = [dict([(n, v)]) for n in ("wgq", "wgs", "wuq", "wus", "wdq", "wds") for v in (Z, MIS)]
FFN = WEIGHTS + [dict(xq=Z), dict(xs=Z), dict(xq=MIS), dict(xs=MIS), dict(src=MIS), dict(off=Z), dict(y=Z),
                 dict(y=MIS), dict(k=0), dict(k=17), dict(E=0), dict(E=1025), dict(cap=-1),
                 dict(cap=1 << 31), dict(d=60), dict(f=36), dict(xr=-1), dict(xr=0),
                 dict(xr=1 << 26, d=64), dict(src=Z, xr=99), dict(d=65536, f=65536), dict(ws=MIS)]
LAYER = WEIGHTS + [dict(x=Z), dict(idx=Z), dict(gate=Z), dict(y=Z), dict(x=MIS), dict(T=-1), dict(k=9),
                   dict(k=0), dict(E=1025), dict(eb=-1), dict(eb=1), dict(el=0), dict(el=9), dict(d=60),
                   dict(f=36), dict(T=1 << 25, k=1), dict(T=1 << 20, d=8192), dict(ws=MIS),
                   dict(eb=2147483647)]


@pytest.mark.parametrize("make,kw", [(m, kw) for m, cases in ((quant, QUANT), (dequant, DEQUANT),
                                                             (ffn, FFN), (layer, LAYER))
                                     for kw in cases], ids=lambda v: str(v) if isinstance(v, dict)
                         else v.__name__)
def test_refuses(lib, make, kw):
    assert make(**kw)(lib) == -1
    assert len(lib.moe_last_error()) > 0


def test_sizes_and_workspaces(lib):
    q, s, n = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.moe_mxfp4_bytes(3, 10, 264, ctypes.byref(q), ctypes.byref(s)) == 0
    assert q.value == 3 * 10 * 16 * 9 and s.value == 3 * 2 * 10 * 8
    assert lib.moe_mxfp4_bytes(3, 10, 260, ctypes.byref(q), ctypes.byref(s)) == -1
    assert lib.moe_mxfp4_bytes(3, 10, 264, None, ctypes.byref(s)) == -1
    w = lib.moe_grouped_swiglu_mxfp4_workspace_bytes
    assert w(24576, 64, 2048, 1408, ctypes.byref(n)) == 0
    # activations of half a byte a value and their scales, the rows' tokens and scales
    assert 24576 * (704 + 48 + 64 + 4) <= n.value <= 24576 * (704 + 48 + 64 + 4) + 8192
    assert w(24576, 64, 2044, 1408, ctypes.byref(n)) == w(1, 1, 8, 8, None) == -1
    assert w(100, 4, 64, 32, ctypes.byref(n)) == 0
    assert ffn(nws=n.value - 1)(lib) == ffn(ws=Z)(lib) == -3
    w = lib.moe_ffn_fwd_mxfp4_workspace_bytes
    assert w(10, 8, 2, 8, 64, 32, ctypes.byref(n)) == 0
    assert layer(nws=n.value - 1)(lib) == layer(ws=Z)(lib) == -3
    for T in (0, 1 << 31, 1 << 40):
        w(T, 1024, 16, 1024, 8, 8, ctypes.byref(n))
    assert w(10, 8, 2, 9, 64, 32, ctypes.byref(n)) == -1


def test_nothing_to_do_needs_no_pointers(lib):
    assert quant(src=Z, q=Z, s=Z, R=0)(lib) == quant(src=Z, q=Z, s=Z, B=0)(lib) == 0
    assert dequant(q=Z, s=Z, dst=Z, rows=0)(lib) == 0
    assert layer(x=Z, idx=Z, gate=Z, y=Z, wgq=Z, wgs=Z, wuq=Z, wus=Z, wdq=Z, wds=Z, ws=Z, nws=0,
                 T=0)(lib) == 0
    assert ffn(xq=Z, xs=Z, y=Z, xr=0, cap=0)(lib) == 0

"""Workspace queries of the router losses, distillation and MXFP4 calls from
one token to the largest sizes: host arithmetic without overflow, never less
for more."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2607_01844_amd import moe
    return moe.lib


def ask(lib, name, *a):
    n = ctypes.c_size_t(1)
    r = getattr(lib, name)(*a, ctypes.byref(n))
    return r, n.value


@pytest.mark.parametrize("name,calls", [
    ("moe_balance_loss_workspace_bytes",
     [(0, 1, 1), (1, 8, 1), (4096, 64, 1), (65536, 128, 64), (1 << 30, 1024, 65535), ((1 << 31) - 1, 1024, 65535)]),
    ("moe_vocab_distill_workspace_bytes",
     [(1, 8, 1, 8, 1), (256, 128, 1000, 256, 8), (4096, 2048, 200000, 16384, 64),
      (1 << 20, 8192, 1 << 20, 1 << 16, 256)]),
    ("moe_grouped_swiglu_mxfp4_workspace_bytes",
     [(1, 1, 8, 8), (1100, 12, 520, 328), (65536, 128, 4096, 1536), (1 << 20, 1024, 8192, 8192)]),
    ("moe_ffn_fwd_mxfp4_workspace_bytes",
     [(1, 8, 2, 8, 64, 64), (4096, 64, 6, 64, 2048, 1408), (65536, 384, 8, 32, 7168, 2048)])])
def test_queries(lib, name, calls):
    last = 0
    for c in calls:
        r, n = ask(lib, name, *c)
        assert r == 0 and last <= n < 1 << 48, (c, r, n)
        last = n


@pytest.mark.parametrize("name,call", [
    ("moe_balance_loss_workspace_bytes", (-1, 8, 1)), ("moe_balance_loss_workspace_bytes", (1, 1025, 1)),
    ("moe_balance_loss_workspace_bytes", (1, 8, 0)), ("moe_balance_loss_workspace_bytes", (1, 8, 65536)),
    ("moe_vocab_distill_workspace_bytes", (1, 8, 10, 8, 257)), ("moe_vocab_distill_workspace_bytes", (1, 8, 10, 12, 1)),
    ("moe_vocab_distill_workspace_bytes", (1 << 62, 8, 10, 8, 1)),
    ("moe_grouped_swiglu_mxfp4_workspace_bytes", (-1, 1, 8, 8)),
    ("moe_grouped_swiglu_mxfp4_workspace_bytes", (1 << 62, 1, 8, 8)),
    ("moe_ffn_fwd_mxfp4_workspace_bytes", (1 << 62, 8, 2, 8, 64, 64)),
    ("moe_ffn_fwd_mxfp4_workspace_bytes", (1, 8, 2, 9, 64, 64))])
def test_absurd_queries_are_refused(lib, name, call):
    assert ask(lib, name, *call)[0] != 0

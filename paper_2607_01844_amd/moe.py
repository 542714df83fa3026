"""Thin Python binding of libmoe.so (the MI355X MoE expert-layer library).

Every function has the name of the C entry point it calls and only marshals
arguments: it checks dtype/device/contiguity, allocates outputs and
workspaces with torch (device memory), and passes raw pointers plus the
current HIP stream.  All arithmetic runs in the library's HIP kernels.  If
the library is not built this module raises on import; there is no fallback.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from ._abi import (C_SYMBOLS, LIB_PATH, MOE_BF16, MOE_BWD_DGRAD, MOE_BWD_WGRAD,  # noqa: F401
                   MOE_F32, MOE_MAX_DIM, MOE_MAX_E, MOE_MAX_K, MOE_OK,
                   MOE_PERMUTE_NOALLOC_MAX_BYTES, AdamWOptions, MoEError, Param)
from ._abi import load as _load

lib = _load()


def _check(status: int, fn: str):
    if status != MOE_OK:
        msg = lib.moe_last_error().decode()
        raise MoEError(f"{fn} -> {lib.moe_status_string(status).decode()}: {msg}")


def _ptr(t):
    return None if t is None else t.data_ptr()


# The host side of a call counts for small layers (a dozen calls a step): the
# raw stream handle comes without building a Stream object each time (2.5 us
# a call), and workspace sizes, pure functions of the call's sizes, are
# queried once per set of sizes.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream():
    # (callers hold device tensors: the runtime is up, and its own call is enough)
    return _raw_stream(torch._C._cuda_getDevice())


@functools.lru_cache(maxsize=512, typed=True)
def _ws_bytes(query: str, *sizes) -> int:
    n = ctypes.c_size_t()
    _check(getattr(lib, query)(*sizes, ctypes.byref(n)), query)
    return n.value


def _need(t, dtype, name, dim=None):
    if t is not None and t.dtype is dtype and t.is_cuda and t.is_contiguous() and (
            dim is None or t.dim() == dim):
        return t
    if t is None:
        raise ValueError(f"{name} is required")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name}: expected {dim} dims, got {t.dim()}")


def _given(t, dtype, name, shape):
    """A tensor argument of exactly this type and shape on the current device
    (kernels run on the current device's current stream)."""
    if (t is not None and t.dtype is dtype and t.is_cuda and t.shape == shape and
            t.is_contiguous() and t.get_device() == torch._C._cuda_getDevice()):
        return t
    _need(t, dtype, name, len(shape))
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} is on {t.device}, not on the current device")


def _out(t, dtype, name, shape, device):
    """An output: the caller's tensor, checked, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    return _given(t, dtype, name, shape)


_ws_cache: dict = {}
_ws_retired: list = []


def workspace(nbytes: int, device, tag: str) -> torch.Tensor:
    """A cached device scratch buffer of at least nbytes, one per (device,
    current stream, tag): calls on one stream are ordered, calls on different
    streams get different buffers.  A buffer replaced by a larger one is
    kept alive until the process ends, so a HIP graph captured with it never
    replays into freed memory (capture with the sizes it will replay).  A graph
    works in the buffers of the stream it was captured on: graphs captured on one
    stream (torch.cuda.graph's own, unless it is given another) replay one after
    the other; to replay two at once, capture each on a stream of its own.
    device: a torch.device, or what names one (text or number)."""
    if type(device) is torch.device and device.type == "cuda":
        index = device.index if device.index is not None else torch.cuda.current_device()
    else:
        index = torch.cuda.current_stream(device).device.index  # refuses what is no GPU
    key = (index, _raw_stream(index), tag)
    buf = _ws_cache.get(key)
    if buf is None or buf.numel() < nbytes:
        if buf is not None:
            _ws_retired.append(buf)
        buf = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=f"cuda:{index}")
        _ws_cache[key] = buf
    return buf


# ---------------------------------------------------------------- router
def moe_route(x, w_router, router_bias, k, renorm=0, logits=None, topk_idx=None, topk_gate=None):
    """Returns (topk_idx [T,k] int32, topk_gate [T,k] fp32)."""
    _need(x, torch.bfloat16, "x", 2)
    _need(w_router, torch.float32, "w_router", 2)
    if router_bias is not None:
        _need(router_bias, torch.float32, "router_bias", 1)
    T, d = x.shape
    E = w_router.shape[1]
    dev = x.device
    if topk_idx is None:
        topk_idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    if topk_gate is None:
        topk_gate = torch.empty((T, k), dtype=torch.float32, device=dev)
    ws, nws = None, 0
    if logits is None:
        ws = workspace(_ws_bytes("moe_route_workspace_bytes", T, E), dev, "route")
        nws = ws.numel()
    else:
        _need(logits, torch.float32, "logits", 2)
    _check(lib.moe_route(_ptr(x), _ptr(w_router), _ptr(router_bias), T, d, E, k, renorm,
                         _ptr(topk_idx), _ptr(topk_gate), _ptr(logits), _ptr(ws), nws, _stream()),
           "moe_route")
    return topk_idx, topk_gate


def moe_route_bwd(x, w_router, logits, topk_idx, topk_gate, dgate, renorm=0, dx=None,
                  dx_accumulate=True, with_dbias=False, dlogits=None, dw_router=None,
                  dlogits_aux=None):
    """Router gradient from the gate gradients, and from logit gradients of
    other losses of the router (dlogits_aux [T,E] fp32, optional).

    Returns (dw_router [d,E] fp32, dbias [E] fp32 or None, dx or None).  When
    dx is given it is updated in place (dx_accumulate) or overwritten with the
    router's share of the input gradient.
    """
    _need(x, torch.bfloat16, "x", 2)
    _need(w_router, torch.float32, "w_router", 2)
    _need(logits, torch.float32, "logits", 2)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    _need(topk_gate, torch.float32, "topk_gate", 2)
    _need(dgate, torch.float32, "dgate", 2)
    if dx is not None:
        _need(dx, torch.bfloat16, "dx", 2)
    if dlogits is not None:
        _need(dlogits, torch.float32, "dlogits", 2)
    T, d = x.shape
    E = w_router.shape[1]
    k = topk_idx.shape[1]
    dev = x.device
    if dw_router is None:
        dw_router = torch.empty((d, E), dtype=torch.float32, device=dev)
    else:
        _need(dw_router, torch.float32, "dw_router", 2)
    dbias = torch.empty((E,), dtype=torch.float32, device=dev) if with_dbias else None
    ws = workspace(_ws_bytes("moe_route_bwd_workspace_bytes", T, d, E), dev, "route_bwd")
    rest = (T, d, E, k, renorm, _ptr(dw_router), _ptr(dbias), _ptr(dx), 1 if dx_accumulate else 0,
            _ptr(dlogits), _ptr(ws), ws.numel(), _stream())
    if dlogits_aux is None:
        _check(lib.moe_route_bwd(_ptr(x), _ptr(w_router), _ptr(logits), _ptr(topk_idx),
                                 _ptr(topk_gate), _ptr(dgate), *rest), "moe_route_bwd")
    else:
        _given(dlogits_aux, torch.float32, "dlogits_aux", (T, E))
        _check(lib.moe_route_bwd_aux(_ptr(x), _ptr(w_router), _ptr(logits), _ptr(topk_idx),
                                     _ptr(topk_gate), _ptr(dgate), _ptr(dlogits_aux), *rest),
               "moe_route_bwd_aux")
    return dw_router, dbias, dx


# ---------------------------------------------------------- balance loss
def _groups(logits, seq_offsets, token_mask):
    """(T, E, G) of a balance loss call, its arguments checked."""
    _need(logits, torch.float32, "logits", 2)
    T, E = _given(logits, torch.float32, "logits", logits.shape).shape
    G = 1
    if seq_offsets is not None:
        _need(seq_offsets, torch.int32, "seq_offsets", 1)
        G = seq_offsets.shape[0] - 1
        if G < 1:
            raise ValueError("seq_offsets needs two entries or more")
        _given(seq_offsets, torch.int32, "seq_offsets", (G + 1,))
    if token_mask is not None:
        if token_mask.dtype not in (torch.bool, torch.uint8):
            raise TypeError(f"token_mask: expected torch.bool or torch.uint8, got {token_mask.dtype}")
        _given(token_mask, token_mask.dtype, "token_mask", (T,))
    return T, E, G


def moe_balance_loss_fwd(logits, topk_idx, seq_offsets=None, token_mask=None):
    """Balance loss and z-loss of the router, per group of consecutive tokens
    (seq_offsets [G+1] int32; None: one group).  logits [T,E] fp32, topk_idx
    [T,k] int32, token_mask [T] bool or uint8 (0: padding).  Returns (balance
    [G], zloss [G], counts [G,E] int32, prob_sum [G,E], n_tokens [G] int32)."""
    T, E, G = _groups(logits, seq_offsets, token_mask)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    k = topk_idx.shape[1]
    _given(topk_idx, torch.int32, "topk_idx", (T, k))
    dev = logits.device
    balance = torch.empty((G,), dtype=torch.float32, device=dev)
    zloss = torch.empty((G,), dtype=torch.float32, device=dev)
    counts = torch.empty((G, E), dtype=torch.int32, device=dev)
    prob_sum = torch.empty((G, E), dtype=torch.float32, device=dev)
    n_tokens = torch.empty((G,), dtype=torch.int32, device=dev)
    ws = workspace(_ws_bytes("moe_balance_loss_workspace_bytes", T, E, G), dev, "balance_loss")
    _check(lib.moe_balance_loss_fwd(_ptr(logits), _ptr(topk_idx), _ptr(seq_offsets),
                                    _ptr(token_mask), T, E, k, G, _ptr(balance), _ptr(zloss),
                                    _ptr(counts), _ptr(prob_sum), _ptr(n_tokens), _ptr(ws),
                                    ws.numel(), _stream()), "moe_balance_loss_fwd")
    return balance, zloss, counts, prob_sum, n_tokens


def moe_balance_loss_bwd(logits, counts, n_tokens, dbalance, dzloss, k, seq_offsets=None,
                         token_mask=None, dlogits=None, accumulate=False):
    """Gradient of the router's logits from dbalance, dzloss [G] fp32, with the
    forward's counts and n_tokens (k: slots per token).  Returns dlogits [T,E]
    fp32, overwritten, or added to where `accumulate`."""
    T, E, G = _groups(logits, seq_offsets, token_mask)
    _given(counts, torch.int32, "counts", (G, E))
    _given(n_tokens, torch.int32, "n_tokens", (G,))
    _given(dbalance, torch.float32, "dbalance", (G,))
    _given(dzloss, torch.float32, "dzloss", (G,))
    if accumulate and dlogits is None:
        raise ValueError("accumulate needs dlogits")
    dlogits = _out(dlogits, torch.float32, "dlogits", (T, E), logits.device)
    _check(lib.moe_balance_loss_bwd(_ptr(logits), _ptr(counts), _ptr(n_tokens), _ptr(dbalance),
                                    _ptr(dzloss), _ptr(seq_offsets), _ptr(token_mask), T, E, k, G,
                                    _ptr(dlogits), 1 if accumulate else 0, _stream()),
           "moe_balance_loss_bwd")
    return dlogits


# ------------------------------------------------------------ permutation
def moe_permute(x, topk_idx, E, expert_begin=0, num_local=None, cap=None, counts_global=True):
    """Returns dict(expert_offsets, counts_global, row_src, dst, x_perm)."""
    _need(x, torch.bfloat16, "x", 2)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    T, d = x.shape
    k = topk_idx.shape[1]
    num_local = E if num_local is None else num_local
    cap = T * min(k, num_local) if cap is None else cap
    dev = x.device
    offsets = torch.empty(num_local + 1, dtype=torch.int32, device=dev)
    cg = torch.empty(E, dtype=torch.int32, device=dev) if counts_global else None
    row_src = torch.empty(max(cap, 1), dtype=torch.int32, device=dev)
    dst = torch.empty(max(T * k, 1), dtype=torch.int32, device=dev)
    x_perm = torch.empty((max(cap, 1), d), dtype=torch.bfloat16, device=dev)
    ws = workspace(_ws_bytes("moe_permute_workspace_bytes", T, E, k, num_local), dev, "permute")
    _check(lib.moe_permute(_ptr(x), _ptr(topk_idx), T, d, E, k, expert_begin, num_local,
                           _ptr(offsets), _ptr(cg), _ptr(row_src), _ptr(dst), _ptr(x_perm),
                           _ptr(ws), ws.numel(), _stream()), "moe_permute")
    return {"expert_offsets": offsets, "counts_global": cg, "row_src": row_src,
            "dst": dst[: T * k].view(T, k), "x_perm": x_perm, "cap": cap}


def moe_permute_noalloc(x, topk_idx, E, expert_begin=0, num_local=None, out=None,
                        counts_global=True):
    """moe_permute on the library's static scratch (no workspace).  `out`:
    optional dict of preallocated outputs as moe_permute returns them
    (expert_offsets, counts_global, row_src, dst, x_perm); otherwise they
    are allocated here.  Returns that dict."""
    _need(x, torch.bfloat16, "x", 2)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    T, d = x.shape
    k = topk_idx.shape[1]
    num_local = E if num_local is None else num_local
    dev = x.device
    if out is None:
        cap = T * min(k, num_local)
        out = {"expert_offsets": torch.empty(num_local + 1, dtype=torch.int32, device=dev),
               "counts_global": torch.empty(E, dtype=torch.int32, device=dev)
               if counts_global else None,
               "row_src": torch.empty(max(cap, 1), dtype=torch.int32, device=dev),
               "dst": torch.empty(max(T * k, 1), dtype=torch.int32, device=dev),
               "x_perm": torch.empty((max(cap, 1), d), dtype=torch.bfloat16, device=dev),
               "cap": cap}
    _check(lib.moe_permute_noalloc(_ptr(x), _ptr(topk_idx), T, d, E, k, expert_begin, num_local,
                                   _ptr(out["expert_offsets"]), _ptr(out.get("counts_global")),
                                   _ptr(out["row_src"]), _ptr(out["dst"]), _ptr(out["x_perm"]),
                                   _stream()), "moe_permute_noalloc")
    return out


# ----------------------------------------------------- grouped SwiGLU FFN
def moe_grouped_swiglu_fwd(x_perm, expert_offsets, w_gate, w_up, w_down, cap=None,
                           h_gate=None, h_up=None, y_perm=None):
    """Returns (h_gate, h_up, y_perm), each with cap rows."""
    _need(x_perm, torch.bfloat16, "x_perm", 2)
    _need(expert_offsets, torch.int32, "expert_offsets", 1)
    for n_, t in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _need(t, torch.bfloat16, n_, 3)
    E_loc, d, f = w_gate.shape
    cap = x_perm.shape[0] if cap is None else cap
    dev = x_perm.device
    if h_gate is None:
        h_gate = torch.empty((max(cap, 1), f), dtype=torch.bfloat16, device=dev)
    if h_up is None:
        h_up = torch.empty((max(cap, 1), f), dtype=torch.bfloat16, device=dev)
    if y_perm is None:
        y_perm = torch.empty((max(cap, 1), d), dtype=torch.bfloat16, device=dev)
    ws = workspace(_ws_bytes("moe_grouped_swiglu_workspace_bytes", cap, E_loc, d, f, 0), dev, "ffn")
    _check(lib.moe_grouped_swiglu_fwd(_ptr(x_perm), _ptr(expert_offsets), E_loc, cap, d, f,
                                      _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(h_gate),
                                      _ptr(h_up), _ptr(y_perm), _ptr(ws), ws.numel(), _stream()),
           "moe_grouped_swiglu_fwd")
    return h_gate, h_up, y_perm


def moe_grouped_swiglu_bwd(dy_perm, x_perm, h_gate, h_up, expert_offsets, w_gate, w_up, w_down,
                           flags=MOE_BWD_DGRAD | MOE_BWD_WGRAD, cap=None, dx_perm=None,
                           dw_gate=None, dw_up=None, dw_down=None):
    """Returns (dx_perm or None, dw_gate, dw_up, dw_down or None)."""
    for n_, t in (("dy_perm", dy_perm), ("x_perm", x_perm), ("h_gate", h_gate), ("h_up", h_up)):
        _need(t, torch.bfloat16, n_, 2)
    _need(expert_offsets, torch.int32, "expert_offsets", 1)
    for n_, t in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _need(t, torch.bfloat16, n_, 3)
    E_loc, d, f = w_gate.shape
    cap = x_perm.shape[0] if cap is None else cap
    dev = x_perm.device
    if flags & MOE_BWD_DGRAD and dx_perm is None:
        dx_perm = torch.empty((max(cap, 1), d), dtype=torch.bfloat16, device=dev)
    if flags & MOE_BWD_WGRAD:
        if dw_gate is None:
            dw_gate = torch.empty_like(w_gate)
        if dw_up is None:
            dw_up = torch.empty_like(w_up)
        if dw_down is None:
            dw_down = torch.empty_like(w_down)
    ws = workspace(_ws_bytes("moe_grouped_swiglu_workspace_bytes", cap, E_loc, d, f, flags), dev,
                   "ffn")
    _check(lib.moe_grouped_swiglu_bwd(_ptr(dy_perm), _ptr(x_perm), _ptr(h_gate), _ptr(h_up),
                                      _ptr(expert_offsets), E_loc, cap, d, f, _ptr(w_gate),
                                      _ptr(w_up), _ptr(w_down), _ptr(dx_perm), _ptr(dw_gate),
                                      _ptr(dw_up), _ptr(dw_down), flags, _ptr(ws), ws.numel(),
                                      _stream()),
           "moe_grouped_swiglu_bwd")
    return (dx_perm if flags & MOE_BWD_DGRAD else None,
            dw_gate if flags & MOE_BWD_WGRAD else None,
            dw_up if flags & MOE_BWD_WGRAD else None,
            dw_down if flags & MOE_BWD_WGRAD else None)


# ----------------------------------------------------------------- combine
def moe_combine(y_perm, dst, topk_gate, out=None):
    """out[t] = sum_i gate[t,i] * y_perm[dst[t,i]] (gate None -> weight 1)."""
    _need(y_perm, torch.bfloat16, "y_perm", 2)
    _need(dst, torch.int32, "dst", 2)
    if topk_gate is not None:
        _need(topk_gate, torch.float32, "topk_gate", 2)
    T, k = dst.shape
    d = y_perm.shape[1]
    if out is None:
        out = torch.empty((T, d), dtype=torch.bfloat16, device=y_perm.device)
    _check(lib.moe_combine(_ptr(y_perm), _ptr(dst), _ptr(topk_gate), T, d, k, _ptr(out),
                           _stream()), "moe_combine")
    return out


def moe_combine_bwd(dout, y_perm, dst, topk_gate, dy_perm=None, dgate=None, with_dgate=True):
    """Returns (dy_perm [cap,d], dgate [T,k] or None)."""
    _need(dout, torch.bfloat16, "dout", 2)
    _need(y_perm, torch.bfloat16, "y_perm", 2)
    _need(dst, torch.int32, "dst", 2)
    if topk_gate is not None:
        _need(topk_gate, torch.float32, "topk_gate", 2)
    T, k = dst.shape
    d = dout.shape[1]
    if dy_perm is None:
        dy_perm = torch.empty_like(y_perm)
    if dgate is None and with_dgate:
        dgate = torch.empty((T, k), dtype=torch.float32, device=dout.device)
    _check(lib.moe_combine_bwd(_ptr(dout), _ptr(y_perm), _ptr(dst), _ptr(topk_gate), T, d, k,
                               _ptr(dy_perm), _ptr(dgate), _stream()), "moe_combine_bwd")
    return dy_perm, dgate


def moe_ffn_fwd_chunked(x, topk_idx, topk_gate, E, w_gate, w_up, w_down, chunk, expert_begin=0,
                        num_local=None, out=None, stream2=None):
    """Memory-efficient forward over token chunks on the current stream and
    `stream2` (a torch.cuda.Stream or None = the current stream).  Returns y."""
    _need(x, torch.bfloat16, "x", 2)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    _need(topk_gate, torch.float32, "topk_gate", 2)
    for n, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _need(w, torch.bfloat16, n, 3)
    T, d = x.shape
    k = topk_idx.shape[1]
    num_local = w_gate.shape[0] if num_local is None else num_local
    f = w_gate.shape[2]
    if out is None:
        out = torch.empty((T, d), dtype=torch.bfloat16, device=x.device)
    ws = workspace(_ws_bytes("moe_ffn_fwd_chunked_workspace_bytes", chunk, E, k, num_local, d, f),
                   x.device, "ffn_fwd_chunked")
    s2 = _stream() if stream2 is None else ctypes.c_void_p(stream2.cuda_stream)
    _check(lib.moe_ffn_fwd_chunked(_ptr(x), _ptr(topk_idx), _ptr(topk_gate), T, d, E, k,
                                   expert_begin, num_local, f, _ptr(w_gate), _ptr(w_up),
                                   _ptr(w_down), chunk, _ptr(out), _ptr(ws), ws.numel(), _stream(),
                                   s2), "moe_ffn_fwd_chunked")
    return out


def moe_ffn_fwd_row_chunked(x, topk_idx, topk_gate, E, w_gate, w_up, w_down, chunk_rows,
                            expert_begin=0, num_local=None, out=None, stream2=None):
    """Memory-efficient forward over chunks of consecutive permuted rows
    (expert ranges) on the current stream and `stream2` (a torch.cuda.Stream
    or None = the current stream).  Returns y."""
    _need(x, torch.bfloat16, "x", 2)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    _need(topk_gate, torch.float32, "topk_gate", 2)
    for n, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _need(w, torch.bfloat16, n, 3)
    T, d = x.shape
    k = topk_idx.shape[1]
    num_local = w_gate.shape[0] if num_local is None else num_local
    f = w_gate.shape[2]
    if out is None:
        out = torch.empty((T, d), dtype=torch.bfloat16, device=x.device)
    ws = workspace(_ws_bytes("moe_ffn_fwd_row_chunked_workspace_bytes", T, E, k, num_local, d, f,
                             chunk_rows), x.device, "ffn_fwd_row_chunked")
    s2 = _stream() if stream2 is None else ctypes.c_void_p(stream2.cuda_stream)
    _check(lib.moe_ffn_fwd_row_chunked(_ptr(x), _ptr(topk_idx), _ptr(topk_gate), T, d, E, k,
                                       expert_begin, num_local, f, _ptr(w_gate), _ptr(w_up),
                                       _ptr(w_down), chunk_rows, _ptr(out), _ptr(ws), ws.numel(),
                                       _stream(), s2), "moe_ffn_fwd_row_chunked")
    return out


# ---------------------------------------------------------------- MXFP4
def _mx_shapes(B, rows, K):
    """Shapes of the values and scales of B MXFP4 matrices of `rows` rows along K."""
    return (B, rows, 16 * (-(-K // 32))), (B, -(-K // 256), rows, 8)


def moe_mxfp4_quantize(src, transpose=False):
    """MXFP4 of src [R,C] or [B,R,C] bf16: matrices of R rows along C, or, with
    transpose, of C rows along R.  Returns (q, s) uint8: q [..., rows,
    16 ceil(K/32)], s [..., ceil(K/256), rows, 8]."""
    _need(src, torch.bfloat16, "src")
    if src.dim() not in (2, 3):
        raise ValueError(f"src: expected 2 or 3 dims, got {src.dim()}")
    _given(src, torch.bfloat16, "src", src.shape)
    B = src.shape[0] if src.dim() == 3 else 1
    R, C = src.shape[-2:]
    qs, ss = _mx_shapes(B, *((C, R) if transpose else (R, C)))
    if src.dim() == 2:
        qs, ss = qs[1:], ss[1:]
    q = torch.empty(qs, dtype=torch.uint8, device=src.device)
    s = torch.empty(ss, dtype=torch.uint8, device=src.device)
    _check(lib.moe_mxfp4_quantize(_ptr(src), B, R, C, 1 if transpose else 0, _ptr(q), _ptr(s),
                                  _stream()), "moe_mxfp4_quantize")
    return q, s


def moe_mxfp4_dequantize(q, s, K, out=None):
    """The values that MXFP4 matrices along K stand for: [..., rows, K] bf16."""
    _need(q, torch.uint8, "q")
    if q.dim() not in (2, 3):
        raise ValueError(f"q: expected 2 or 3 dims, got {q.dim()}")
    B = q.shape[0] if q.dim() == 3 else 1
    rows = q.shape[-2]
    qs, ss = _mx_shapes(B, rows, K)
    if q.dim() == 2:
        qs, ss = qs[1:], ss[1:]
    _given(q, torch.uint8, "q", qs)
    _given(s, torch.uint8, "s", ss)
    out = _out(out, torch.bfloat16, "out", (*q.shape[:-1], K), q.device)
    _check(lib.moe_mxfp4_dequantize(_ptr(q), _ptr(s), B, rows, K, _ptr(out), _stream()),
           "moe_mxfp4_dequantize")
    return out


def _mx_weights(w_gate, w_up, w_down, d):
    """(num_local, f, six pointers) of MXFP4 expert weights, each a (q, s) pair."""
    for name, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        if not isinstance(w, (tuple, list)) or len(w) != 2:
            raise TypeError(f"{name}: expected the (q, s) pair of moe_mxfp4_quantize")
    _need(w_gate[0], torch.uint8, "w_gate q", 3)
    num_local, f = w_gate[0].shape[:2]
    ptrs = []
    for name, w, rows, K in (("w_gate", w_gate, f, d), ("w_up", w_up, f, d),
                             ("w_down", w_down, d, f)):
        qs, ss = _mx_shapes(num_local, rows, K)
        ptrs += [_ptr(_given(w[0], torch.uint8, f"{name} q", qs)),
                 _ptr(_given(w[1], torch.uint8, f"{name} s", ss))]
    return num_local, f, ptrs


def moe_grouped_swiglu_fwd_mxfp4(x, expert_offsets, w_gate, w_up, w_down, d, row_src=None, k=1,
                                 cap=None, y_perm=None):
    """Grouped SwiGLU on MXFP4 operands, each a (q, s) pair: x of moe_mxfp4_
    quantize(x [rows,d]), w_gate and w_up of the transposed [E_loc,d,f], w_down
    of the transposed [E_loc,f,d].  row_src [cap] int32 (moe_permute's): row p
    is x row row_src[p] // k; None: row p.  Returns y_perm [cap,d] bf16."""
    if not isinstance(x, (tuple, list)) or len(x) != 2:
        raise TypeError("x: expected the (q, s) pair of moe_mxfp4_quantize")
    _need(x[0], torch.uint8, "x q", 2)
    x_rows = x[0].shape[0]
    qs, ss = _mx_shapes(1, x_rows, d)
    _given(x[0], torch.uint8, "x q", qs[1:])
    _given(x[1], torch.uint8, "x s", ss[1:])
    num_local, f, wp = _mx_weights(w_gate, w_up, w_down, d)
    _given(expert_offsets, torch.int32, "expert_offsets", (num_local + 1,))
    if row_src is not None:
        _need(row_src, torch.int32, "row_src", 1)
        cap = row_src.shape[0] if cap is None else cap
        _given(row_src, torch.int32, "row_src", (max(cap, 1),))
    cap = x_rows if cap is None else cap
    y_perm = _out(y_perm, torch.bfloat16, "y_perm", (max(cap, 1), d), x[0].device)
    ws = workspace(_ws_bytes("moe_grouped_swiglu_mxfp4_workspace_bytes", cap, num_local, d, f),
                   x[0].device, "ffn_mxfp4")
    _check(lib.moe_grouped_swiglu_fwd_mxfp4(_ptr(x[0]), _ptr(x[1]), x_rows, _ptr(row_src), k,
                                            _ptr(expert_offsets), num_local, cap, d, f, *wp,
                                            _ptr(y_perm), _ptr(ws), ws.numel(), _stream()),
           "moe_grouped_swiglu_fwd_mxfp4")
    return y_perm


def moe_ffn_fwd_mxfp4(x, topk_idx, topk_gate, E, w_gate, w_up, w_down, expert_begin=0, out=None):
    """The expert layer's forward on MXFP4 weights (see moe_grouped_swiglu_fwd_
    mxfp4) of experts [expert_begin, + num_local).  x [T,d] bf16, topk_idx [T,k]
    int32, topk_gate [T,k] fp32.  Returns y [T,d] bf16."""
    _need(x, torch.bfloat16, "x", 2)
    T, d = x.shape
    _given(x, torch.bfloat16, "x", (T, d))
    _need(topk_idx, torch.int32, "topk_idx", 2)
    k = topk_idx.shape[1]
    _given(topk_idx, torch.int32, "topk_idx", (T, k))
    _given(topk_gate, torch.float32, "topk_gate", (T, k))
    num_local, f, wp = _mx_weights(w_gate, w_up, w_down, d)
    out = _out(out, torch.bfloat16, "out", (T, d), x.device)
    ws = workspace(_ws_bytes("moe_ffn_fwd_mxfp4_workspace_bytes", T, E, k, num_local, d, f),
                   x.device, "ffn_fwd_mxfp4")
    _check(lib.moe_ffn_fwd_mxfp4(_ptr(x), _ptr(topk_idx), _ptr(topk_gate), T, d, E, k,
                                 expert_begin, num_local, f, *wp, _ptr(out), _ptr(ws), ws.numel(),
                                 _stream()), "moe_ffn_fwd_mxfp4")
    return out


# ------------------------------------------------------- vocabulary loss
def _vocab_ws(N, H, V, vblock, device):
    return workspace(_ws_bytes("moe_vocab_loss_workspace_bytes", N, H, V, vblock), device,
                     "vocab_loss")


def moe_vocab_loss_fwd(x, w_voc, target, vblock, loss=None, lse=None):
    """Blockwise online loss of the vocabulary projection.  x [N,H] bf16,
    w_voc [H,V] bf16, target [N] int32.  Returns (loss [N], lse [N]) fp32."""
    _need(x, torch.bfloat16, "x", 2)
    _need(w_voc, torch.bfloat16, "w_voc", 2)
    _need(target, torch.int32, "target", 1)
    N, H = x.shape
    V = w_voc.shape[1]
    if loss is None:
        loss = torch.empty((N,), dtype=torch.float32, device=x.device)
    if lse is None:
        lse = torch.empty((N,), dtype=torch.float32, device=x.device)
    ws = _vocab_ws(N, H, V, vblock, x.device)
    _check(lib.moe_vocab_loss_fwd(_ptr(x), _ptr(w_voc), _ptr(target), N, H, V, vblock,
                                  _ptr(loss), _ptr(lse), _ptr(ws), ws.numel(), _stream()),
           "moe_vocab_loss_fwd")
    return loss, lse


def moe_vocab_loss_bwd(x, w_voc, target, lse, dloss, vblock, dx=None, dw_voc=None):
    """Gradients of the vocabulary loss given dloss [N] fp32.  Returns
    (dx [N,H] bf16, dw_voc [H,V] bf16)."""
    _need(x, torch.bfloat16, "x", 2)
    _need(w_voc, torch.bfloat16, "w_voc", 2)
    _need(target, torch.int32, "target", 1)
    _need(lse, torch.float32, "lse", 1)
    _need(dloss, torch.float32, "dloss", 1)
    N, H = x.shape
    V = w_voc.shape[1]
    if dx is None:
        dx = torch.empty((N, H), dtype=torch.bfloat16, device=x.device)
    if dw_voc is None:
        dw_voc = torch.empty((H, V), dtype=torch.bfloat16, device=x.device)
    ws = _vocab_ws(N, H, V, vblock, x.device)
    _check(lib.moe_vocab_loss_bwd(_ptr(x), _ptr(w_voc), _ptr(target), _ptr(lse), _ptr(dloss), N,
                                  H, V, vblock, _ptr(dx), _ptr(dw_voc), _ptr(ws), ws.numel(),
                                  _stream()), "moe_vocab_loss_bwd")
    return dx, dw_voc


# ---------------------------------------------------------- distillation
def _teacher(x, w_voc, topk_idx, topk_logit, vblock, teacher_lse):
    """(N, H, V, K, workspace) of a distillation call, its arguments checked."""
    _need(x, torch.bfloat16, "x", 2)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    _need(w_voc, torch.bfloat16, "w_voc", 2)
    N, H = x.shape
    V = w_voc.shape[1]
    K = topk_idx.shape[1]
    _given(x, torch.bfloat16, "x", (N, H))
    _given(w_voc, torch.bfloat16, "w_voc", (H, V))
    _given(topk_idx, torch.int32, "topk_idx", (N, K))
    _given(topk_logit, torch.float32, "topk_logit", (N, K))
    if teacher_lse is not None:
        _given(teacher_lse, torch.float32, "teacher_lse", (N,))
    ws = workspace(_ws_bytes("moe_vocab_distill_workspace_bytes", N, H, V, vblock, K), x.device,
                   "vocab_distill")
    return N, H, V, K, ws


def moe_vocab_distill_fwd(x, w_voc, topk_idx, topk_logit, vblock, temperature=1.0,
                          teacher_lse=None, loss=None, lse=None, y_topk=None):
    """Loss of the vocabulary projection against a teacher's top logits.  x
    [N,H] bf16, w_voc [H,V] bf16, topk_idx [N,K] int32 (outside [0, V): no
    slot), topk_logit [N,K] fp32, teacher_lse [N] fp32 (None: the slots'
    probabilities sum to one).  Returns (loss [N], lse [N], y_topk [N,K]) fp32."""
    N, H, V, K, ws = _teacher(x, w_voc, topk_idx, topk_logit, vblock, teacher_lse)
    loss = _out(loss, torch.float32, "loss", (N,), x.device)
    lse = _out(lse, torch.float32, "lse", (N,), x.device)
    y_topk = _out(y_topk, torch.float32, "y_topk", (N, K), x.device)
    _check(lib.moe_vocab_distill_fwd(_ptr(x), _ptr(w_voc), _ptr(topk_idx), _ptr(topk_logit),
                                     _ptr(teacher_lse), temperature, N, H, V, vblock, K,
                                     _ptr(loss), _ptr(lse), _ptr(y_topk), _ptr(ws), ws.numel(),
                                     _stream()), "moe_vocab_distill_fwd")
    return loss, lse, y_topk


def moe_vocab_distill_bwd(x, w_voc, topk_idx, topk_logit, lse, y_topk, dloss, vblock,
                          temperature=1.0, teacher_lse=None, dx=None, dw_voc=None):
    """Gradients of the distillation loss given dloss [N] fp32 and the
    forward's lse and y_topk.  Returns (dx [N,H] bf16, dw_voc [H,V] bf16)."""
    N, H, V, K, ws = _teacher(x, w_voc, topk_idx, topk_logit, vblock, teacher_lse)
    _given(lse, torch.float32, "lse", (N,))
    _given(y_topk, torch.float32, "y_topk", (N, K))
    _given(dloss, torch.float32, "dloss", (N,))
    dx = _out(dx, torch.bfloat16, "dx", (N, H), x.device)
    dw_voc = _out(dw_voc, torch.bfloat16, "dw_voc", (H, V), x.device)
    _check(lib.moe_vocab_distill_bwd(_ptr(x), _ptr(w_voc), _ptr(topk_idx), _ptr(topk_logit),
                                     _ptr(teacher_lse), temperature, _ptr(lse), _ptr(y_topk),
                                     _ptr(dloss), N, H, V, vblock, K, _ptr(dx), _ptr(dw_voc),
                                     _ptr(ws), ws.numel(), _stream()), "moe_vocab_distill_bwd")
    return dx, dw_voc


# --------------------------------------------------------------- embedding
def _shape(t, dtype, name, dim):
    """The shape of a tensor argument of this type and rank on the current device."""
    if (t is not None and t.dtype is dtype and t.is_cuda and t.dim() == dim and
            t.is_contiguous() and t.get_device() == torch._C._cuda_getDevice()):
        return t.shape
    _need(t, dtype, name, dim)
    return _given(t, dtype, name, t.shape).shape


def _like(t, like, name):
    """An output of the shape and type of `like`: the caller's, checked, or new."""
    if t is None:
        return torch.empty_like(like)
    return _given(t, like.dtype, name, like.shape)


def moe_embedding_fwd(ids, w, scale=1.0, vocab_begin=0, y=None):
    """Rows of w [rows,H] bf16 (vocabulary entries [vocab_begin, vocab_begin +
    rows)) for ids [N] int32, times scale; zeros for ids outside them (another
    rank's, or -1 for padding).  Returns y [N,H] bf16."""
    rows, H = _shape(w, torch.bfloat16, "w", 2)
    N, = _shape(ids, torch.int32, "ids", 1)
    y = w.new_empty((N, H)) if y is None else _given(y, torch.bfloat16, "y", (N, H))
    _check(lib.moe_embedding_fwd(ids.data_ptr(), w.data_ptr(), N, H, vocab_begin, rows, scale,
                                 y.data_ptr(), _stream()), "moe_embedding_fwd")
    return y


def moe_embedding_bwd(ids, dy, rows, scale=1.0, vocab_begin=0, dw=None):
    """Gradient of the embedding's weights from dy [N,H] bf16: dw [rows,H] bf16,
    every row written (zeros where no token named it)."""
    N, H = _shape(dy, torch.bfloat16, "dy", 2)
    _given(ids, torch.int32, "ids", (N,))
    ws = workspace(_ws_bytes("moe_embedding_bwd_workspace_bytes", N, H, rows), dy.device,
                   "embedding_bwd")
    dw = dy.new_empty((rows, H)) if dw is None else _given(dw, torch.bfloat16, "dw", (rows, H))
    _check(lib.moe_embedding_bwd(ids.data_ptr(), dy.data_ptr(), N, H, vocab_begin, rows, scale,
                                 dw.data_ptr(), ws.data_ptr(), ws.numel(), _stream()),
           "moe_embedding_bwd")
    return dw


# -------------------------------------------------------------- layer norm
def moe_layer_norm_fwd(x, gamma, beta=None, eps=1e-5, residual=None, y=None, h=None, stats=True):
    """Layer norm of h = x + residual (rounded to bf16; h is x without a
    residual), rows [T,d] bf16, gamma and beta [d] fp32.  Returns (y, h, mean
    [T], rstd [T]); stats=False: None in the place of the last two."""
    T, d = shape = _shape(x, torch.bfloat16, "x", 2)
    _given(gamma, torch.float32, "gamma", (d,))
    if beta is not None:
        _given(beta, torch.float32, "beta", (d,))
    if residual is not None:
        _given(residual, torch.bfloat16, "residual", shape)
        h = _like(h, x, "h")
    elif h is not None:
        raise ValueError("h is an output of a residual sum: without residual it is x")
    y = _like(y, x, "y")
    mean = rstd = None
    if stats:
        mean, rstd = gamma.new_empty((T,)), gamma.new_empty((T,))
    _check(lib.moe_layer_norm_fwd(x.data_ptr(), _ptr(residual), gamma.data_ptr(), _ptr(beta), T, d,
                                  eps, _ptr(h), y.data_ptr(), _ptr(mean), _ptr(rstd), _stream()),
           "moe_layer_norm_fwd")
    return y, x if residual is None else h, mean, rstd


def moe_layer_norm_bwd(dy, h, gamma, mean, rstd, dh=None, dx=None, with_dbeta=True):
    """Gradients of the layer norm from dy [T,d] and the forward's h, mean and
    rstd; dh [T,d]: the gradient that reaches h by another way (the residual
    stream's), added to dx.  Returns (dx [T,d] bf16, dgamma [d], dbeta [d] or
    None, fp32); dx is the gradient of x and of the residual alike, and may be dy, h
    or dh itself."""
    T, d = shape = _shape(h, torch.bfloat16, "h", 2)
    _given(dy, torch.bfloat16, "dy", shape)
    _given(gamma, torch.float32, "gamma", (d,))
    _given(mean, torch.float32, "mean", (T,))
    _given(rstd, torch.float32, "rstd", (T,))
    if dh is not None:
        _given(dh, torch.bfloat16, "dh", shape)
    ws = workspace(_ws_bytes("moe_layer_norm_bwd_workspace_bytes", T, d), h.device, "layer_norm_bwd")
    dx = _like(dx, h, "dx")
    dgamma = torch.empty_like(gamma)
    dbeta = torch.empty_like(gamma) if with_dbeta else None
    _check(lib.moe_layer_norm_bwd(dy.data_ptr(), h.data_ptr(), gamma.data_ptr(), mean.data_ptr(),
                                  rstd.data_ptr(), _ptr(dh), T, d, dx.data_ptr(),
                                  dgamma.data_ptr(), _ptr(dbeta), ws.data_ptr(), ws.numel(),
                                  _stream()), "moe_layer_norm_bwd")
    return dx, dgamma, dbeta


# ---------------------------------------------------------- weight updates
_TYPES = {torch.float32: MOE_F32, torch.bfloat16: MOE_BF16}
STATE_BLOCK = 128  # elements of one scale of an 8-bit state


def _same_order(a, b):
    """Whether two shapes of as many elements name them in one order: the places where
    the axes of one end are among those of the other (neighbouring axes are taken
    together, all of them in a flat tensor; axes of 1 aside)."""
    if a == b or 0 in a:
        return True
    ends = []
    for shape in (a, b):
        n, at = 1, set()
        for size in shape:
            n *= size
            at.add(n)
        ends.append(at - {1, n})
    return ends[0] <= ends[1] or ends[1] <= ends[0]


class Params:
    """The tensors of a weight update, checked once and kept: weights w (fp32 or
    bf16), gradients g (fp32 or bf16), states m and v, and optionally bf16 copies
    of fp32 weights that each step writes (w_copy; None where a weight has none).
    Lists of the same length; tensors of any shape, contiguous, those of one weight in
    its order of elements: its shape, or one with neighbouring axes taken together, as
    in a flat one ([n], or [E d, f] for [E, d, f]; a transposed gradient is refused).
    A state is an fp32 tensor, or in 8 bits a pair (codes [n] uint8, scales
    [ceil(n / 128)] uint8); without m and v they start as zeros, in `bits` bits.
    w=None: gradients alone, for moe_grad_sumsq.  The tensors stay alive as long as
    this does, and gradients are read from where they are at every step
    (`set_grads` names others)."""

    def __init__(self, w, g, m=None, v=None, w_copy=None, bits=None):
        self.g = list(g)
        self.count = count = len(self.g)
        self.device = self.torch_device = None
        self.array = (Param * max(count, 1))()
        self.w = None if w is None else list(w)
        self.w_copy = [None] * count if w_copy is None else list(w_copy)
        self.m, self.v, self.bits = m, v, bits
        sized, name = (self.g, "g") if w is None else (self.w, "w")
        for i, t in enumerate(sized):
            if not isinstance(t, torch.Tensor):
                raise ValueError(f"{name}[{i}] is required")
        sizes = [t.numel() for t in sized]
        # the sum of squares of gradients alone goes by no order
        self.shapes = [None if w is None else tuple(t.shape) for t in sized]
        spans = []
        if w is None:
            if m is not None or v is not None or w_copy is not None or bits is not None:
                raise ValueError("states and copies need weights")
        else:
            if len(self.w) != count or len(self.w_copy) != count:
                raise ValueError("w, g and w_copy need one entry for each tensor")
            if (m is None) != (v is None):
                raise ValueError("m and v come together")
            if m is None:
                self._new_states(sizes, 32 if bits is None else bits)
            else:
                self._given_states(m, v, bits)
            for i, (p, n, like) in enumerate(zip(self.array, sizes, self.shapes)):
                p.w, p.w_type = self._take(self.w[i], tuple(_TYPES), f"w[{i}]", n, spans)
                if self.w_copy[i] is not None:
                    if p.w_type != MOE_F32:
                        raise TypeError(f"w_copy[{i}]: only fp32 weights have a copy")
                    p.w_copy, _ = self._take(self.w_copy[i], (torch.bfloat16,), f"w_copy[{i}]", n,
                                             spans, like)
                for name, state in (("m", self.m[i]), ("v", self.v[i])):
                    at = f"{name}[{i}]"
                    if self.bits == 32:
                        a, _ = self._take(state, (torch.float32,), at, n, spans, like)
                    else:
                        codes, scales = state
                        a, _ = self._take(codes, (torch.uint8,), at, n, spans, like)
                        b, _ = self._take(scales, (torch.uint8,), at + " scales",
                                          -(-n // STATE_BLOCK), spans)
                        setattr(p, name + "_scale", b)
                    setattr(p, name, a)
        self.sizes = sizes
        self._written = spans
        self.set_grads(self.g)

    def _new_states(self, sizes, bits):
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        self.bits = bits

        def zeros(i, n):
            dev = self.w[i].device
            if bits == 32:
                return torch.zeros((n,), dtype=torch.float32, device=dev)
            return (torch.zeros((n,), dtype=torch.uint8, device=dev),
                    torch.zeros((-(-n // STATE_BLOCK),), dtype=torch.uint8, device=dev))
        self.m = [zeros(i, n) for i, n in enumerate(sizes)]
        self.v = [zeros(i, n) for i, n in enumerate(sizes)]

    def _given_states(self, m, v, bits):
        self.m, self.v = list(m), list(v)
        if len(self.m) != self.count or len(self.v) != self.count:
            raise ValueError("m and v need one entry for each tensor")
        pairs = {isinstance(t, (tuple, list)) for t in self.m + self.v}
        if len(pairs) > 1:
            raise ValueError("states are all in 32 bits or all in 8")
        held = 8 if pairs == {True} else 32 if pairs else bits or 32
        if bits is not None and bits != held:
            raise ValueError(f"states are in {held} bits, not in {bits}")
        self.bits = held

    def _take(self, t, dtypes, name, n, spans, like=None):
        """(address, type) of a tensor of n elements, in the order of a tensor of shape
        `like` (None: any); its span joins `spans`."""
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name} is required")
        if t.dtype not in dtypes:
            raise TypeError(f"{name}: expected {' or '.join(map(str, dtypes))}, got {t.dtype}")
        if not t.is_cuda:
            raise TypeError(f"{name} must be a device tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.numel() != n:
            raise ValueError(f"{name}: expected {n} elements, got {t.numel()}")
        if like is not None and t.shape != like and not _same_order(tuple(t.shape), like):
            raise ValueError(f"{name}: shape {tuple(t.shape)} is in another order than the "
                             f"weight's {like}")
        if self.device is None:
            self.device, self.torch_device = t.get_device(), t.device
        if t.get_device() != self.device:
            raise ValueError(f"{name} is on {t.device}, not on the other tensors' device")
        if n:
            spans.append((t.data_ptr(), t.data_ptr() + n * t.element_size(), name))
        return t.data_ptr(), _TYPES.get(t.dtype, 0)

    def set_grads(self, g):
        """Other gradient tensors, one for each weight.  (A captured step reads those it
        was captured with: keep them.)"""
        g = list(g)
        if len(g) != self.count:
            raise ValueError("g needs one entry for each tensor")
        read = []
        at = [self._take(t, tuple(_TYPES), f"g[{i}]", n, read, like)
              for i, (t, n, like) in enumerate(zip(g, self.sizes, self.shapes))]
        # what a step writes lies apart from all else that it reads or writes
        spans = sorted([s + (True,) for s in self._written] + [s + (False,) for s in read])
        last, last_written = (0, 0, None), (0, 0, None)  # the spans that reach furthest
        for s in spans:
            over = last if s[3] else last_written
            if s[0] < over[1]:
                raise ValueError(f"{s[2]} overlaps {over[2]}")
            last = max(last, s, key=lambda x: x[1])
            if s[3]:
                last_written = max(last_written, s, key=lambda x: x[1])
        for p, n, (a, kind) in zip(self.array, self.sizes, at):
            p.g, p.g_type, p.n = a, kind, n
        self.g = g
        need = ctypes.c_size_t()
        _check(lib.moe_grad_sumsq_workspace_bytes(self.array, self.count, ctypes.byref(need)),
               "moe_grad_sumsq_workspace_bytes")
        self.sumsq_bytes = need.value

    def on_device(self):
        """Refuses a current device that is not the tensors' own."""
        if self.device is not None and self.device != torch._C._cuda_getDevice():
            raise ValueError(f"the tensors are on cuda:{self.device}, not on the current device")
        return self


def moe_grad_sumsq(params, sumsq=None):
    """Sum of squares of all gradients of `params` (a Params, or a list of bf16
    and fp32 tensors).  Returns sumsq [1] fp32; ranks that hold parts of a model
    add theirs up before moe_adamw_step clips by it."""
    if not isinstance(params, Params):
        params = Params(None, params)
    params.on_device()
    dev = params.torch_device or torch.device("cuda", torch.cuda.current_device())
    sumsq = _out(sumsq, torch.float32, "sumsq", (1,), dev)
    ws = workspace(params.sumsq_bytes, dev, "grad_sumsq")
    _check(lib.moe_grad_sumsq(params.array, params.count, _ptr(sumsq), _ptr(ws), ws.numel(),
                              _stream()), "moe_grad_sumsq")
    return sumsq


def _number(v, dtype, name):
    """(host number or 0, address or None) of a number or a device scalar [1]."""
    if isinstance(v, torch.Tensor):
        return 0, _given(v, dtype, name, (1,)).data_ptr()
    return v, None


def moe_adamw_step(params, lr, step, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1,
                   grad_sumsq=None, max_norm=float("inf"), seed=0):
    """One AdamW step of all tensors of `params`, in place.  lr and step (1 for the
    first) are numbers, or device tensors [1] (fp32, int32) that a captured step
    reads at every replay.  grad_sumsq [1] fp32: gradients are clipped to a norm of
    max_norm by it, and a step with a sum that is not finite is left out.  seed: of
    the random rounding of 8-bit states and of bf16 weights (with the step and the
    tensor's place in the list; give lists of one model seeds of their own)."""
    params.on_device()
    if params.w is None:
        raise ValueError("these params have no weights")
    if not params.count:
        return
    if grad_sumsq is not None:
        _given(grad_sumsq, torch.float32, "grad_sumsq", (1,))
    lr, lr_device = _number(lr, torch.float32, "lr")
    step, step_device = _number(step, torch.int32, "step")
    o = AdamWOptions(lr, beta1, beta2, eps, weight_decay, step, lr_device, step_device,
                     _ptr(grad_sumsq), max_norm, seed & 0xFFFFFFFF)
    _check(lib.moe_adamw_step(params.array, params.count, params.bits, ctypes.byref(o), _stream()),
           "moe_adamw_step")


def moe_adamw_states(params, m=None, v=None):
    """The values of 8-bit states: two lists of fp32 tensors [n] (m, v: given ones
    to write, apart from each other and from what `params` names)."""
    params.on_device()
    if params.w is None or params.bits != 8:
        raise ValueError("these params have no 8-bit states")
    if not params.count:
        return [], []
    out = []
    for name, given in (("m", m), ("v", v)):
        given = [None] * params.count if given is None else list(given)
        if len(given) != params.count:
            raise ValueError(f"{name} needs one entry for each tensor")
        out.append([_out(t, torch.float32, f"{name}[{i}]", (n,), params.torch_device)
                    for i, (t, n) in enumerate(zip(given, params.sizes))])
    at = [(ctypes.c_void_p * max(params.count, 1))(*[t.data_ptr() for t in o]) for o in out]
    _check(lib.moe_adamw_states(params.array, params.count, *at, _stream()), "moe_adamw_states")
    return tuple(out)


# ------------------------------------------ least-loaded expert parallelism
def moe_llep_plan(counts, E_p, capacity=0, granule=1):
    """Plan of which rank computes which rows of every expert, load counted
    in units of `granule` rows (1: rows; the GEMM row tile, 256: tiles).
    counts [E] int32 (device).  Returns (win_lo [E_p,E], win_hi [E_p,E],
    load [E_p] rows, n_ship [1]), int32 device tensors."""
    _need(counts, torch.int32, "counts", 1)
    E = counts.shape[0]
    dev = counts.device
    lo = torch.empty((E_p, E), dtype=torch.int32, device=dev)
    hi = torch.empty((E_p, E), dtype=torch.int32, device=dev)
    load = torch.empty((E_p,), dtype=torch.int32, device=dev)
    n_ship = torch.empty((1,), dtype=torch.int32, device=dev)
    _check(lib.moe_llep_plan(_ptr(counts), E, E_p, capacity, granule, _ptr(lo), _ptr(hi),
                             _ptr(load), _ptr(n_ship), _stream()), "moe_llep_plan")
    return lo, hi, load, n_ship


def moe_llep_dispatch(x, topk_idx, offsets_all, dst_all, win_lo, win_hi, rank, cap):
    """Rank `rank`'s rows under a plan, from the all-expert permutation.
    Returns {expert_offsets [E+1], row_src [cap], dst [T,k], x_perm [cap,d]}."""
    _need(x, torch.bfloat16, "x", 2)
    _need(topk_idx, torch.int32, "topk_idx", 2)
    _need(offsets_all, torch.int32, "offsets_all", 1)
    _need(dst_all, torch.int32, "dst_all")
    _need(win_lo, torch.int32, "win_lo", 2)
    _need(win_hi, torch.int32, "win_hi", 2)
    T, d = x.shape
    k = topk_idx.shape[1]
    E_p, E = win_lo.shape
    dev = x.device
    out = {"expert_offsets": torch.empty((E + 1,), dtype=torch.int32, device=dev),
           "row_src": torch.empty((max(cap, 1),), dtype=torch.int32, device=dev),
           "dst": torch.empty((T, k), dtype=torch.int32, device=dev),
           "x_perm": torch.empty((max(cap, 1), d), dtype=torch.bfloat16, device=dev)}
    _check(lib.moe_llep_dispatch(_ptr(x), _ptr(topk_idx), _ptr(offsets_all), _ptr(dst_all),
                                 _ptr(win_lo), _ptr(win_hi), E_p, rank, T, d, E, k, cap,
                                 _ptr(out["expert_offsets"]), _ptr(out["row_src"]),
                                 _ptr(out["dst"]), _ptr(out["x_perm"]), _stream()),
           "moe_llep_dispatch")
    return out


# ------------------------------------------------------------- profiling
def profile_enable(on: bool):
    _check(lib.moe_profile_enable(1 if on else 0), "moe_profile_enable")


def profile_reset():
    _check(lib.moe_profile_reset(), "moe_profile_reset")


def profile_query() -> dict:
    """{kernel name: (total ms, launches)} over the recorded events."""
    out = {}
    for i in range(lib.moe_profile_num_kernels()):
        ms = ctypes.c_double()
        n = ctypes.c_int64()
        _check(lib.moe_profile_query(i, ctypes.byref(ms), ctypes.byref(n)), "moe_profile_query")
        if n.value:
            out[lib.moe_profile_kernel_name(i).decode()] = (ms.value, n.value)
    return out


# ------------------------------------------------------------- whole layer
def layer_fwd_bwd(inp: dict, k: int, expert_begin=0, num_local=None, renorm=0,
                  keep: bool = True, router_loss=None) -> dict:
    """One forward + backward pass of the MoE expert layer through the C ABI.

    inp: x, w_router, router_bias, w_gate, w_up, w_down, dy (device tensors).
    Returns every intermediate (routing, permutation, activations, grads).

    router_loss = (cb, cz) trains the router too: the step's loss also has cb
    times the balance loss and cz times the z-loss of the whole batch (or, with
    inp["seq_offsets"] and inp["token_mask"], their means over its sequences
    and without its padding), dx becomes the whole layer's, and dw_router,
    dbias (with a router bias), balance, zloss and expert_counts are returned.
    With num_local < E experts (an expert-parallel rank, which sees the same
    tokens as its peers) dx, dw_router and dbias are this rank's terms of sums
    over the ranks; num_local / E of the two losses' gradient is in each, so
    that the sums hold it once.  balance and zloss are whole on every rank.

    With inp["norm_gamma"] (and, optionally, norm_beta, norm_eps and residual) the
    layer stands in a pre-norm block: h = x + residual, y is the layer's output on
    the layer norm of h, and dy the gradient of h + y (the next norm's sum), which
    reaches h both ways; dx is then the gradient of h (as without a norm, the router's
    share is in it with router_loss only), and h, dgamma and dbeta are returned.  All
    experts have to be local: the ranks' dx would each hold dy.
    """
    x = inp["x"]
    norm = None
    if inp.get("norm_gamma") is not None:
        if num_local not in (None, inp["w_router"].shape[1]):
            raise ValueError("a block's norm needs all experts on this rank")
        norm = moe_layer_norm_fwd(x, inp["norm_gamma"], inp.get("norm_beta"),
                                  inp.get("norm_eps", 1e-5), inp.get("residual"))
        x = norm[0]
    elif inp.get("residual") is not None:
        raise ValueError("residual needs norm_gamma")
    E = inp["w_router"].shape[1]
    num_local = E if num_local is None else num_local
    logits = None
    if router_loss is not None:
        logits = torch.empty((x.shape[0], E), dtype=torch.float32, device=x.device)
    idx, gate = moe_route(x, inp["w_router"], inp.get("router_bias"), k, renorm, logits=logits)
    pm = moe_permute(x, idx, E, expert_begin, num_local)
    off = pm["expert_offsets"]
    hg, hu, y_perm = moe_grouped_swiglu_fwd(pm["x_perm"], off, inp["w_gate"], inp["w_up"],
                                            inp["w_down"])
    y = moe_combine(y_perm, pm["dst"], gate)
    dy_perm, dgate = moe_combine_bwd(inp["dy"], y_perm, pm["dst"], gate)
    dx_perm, dwg, dwu, dwd = moe_grouped_swiglu_bwd(dy_perm, pm["x_perm"], hg, hu, off,
                                                    inp["w_gate"], inp["w_up"], inp["w_down"])
    dx = moe_combine(dx_perm, pm["dst"], None)
    out = {"topk_idx": idx, "topk_gate": gate, "y": y, "dgate": dgate, "dx": dx,
           "dw_gate": dwg, "dw_up": dwu, "dw_down": dwd}
    if router_loss is not None:
        seq, mask = inp.get("seq_offsets"), inp.get("token_mask")
        balance, zloss, counts, _, n = moe_balance_loss_fwd(logits, idx, seq, mask)
        G = n.shape[0]
        db, dz = (torch.full((G,), c / G * (num_local / E), dtype=torch.float32, device=x.device)
                  for c in router_loss)
        aux = moe_balance_loss_bwd(logits, counts, n, db, dz, k, seq, mask)
        dwr, dbias, _ = moe_route_bwd(x, inp["w_router"], logits, idx, gate, dgate, renorm, dx=dx,
                                      with_dbias=inp.get("router_bias") is not None,
                                      dlogits_aux=aux)
        out.update(balance=balance, zloss=zloss, expert_counts=counts, dw_router=dwr)
        if dbias is not None:
            out["dbias"] = dbias
    if norm is not None:
        _, h, mean, rstd = norm
        dx, dgamma, dbeta = moe_layer_norm_bwd(dx, h, inp["norm_gamma"], mean, rstd, inp["dy"],
                                               with_dbeta=inp.get("norm_beta") is not None)
        out.update(dx=dx, h=h, dgamma=dgamma, dbeta=dbeta)
    if keep:
        out.update(pm)
        out.update(h_gate=hg, h_up=hu, y_perm=y_perm, dy_perm=dy_perm, dx_perm=dx_perm)
    return out

"""Python binding of the LAEP MoE C ABI on torch tensors.

Argument marshalling only: each function checks tensor placement and
layout, allocates missing outputs with torch (device memory is PyTorch's
job), and calls the same-named C entry point on the current HIP stream.
Every step of the layer runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional, Tuple

import torch

from ._lib import (LAEP_ACT8_BLOCK, LAEP_BF16, LAEP_CALL_BALANCE, LAEP_CALL_COUNTS,
                   LAEP_CALL_FFN_BWD, LAEP_CALL_FFN_FWD, LAEP_CALL_LAYER_NORM_BWD,
                   LAEP_CALL_MX4_FFN, LAEP_CALL_MX4_PRODUCT, LAEP_CALL_ROUTE_BWD, LAEP_F32,
                   LAEP_MX4_GROUP, LaepError, check, lib)

_DT = {torch.float32: LAEP_F32, torch.bfloat16: LAEP_BF16}


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype not in _DT:
        raise LaepError(2, f"unsupported dtype {t.dtype}")
    return _DT[t.dtype]


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _dev(t: torch.Tensor, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _stream(device) -> int:
    # the current stream's handle without the Stream object around it, whose making
    # costs 2 us of every call
    return torch._C._cuda_getCurrentRawStream(device.index)


def workspace_bytes(which: int, T: int, k: int, E: int, d_model: int = 0, d_ff: int = 0) -> int:
    return int(lib().moe_workspace_bytes(which, T, k, E, d_model, d_ff))


def _workspace(ws, nbytes, device):
    if ws is None:
        return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
    if ws.numel() * ws.element_size() < nbytes:
        raise LaepError(3, f"workspace {ws.numel() * ws.element_size()} < {nbytes} bytes")
    return ws


# ---------------------------------------------------------------------------
def moe_route(x: torch.Tensor, w_router: torch.Tensor, k: int, *, bias=None, alive=None,
              renorm: bool = True, want_logits: bool = False, topk_idx=None, topk_gate=None):
    """Router scoring + top-k gating.  Returns (topk_idx, topk_gate[, logits])."""
    _dev(x, "x"), _dev(w_router, "w_router")
    T, d = x.shape
    E = w_router.shape[0]
    dev = x.device
    if topk_idx is None:
        topk_idx = torch.empty((T, k), dtype=torch.int32, device=dev)
    if topk_gate is None:
        topk_gate = torch.empty((T, k), dtype=torch.float32, device=dev)
    logits = torch.empty((T, E), dtype=torch.float32, device=dev) if want_logits else None
    if bias is not None:
        _dev(bias, "bias")
    if alive is not None:
        _dev(alive, "alive")
    check(lib().moe_route(_ptr(x), _ptr(w_router), _ptr(bias), _ptr(alive), _dtype_code(x), T, d,
                          E, k, int(renorm), _ptr(logits), _ptr(topk_idx), _ptr(topk_gate), None,
                          0, _stream(dev)))
    return (topk_idx, topk_gate, logits) if want_logits else (topk_idx, topk_gate)


def moe_route_bwd(dgate: torch.Tensor, topk_idx: torch.Tensor, topk_gate: torch.Tensor,
                  x: torch.Tensor, w_router: torch.Tensor, *, renorm: bool = True,
                  logits=None, alive=None, offsets=None, row_src=None, dx=None,
                  accumulate_dx: bool = False, want_dlogits: bool = False,
                  want_dbias: bool = False, dw_router=None, dlogits=None, dbias=None, ws=None,
                  data: bool = True, weights: bool = True):
    """Router/gate backward with the selection fixed.  ``data=False`` skips dx,
    ``weights=False`` skips dw_router and dbias.
    Returns (dx, dw_router, dbias, dlogits), None for what was not computed."""
    for t, n in ((dgate, "dgate"), (topk_idx, "topk_idx"), (topk_gate, "topk_gate"), (x, "x"),
                 (w_router, "w_router")):
        _dev(t, n)
    T, k = topk_idx.shape
    E, d = w_router.shape
    dev = x.device
    if data:
        if dx is None:   # overwritten whole unless accumulated onto
            dx = torch.zeros_like(x) if accumulate_dx else torch.empty_like(x)
    else:
        dx = None
    if weights:
        dw_router = (torch.empty((E, d), dtype=torch.float32, device=dev) if dw_router is None
                     else dw_router)
        if want_dbias and dbias is None:
            dbias = torch.empty(E, dtype=torch.float32, device=dev)
    else:
        dw_router, dbias = None, None
    if want_dlogits and dlogits is None:
        dlogits = torch.empty((T, E), dtype=torch.float32, device=dev)
    ws = _workspace(ws, workspace_bytes(LAEP_CALL_ROUTE_BWD, T, k, E, d), dev)
    check(lib().moe_route_bwd(_ptr(dgate), _ptr(topk_idx), _ptr(topk_gate), _ptr(logits),
                              _ptr(alive), _ptr(x), _ptr(w_router), _ptr(offsets), _ptr(row_src),
                              _dtype_code(x), T, d, E, k, int(renorm), _ptr(dlogits),
                              _ptr(dw_router), _ptr(dbias), _ptr(dx), int(accumulate_dx),
                              _ptr(ws), ws.numel(), _stream(dev)))
    return dx, dw_router, dbias, dlogits


def moe_expert_counts(topk_idx: torch.Tensor, E: int, *, want_row_src: bool = False,
                      etn_accum=None, ws=None, counts=None, offsets=None, dest_row=None,
                      row_src=None):
    """Returns (counts [E] i32, offsets [E+1] i32, dest_row [T*k] i32[, row_src])."""
    _dev(topk_idx, "topk_idx")
    T, k = topk_idx.shape
    dev = topk_idx.device
    counts = torch.empty(E, dtype=torch.int32, device=dev) if counts is None else counts
    offsets = torch.empty(E + 1, dtype=torch.int32, device=dev) if offsets is None else offsets
    dest_row = torch.empty(T * k, dtype=torch.int32, device=dev) if dest_row is None else dest_row
    want_row_src = want_row_src or row_src is not None
    if want_row_src and row_src is None:
        row_src = torch.empty(T * k, dtype=torch.int32, device=dev)
    nbytes = workspace_bytes(LAEP_CALL_COUNTS, T, k, E)
    ws = _workspace(ws, nbytes, dev)
    check(lib().moe_expert_counts(_ptr(topk_idx), T, k, E, _ptr(counts), _ptr(offsets),
                                  _ptr(dest_row), _ptr(row_src), _ptr(etn_accum), _ptr(ws),
                                  ws.numel(), _stream(dev)))
    out = (counts, offsets, dest_row)
    return out + (row_src,) if want_row_src else out


def moe_route_count(x: torch.Tensor, w_router: torch.Tensor, k: int, *, bias=None, alive=None,
                    renorm: bool = True, want_logits: bool = False, want_row_src: bool = False,
                    etn_accum=None, ws=None, topk_idx=None, topk_gate=None, counts=None,
                    offsets=None, dest_row=None, row_src=None, logits=None):
    """Routing and expert counts in one call.  Returns (topk_idx, topk_gate,
    counts, offsets, dest_row, row_src or None, logits or None)."""
    _dev(x, "x"), _dev(w_router, "w_router")
    T, d = x.shape
    E = w_router.shape[0]
    dev = x.device
    i32 = torch.int32
    topk_idx = torch.empty((T, k), dtype=i32, device=dev) if topk_idx is None else topk_idx
    topk_gate = (torch.empty((T, k), dtype=torch.float32, device=dev) if topk_gate is None
                 else topk_gate)
    counts = torch.empty(E, dtype=i32, device=dev) if counts is None else counts
    offsets = torch.empty(E + 1, dtype=i32, device=dev) if offsets is None else offsets
    dest_row = torch.empty(T * k, dtype=i32, device=dev) if dest_row is None else dest_row
    if want_row_src and row_src is None:
        row_src = torch.empty(T * k, dtype=i32, device=dev)
    if want_logits or logits is not None:
        logits = _out(logits, "logits", (T, E), torch.float32, dev)
    ws = _workspace(ws, workspace_bytes(LAEP_CALL_COUNTS, T, k, E), dev)
    check(lib().moe_route_count(_ptr(x), _ptr(w_router), _ptr(bias), _ptr(alive), _dtype_code(x),
                                T, d, E, k, int(renorm), _ptr(logits), _ptr(topk_idx),
                                _ptr(topk_gate), _ptr(counts), _ptr(offsets), _ptr(dest_row),
                                _ptr(row_src), _ptr(etn_accum), _ptr(ws), ws.numel(),
                                _stream(dev)))
    return topk_idx, topk_gate, counts, offsets, dest_row, row_src, logits


def moe_route_count_noalloc(x: torch.Tensor, w_router: torch.Tensor, k: int, *, bias=None,
                            alive=None, renorm: bool = True, want_logits: bool = False,
                            want_row_src: bool = False, etn_accum=None, topk_idx=None,
                            topk_gate=None, counts=None, offsets=None, dest_row=None,
                            row_src=None, logits=None):
    """moe_route_count with the library's own scratch array (no workspace;
    the C call allocates nothing).  Pass every output to keep this wrapper
    allocation-free too.  Returns as moe_route_count."""
    _dev(x, "x"), _dev(w_router, "w_router")
    T, d = x.shape
    E = w_router.shape[0]
    dev = x.device
    i32 = torch.int32
    topk_idx = torch.empty((T, k), dtype=i32, device=dev) if topk_idx is None else topk_idx
    topk_gate = (torch.empty((T, k), dtype=torch.float32, device=dev) if topk_gate is None
                 else topk_gate)
    counts = torch.empty(E, dtype=i32, device=dev) if counts is None else counts
    offsets = torch.empty(E + 1, dtype=i32, device=dev) if offsets is None else offsets
    dest_row = torch.empty(T * k, dtype=i32, device=dev) if dest_row is None else dest_row
    if want_row_src and row_src is None:
        row_src = torch.empty(T * k, dtype=i32, device=dev)
    if want_logits and logits is None:
        logits = torch.empty((T, E), dtype=torch.float32, device=dev)
    check(lib().moe_route_count_noalloc(_ptr(x), _ptr(w_router), _ptr(bias), _ptr(alive),
                                        _dtype_code(x), T, d, E, k, int(renorm), _ptr(logits),
                                        _ptr(topk_idx), _ptr(topk_gate), _ptr(counts),
                                        _ptr(offsets), _ptr(dest_row), _ptr(row_src),
                                        _ptr(etn_accum), _stream(dev)))
    return topk_idx, topk_gate, counts, offsets, dest_row, row_src, logits


def laep_prune_mask(counts: torch.Tensor, total: int, alpha: float = math.inf,
                    beta: float = 0.0, *, alive=None, n_pruned=None):
    """LAEP prune decision.  Returns (alive [E] uint8, n_pruned [1] int32)."""
    _dev(counts, "counts")
    E = counts.shape[0]
    dev = counts.device
    alive = torch.empty(E, dtype=torch.uint8, device=dev) if alive is None else alive
    n_pruned = torch.empty(1, dtype=torch.int32, device=dev) if n_pruned is None else n_pruned
    check(lib().laep_prune_mask(_ptr(counts), E, int(total), float(alpha), float(beta),
                                _ptr(alive), _ptr(n_pruned), _stream(dev)))
    return alive, n_pruned


def laep_expert_pruning(etn: torch.Tensor, total: int, alpha, beta: float, *,
                        alive=None, n_pruned=None, want_marker: bool = False):
    """Algorithm 1 over a recorded window etn [ITER, L, E] int64.  ``alpha`` is a
    float or a per-layer sequence.  Returns (alive [L, E] uint8, n_pruned [L]
    int32, marker [L, E] int32 or None)."""
    _dev(etn, "etn")
    if etn.dtype != torch.int64 or etn.dim() != 3:
        raise ValueError("etn must be an int64 tensor [ITER, L, E]")
    iters, L, E = etn.shape
    alphas = [float(alpha)] * L if isinstance(alpha, (int, float)) else [float(a) for a in alpha]
    if len(alphas) != L:
        raise ValueError(f"alpha has {len(alphas)} entries for {L} layers")
    dev = etn.device
    alive = torch.empty((L, E), dtype=torch.uint8, device=dev) if alive is None else alive
    n_pruned = torch.empty(L, dtype=torch.int32, device=dev) if n_pruned is None else n_pruned
    marker = torch.empty((L, E), dtype=torch.int32, device=dev) if want_marker else None
    a_host = (ctypes.c_double * L)(*alphas)
    check(lib().laep_expert_pruning(_ptr(etn), iters, L, E, int(total), a_host, float(beta),
                                    _ptr(alive), _ptr(n_pruned), _ptr(marker), _stream(dev)))
    return alive, n_pruned, marker


def laep_compact_experts(alive: torch.Tensor, *, expert_map=None, n_alive=None):
    """Slots of the surviving experts.  alive [E] or [L, E] uint8.
    Returns (expert_map of alive's shape int32, n_alive [L] int32)."""
    _dev(alive, "alive")
    a2 = alive.reshape(-1, alive.shape[-1])
    L, E = a2.shape
    dev = alive.device
    expert_map = (torch.empty(alive.shape, dtype=torch.int32, device=dev) if expert_map is None
                  else expert_map)
    n_alive = torch.empty(L, dtype=torch.int32, device=dev) if n_alive is None else n_alive
    check(lib().laep_compact_experts(_ptr(alive), L, E, _ptr(expert_map), _ptr(n_alive),
                                     _stream(dev)))
    return expert_map, n_alive


def laep_repack_experts(expert_map: torch.Tensor, n_out: int, *, w_router=None, bias=None,
                        w_gate_up=None, w_down=None, out=None):
    """Copy the surviving experts' parameters (one layer) into n_out slots.
    Returns a dict with the repacked tensors that were given."""
    _dev(expert_map, "expert_map")
    E = expert_map.shape[0]
    given = {n: t for n, t in (("w_router", w_router), ("bias", bias), ("w_gate_up", w_gate_up),
                               ("w_down", w_down)) if t is not None}
    mats = [t for n, t in given.items() if n != "bias"]
    dtype = mats[0].dtype if mats else torch.float32
    if any(t.dtype != dtype for t in mats):
        raise ValueError("the repacked matrices must share one dtype")
    d_model = (w_router.shape[1] if w_router is not None else
               w_gate_up.shape[2] if w_gate_up is not None else
               w_down.shape[1] if w_down is not None else 8)
    d_ff = (w_gate_up.shape[1] // 2 if w_gate_up is not None else
            w_down.shape[2] if w_down is not None else 0)
    for n, t in given.items():
        _dev(t, n)
        if t.shape[0] != E:
            raise ValueError(f"{n} has {t.shape[0]} experts, expert_map {E}")
    out = {} if out is None else dict(out)
    for n, t in given.items():
        if n not in out:
            out[n] = torch.empty((n_out, *t.shape[1:]), dtype=t.dtype, device=t.device)
    code = _dtype_code(mats[0]) if mats else LAEP_F32
    check(lib().laep_repack_experts(_ptr(expert_map), E, int(n_out), code, d_model, d_ff,
                                    _ptr(w_router), _ptr(bias), _ptr(w_gate_up), _ptr(w_down),
                                    _ptr(out.get("w_router")), _ptr(out.get("bias")),
                                    _ptr(out.get("w_gate_up")), _ptr(out.get("w_down")),
                                    _stream(expert_map.device)))
    return out


def moe_permute(x: torch.Tensor, dest_row: torch.Tensor, k: int, rows: Optional[int] = None,
                *, out=None):
    """x_perm[dest_row[t*k+j]] = x[t].  ``rows`` defaults to T*k."""
    _dev(x, "x"), _dev(dest_row, "dest_row")
    T, d = x.shape
    rows = T * k if rows is None else rows
    out = torch.empty((rows, d), dtype=x.dtype, device=x.device) if out is None else out
    check(lib().moe_permute(_ptr(x), _dtype_code(x), _ptr(dest_row), T, k, d, _ptr(out),
                            _stream(x.device)))
    return out


def moe_grouped_ffn_fwd(x_perm: torch.Tensor, w_gate_up: torch.Tensor, w_down: torch.Tensor,
                        offsets: torch.Tensor, *, expert_map=None, save_act: bool = True,
                        ws=None, y_perm=None, act_save=None):
    """Grouped SwiGLU FFN.  Returns (y_perm, act_save or None)."""
    for t, n in ((x_perm, "x_perm"), (w_gate_up, "w_gate_up"), (w_down, "w_down"),
                 (offsets, "offsets")):
        _dev(t, n)
    R, d = x_perm.shape
    f = w_down.shape[2]
    E = offsets.shape[0] - 1
    dev = x_perm.device
    y_perm = torch.empty_like(x_perm) if y_perm is None else y_perm
    if save_act and act_save is None:
        act_save = torch.empty((R, 2 * f), dtype=x_perm.dtype, device=dev)
    if not save_act:
        act_save = None
    ws = _workspace(ws, workspace_bytes(LAEP_CALL_FFN_FWD, R, 1, E, d, f), dev)
    check(lib().moe_grouped_ffn_fwd(_ptr(x_perm), _ptr(w_gate_up), _ptr(w_down), _ptr(offsets),
                                    _ptr(expert_map), _dtype_code(x_perm), E, d, f, R,
                                    _ptr(y_perm), _ptr(act_save), _ptr(ws), ws.numel(),
                                    _stream(dev)))
    return y_perm, act_save


def moe_grouped_ffn_fwd_gather(x: torch.Tensor, row_src: torch.Tensor, k: int,
                               w_gate_up: torch.Tensor, w_down: torch.Tensor,
                               offsets: torch.Tensor, *, rows: Optional[int] = None,
                               expert_map=None, save_act: bool = False, ws=None, y_perm=None,
                               act_save=None, x_perm_out=None):
    """moe_permute + moe_grouped_ffn_fwd in one pass (bf16): routed row r reads
    token row row_src[r] // k; ``x_perm_out`` [R, d] (optional) also receives
    the dispatched rows, copied beside the FFN.  Returns (y_perm, act_save or None)."""
    for t, n in ((x, "x"), (row_src, "row_src"), (w_gate_up, "w_gate_up"), (w_down, "w_down"),
                 (offsets, "offsets")):
        _dev(t, n)
    T, d = x.shape
    R = T * k if rows is None else rows
    f = w_down.shape[2]
    E = offsets.shape[0] - 1
    dev = x.device
    y_perm = torch.empty((R, d), dtype=x.dtype, device=dev) if y_perm is None else y_perm
    if save_act and act_save is None:
        act_save = torch.empty((R, 2 * f), dtype=x.dtype, device=dev)
    if not save_act:
        act_save = None
    ws = _workspace(ws, workspace_bytes(LAEP_CALL_FFN_FWD, R, 1, E, d, f), dev)
    check(lib().moe_grouped_ffn_fwd_gather(_ptr(x), _ptr(row_src), T, k, _ptr(w_gate_up),
                                           _ptr(w_down), _ptr(offsets), _ptr(expert_map),
                                           _dtype_code(x), E, d, f, R, _ptr(y_perm),
                                           _ptr(act_save), _ptr(x_perm_out), _ptr(ws), ws.numel(),
                                           _stream(dev)))
    return y_perm, act_save


def moe_grouped_ffn_fwd_gather_combine(x: torch.Tensor, row_src: torch.Tensor,
                                       topk_gate: torch.Tensor, w_gate_up: torch.Tensor,
                                       w_down: torch.Tensor, offsets: torch.Tensor, *,
                                       rows: Optional[int] = None, expert_map=None,
                                       keep_y: bool = False, save_act: bool = False, ws=None,
                                       out=None, y_perm=None, act_save=None, x_perm_out=None):
    """moe_grouped_ffn_fwd_gather + moe_combine for one slot per token (bf16):
    routed row r goes straight to token row row_src[r], times its gate.
    Returns (out, y_perm or None, act_save or None)."""
    for t, n in ((x, "x"), (row_src, "row_src"), (topk_gate, "topk_gate"),
                 (w_gate_up, "w_gate_up"), (w_down, "w_down"), (offsets, "offsets")):
        _dev(t, n)
    T, d = x.shape
    R = T if rows is None else rows
    f = w_down.shape[2]
    E = offsets.shape[0] - 1
    dev = x.device
    out = torch.empty((T, d), dtype=x.dtype, device=dev) if out is None else out
    if keep_y and y_perm is None:
        y_perm = torch.empty((R, d), dtype=x.dtype, device=dev)
    if not keep_y:
        y_perm = None
    if save_act and act_save is None:
        act_save = torch.empty((R, 2 * f), dtype=x.dtype, device=dev)
    if not save_act:
        act_save = None
    ws = _workspace(ws, workspace_bytes(LAEP_CALL_FFN_FWD, R, 1, E, d, f), dev)
    check(lib().moe_grouped_ffn_fwd_gather_combine(
        _ptr(x), _ptr(row_src), T, 1, _ptr(w_gate_up), _ptr(w_down), _ptr(offsets),
        _ptr(expert_map), _ptr(topk_gate), _dtype_code(x), E, d, f, R, _ptr(out), _ptr(y_perm),
        _ptr(act_save), _ptr(x_perm_out), _ptr(ws), ws.numel(), _stream(dev)))
    return out, y_perm, act_save


def moe_grouped_ffn_bwd(dy_perm, x_perm, act_save, w_gate_up, w_down, offsets, *,
                        h_fwd=None, expert_map=None, dw_gate_up=None, dw_down=None,
                        accumulate=False, ws=None, dx_perm=None, return_ws: bool = False):
    """Backward of the grouped FFN.  ``h_fwd``: the forward's H [R, f] (see
    ffn_fwd_h_view); dW_d then uses it, else H_b recomputed at act_save.
    Returns (dx_perm, dw_gate_up, dw_down[, ws])."""
    for t, n in ((dy_perm, "dy_perm"), (x_perm, "x_perm"), (act_save, "act_save"),
                 (w_gate_up, "w_gate_up"), (w_down, "w_down"), (offsets, "offsets")):
        _dev(t, n)
    if h_fwd is not None:
        _dev(h_fwd, "h_fwd")
    R, d = x_perm.shape
    f = w_down.shape[2]
    E = offsets.shape[0] - 1
    dev = x_perm.device
    dx_perm = torch.empty_like(x_perm) if dx_perm is None else dx_perm
    if dw_gate_up is None:
        dw_gate_up = torch.empty(w_gate_up.shape, dtype=torch.float32, device=dev)
    if dw_down is None:
        dw_down = torch.empty(w_down.shape, dtype=torch.float32, device=dev)
    ws = _workspace(ws, workspace_bytes(LAEP_CALL_FFN_BWD, R, 1, E, d, f), dev)
    check(lib().moe_grouped_ffn_bwd(_ptr(dy_perm), _ptr(x_perm), _ptr(act_save), _ptr(h_fwd),
                                    _ptr(w_gate_up), _ptr(w_down), _ptr(offsets),
                                    _ptr(expert_map), _dtype_code(x_perm), E, d, f, R,
                                    _ptr(dx_perm), _ptr(dw_gate_up), _ptr(dw_down),
                                    int(accumulate), _ptr(ws), ws.numel(), _stream(dev)))
    out = (dx_perm, dw_gate_up, dw_down)
    return out + (ws,) if return_ws else out


def moe_grouped_ffn_bwd_gather(dy_perm, x, row_src, k: int, act_save, w_gate_up, w_down,
                               offsets, *, dout=None, topk_gate=None, h_fwd=None,
                               expert_map=None, dw_gate_up=None, dw_down=None, accumulate=False,
                               ws=None, dx_perm=None, return_ws: bool = False):
    """moe_grouped_ffn_bwd with the weight gradient reading X's routed rows
    from the token rows x through row_src (no x_perm).  With dy_perm None,
    dY is formed on load from ``dout`` [T, d] and ``topk_gate`` [T, k] (no
    dy_perm).  Returns as moe_grouped_ffn_bwd."""
    for t, n in ((x, "x"), (row_src, "row_src"), (act_save, "act_save"),
                 (w_gate_up, "w_gate_up"), (w_down, "w_down"), (offsets, "offsets")):
        _dev(t, n)
    if dy_perm is None:
        if dout is None or topk_gate is None:
            raise ValueError("without dy_perm, dout and topk_gate are needed")
        _dev(dout, "dout"), _dev(topk_gate, "topk_gate")
    else:
        _dev(dy_perm, "dy_perm")
    if h_fwd is not None:
        _dev(h_fwd, "h_fwd")
    T, d = x.shape
    R = row_src.shape[0]
    f = w_down.shape[2]
    E = offsets.shape[0] - 1
    dev = x.device
    dx_perm = torch.empty((R, d), dtype=x.dtype, device=dev) if dx_perm is None else dx_perm
    if dw_gate_up is None:
        dw_gate_up = torch.empty(w_gate_up.shape, dtype=torch.float32, device=dev)
    if dw_down is None:
        dw_down = torch.empty(w_down.shape, dtype=torch.float32, device=dev)
    ws = _workspace(ws, workspace_bytes(LAEP_CALL_FFN_BWD, R, 1, E, d, f), dev)
    check(lib().moe_grouped_ffn_bwd_gather(
        _ptr(dy_perm), _ptr(dout), _ptr(topk_gate), _ptr(x), _ptr(row_src), T, k,
        _ptr(act_save), _ptr(h_fwd),
        _ptr(w_gate_up), _ptr(w_down), _ptr(offsets), _ptr(expert_map), _dtype_code(x), E, d, f,
        R, _ptr(dx_perm), _ptr(dw_gate_up), _ptr(dw_down), int(accumulate), _ptr(ws), ws.numel(),
        _stream(dev)))
    out = (dx_perm, dw_gate_up, dw_down)
    return out + (ws,) if return_ws else out


def ffn_fwd_h_view(ws: torch.Tensor, R: int, d_ff: int, dtype: torch.dtype):
    """H [R, f] as the forward leaves it in its workspace (byte offset 0)."""
    esz = torch.empty((), dtype=dtype).element_size()
    return ws.view(torch.uint8)[: R * d_ff * esz].view(dtype).view(R, d_ff)


def ffn_bwd_ws_views(ws: torch.Tensor, R: int, d_ff: int, dtype: torch.dtype):
    """dA [R, 2f] and the H_b buffer [R, f] (H_b, or dH when the backward
    used the forward's H) as left in the backward workspace."""
    code = _DT[dtype]
    esz = torch.empty((), dtype=dtype).element_size()
    off = int(lib().laep_ws_hb_offset(R, d_ff, code))
    raw = ws.view(torch.uint8)
    dA = raw[: R * 2 * d_ff * esz].view(dtype).view(R, 2 * d_ff)
    hb = raw[off: off + R * d_ff * esz].view(dtype).view(R, d_ff)
    return dA, hb


def moe_combine(y_perm: torch.Tensor, topk_gate: torch.Tensor, dest_row: torch.Tensor,
                *, out=None):
    """out[t] = sum_j g[t,j] * y_perm[dest_row[t*k+j]]."""
    _dev(y_perm, "y_perm"), _dev(topk_gate, "topk_gate"), _dev(dest_row, "dest_row")
    T, k = topk_gate.shape
    d = y_perm.shape[1]
    out = torch.empty((T, d), dtype=y_perm.dtype, device=y_perm.device) if out is None else out
    check(lib().moe_combine(_ptr(y_perm), _ptr(topk_gate), _ptr(dest_row), T, k, d,
                            _dtype_code(y_perm), _ptr(out), _stream(y_perm.device)))
    return out


def moe_combine_bwd(dout: torch.Tensor, y_perm: torch.Tensor, topk_gate: torch.Tensor,
                    dest_row: torch.Tensor, *, dy_perm=None, dgate=None, want_dy: bool = True):
    """Returns (dy_perm, dgate); with want_dy False only dgate is computed
    (dy_perm None: moe_grouped_ffn_bwd_gather forms dY itself)."""
    for t, n in ((dout, "dout"), (y_perm, "y_perm"), (topk_gate, "topk_gate"),
                 (dest_row, "dest_row")):
        _dev(t, n)
    T, k = topk_gate.shape
    d = dout.shape[1]
    dev = dout.device
    if want_dy and dy_perm is None:
        dy_perm = torch.empty_like(y_perm)
    if not want_dy:
        dy_perm = None
    dgate = torch.empty((T, k), dtype=torch.float32, device=dev) if dgate is None else dgate
    check(lib().moe_combine_bwd(_ptr(dout), _ptr(y_perm), _ptr(topk_gate), _ptr(dest_row), T, k,
                                d, _dtype_code(dout), _ptr(dy_perm), _ptr(dgate), _stream(dev)))
    return dy_perm, dgate


def moe_permute_bwd(dx_perm: torch.Tensor, dest_row: torch.Tensor, T: int, k: int, *, out=None):
    """dx[t] = sum_j dx_perm[dest_row[t*k+j]]."""
    _dev(dx_perm, "dx_perm"), _dev(dest_row, "dest_row")
    d = dx_perm.shape[1]
    out = torch.empty((T, d), dtype=dx_perm.dtype, device=dx_perm.device) if out is None else out
    check(lib().moe_permute_bwd(_ptr(dx_perm), _ptr(dest_row), T, k, d, _dtype_code(dx_perm),
                                _ptr(out), _stream(dx_perm.device)))
    return out


def laep_rearrange(loads, n_groups: int):
    """Host utility (Algorithm 2).  Returns dict(group_of, order, sums)."""
    import numpy as np

    loads = np.ascontiguousarray(loads, dtype=np.float64)
    n = loads.shape[0]
    group_of = np.empty(n, dtype=np.int32)
    order = np.empty(n, dtype=np.int32)
    sums = np.empty(max(n_groups, 1), dtype=np.float64)
    check(lib().laep_rearrange(loads.ctypes.data, n, n_groups, group_of.ctypes.data,
                               order.ctypes.data, sums.ctypes.data))
    return dict(group_of=group_of, order=order, sums=sums[:n_groups])


# ---- the block around the experts (laep_block.h) ---------------------------------------
def _want(t: Optional[torch.Tensor], name: str, shape, dtype) -> Optional[torch.Tensor]:
    """A given device tensor of this shape and dtype (None passes)."""
    if t is None:
        return None
    if t.shape == shape and t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")
    return _dev(t, name)


def _out(t: Optional[torch.Tensor], name: str, shape, dtype, device) -> torch.Tensor:
    """The given output buffer, checked, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if t.shape == shape and t.dtype is dtype and t.is_cuda and t.is_contiguous():
        return t
    return _want(t, name, shape, dtype)


def moe_layer_norm(x: torch.Tensor, gamma: torch.Tensor, beta: Optional[torch.Tensor] = None, *,
                   residual=None, eps: float = 1e-5, out=None, sum_out=None, mean=None,
                   rstd=None):
    """Residual add and layer norm of the rows of x [T, d]; gamma and beta are
    float32 [d].  Returns (y, s, mean, rstd): s = x + residual as stored (x
    itself without a residual), the row statistics float32 [T].  ``sum_out``
    may be x or residual."""
    _dev(x, "x")
    T, d = x.shape
    dev = x.device
    _want(gamma, "gamma", (d,), torch.float32), _want(beta, "beta", (d,), torch.float32)
    _want(residual, "residual", (T, d), x.dtype)
    code = _dtype_code(x)
    y = _out(out, "out", (T, d), x.dtype, dev)
    if residual is not None or sum_out is not None:   # the C call refuses one without the other
        sum_out = _out(sum_out, "sum_out", (T, d), x.dtype, dev)
    mean = _out(mean, "mean", (T,), torch.float32, dev)
    rstd = _out(rstd, "rstd", (T,), torch.float32, dev)
    check(lib().moe_layer_norm(_ptr(x), _ptr(residual), _ptr(gamma), _ptr(beta), code, T, d,
                               float(eps), _ptr(sum_out), _ptr(y), _ptr(mean), _ptr(rstd),
                               _stream(dev)))
    return y, (x if sum_out is None else sum_out), mean, rstd


def moe_layer_norm_bwd(dy: torch.Tensor, s: torch.Tensor, gamma: torch.Tensor,
                       mean: torch.Tensor, rstd: torch.Tensor, *, dres=None,
                       weights: bool = True, want_dbeta: bool = True, dx=None, dgamma=None,
                       dbeta=None, ws=None):
    """Backward of moe_layer_norm: s, mean and rstd as it returned them, ``dres``
    [T, d] the gradient that reaches s past the norm.  ``weights=False`` skips
    dgamma and dbeta.  ``dx`` may be dy or dres.  Returns (dx, dgamma, dbeta),
    None for what was not computed."""
    _dev(s, "s")
    T, d = s.shape
    dev = s.device
    f32 = torch.float32
    _want(dy, "dy", (T, d), s.dtype), _want(dres, "dres", (T, d), s.dtype)
    _want(gamma, "gamma", (d,), f32)
    _want(mean, "mean", (T,), f32), _want(rstd, "rstd", (T,), f32)
    code = _dtype_code(s)
    dx = _out(dx, "dx", (T, d), s.dtype, dev)
    dgamma = _out(dgamma, "dgamma", (d,), f32, dev) if weights else None
    dbeta = _out(dbeta, "dbeta", (d,), f32, dev) if weights and want_dbeta else None
    if weights:
        ws = _given_ws(ws, dev, LAEP_CALL_LAYER_NORM_BWD, T, 1, 1, d)
    check(lib().moe_layer_norm_bwd(_ptr(dy), _ptr(s), _ptr(gamma), _ptr(mean), _ptr(rstd),
                                   _ptr(dres), code, T, d, _ptr(dx), _ptr(dgamma), _ptr(dbeta),
                                   _ptr(ws) if weights else None,
                                   ws.numel() * ws.element_size() if weights else 0,
                                   _stream(dev)))
    return dx, dgamma, dbeta


def _sequences(seq_offsets) -> int:
    if seq_offsets is None:
        return 1
    if seq_offsets.dtype != torch.int32 or seq_offsets.dim() != 1 or seq_offsets.numel() < 2:
        raise ValueError("seq_offsets must be an int32 tensor [n_seq + 1]")
    _dev(seq_offsets, "seq_offsets")
    return seq_offsets.numel() - 1


def _given_ws(ws, device, which, *sizes):
    """The given workspace (its size is the C call's to check) or a new one."""
    if ws is None:
        return torch.empty(max(workspace_bytes(which, *sizes), 1), dtype=torch.uint8,
                           device=device)
    return _dev(ws, "ws")


def _scalar(t, name: str):
    if t is not None and (t.dtype is not torch.float32 or t.numel() != 1 or not t.is_cuda):
        raise ValueError(f"{name} must be a float32 device tensor of one element")


def moe_balance_loss(logits: torch.Tensor, topk_idx: torch.Tensor, *, coef: float = 1.0,
                     alive=None, seq_offsets=None, loss=None, counts=None, prob_mean=None,
                     grad_coef=None, ws=None):
    """Balance loss of the router's float32 logits [T, E] and its selection
    topk_idx [T, k], over the batch or per sequence (``seq_offsets`` int32
    [n_seq + 1] on the device).  Returns (loss [1], counts [n_seq, E] int32,
    prob_mean [n_seq, E], grad_coef [n_seq, E]); grad_coef goes to
    moe_balance_loss_bwd or moe_route_bwd_balance."""
    _dev(logits, "logits")
    T, E = logits.shape
    k = topk_idx.shape[1]
    dev = logits.device
    f32 = torch.float32
    _want(logits, "logits", (T, E), f32), _want(topk_idx, "topk_idx", (T, k), torch.int32)
    _want(alive, "alive", (E,), torch.uint8)
    S = _sequences(seq_offsets)
    loss = _out(loss, "loss", (1,), f32, dev)
    counts = _out(counts, "counts", (S, E), torch.int32, dev)
    prob_mean = _out(prob_mean, "prob_mean", (S, E), f32, dev)
    grad_coef = _out(grad_coef, "grad_coef", (S, E), f32, dev)
    ws = _given_ws(ws, dev, LAEP_CALL_BALANCE, T, S, E)
    check(lib().moe_balance_loss(_ptr(logits), _ptr(topk_idx), _ptr(alive), _ptr(seq_offsets), T,
                                 E, k, S, float(coef), _ptr(loss), _ptr(counts), _ptr(prob_mean),
                                 _ptr(grad_coef), _ptr(ws), ws.numel() * ws.element_size(),
                                 _stream(dev)))
    return loss, counts, prob_mean, grad_coef


def moe_balance_loss_bwd(logits: torch.Tensor, grad_coef: torch.Tensor, *, dloss=None,
                         alive=None, seq_offsets=None, dlogits=None, accumulate: bool = False):
    """Gradient of the balance loss with respect to the logits, the counts held
    fixed; ``dloss`` is a float32 device tensor of one element (None: 1).
    ``accumulate`` adds to the given dlogits, which must then not be the logits'
    buffer (it may be otherwise)."""
    _dev(logits, "logits")
    T, E = logits.shape
    S = _sequences(seq_offsets)
    f32 = torch.float32
    _want(logits, "logits", (T, E), f32), _want(grad_coef, "grad_coef", (S, E), f32)
    _want(alive, "alive", (E,), torch.uint8)
    _scalar(dloss, "dloss")
    if accumulate and dlogits is None:
        raise ValueError("accumulate needs dlogits")
    dlogits = _out(dlogits, "dlogits", (T, E), f32, logits.device)
    check(lib().moe_balance_loss_bwd(_ptr(logits), _ptr(grad_coef), _ptr(alive),
                                     _ptr(seq_offsets), _ptr(dloss), T, E, S, _ptr(dlogits),
                                     int(accumulate), _stream(logits.device)))
    return dlogits


def moe_route_bwd_balance(dgate: torch.Tensor, topk_idx: torch.Tensor, topk_gate: torch.Tensor,
                          logits: torch.Tensor, x: torch.Tensor, w_router: torch.Tensor,
                          grad_coef: torch.Tensor, *, seq_offsets=None, dloss=None,
                          renorm: bool = True, alive=None, dx=None, accumulate_dx: bool = False,
                          want_dlogits: bool = False, want_dbias: bool = False, dw_router=None,
                          dlogits=None, dbias=None, ws=None, data: bool = True,
                          weights: bool = True):
    """moe_route_bwd with the balance loss's gradient (moe_balance_loss's
    grad_coef) added to the gates' before the products.  ``dlogits`` must not be the
    logits' buffer.  Returns as moe_route_bwd."""
    T, k = topk_idx.shape
    E, d = w_router.shape
    dev = x.device
    f32 = torch.float32
    S = _sequences(seq_offsets)
    _want(dgate, "dgate", (T, k), f32), _want(topk_gate, "topk_gate", (T, k), f32)
    _want(topk_idx, "topk_idx", (T, k), torch.int32)
    _want(x, "x", (T, d), x.dtype), _want(w_router, "w_router", (E, d), x.dtype)
    _want(logits, "logits", (T, E), f32), _want(grad_coef, "grad_coef", (S, E), f32)
    _want(alive, "alive", (E,), torch.uint8)
    _scalar(dloss, "dloss")
    if not data:
        dx = None
    elif dx is None and accumulate_dx:
        dx = torch.zeros_like(x)
    else:   # overwritten whole unless accumulated onto
        dx = _out(dx, "dx", (T, d), x.dtype, dev)
    if weights:
        dw_router = _out(dw_router, "dw_router", (E, d), f32, dev)
        if want_dbias or dbias is not None:
            dbias = _out(dbias, "dbias", (E,), f32, dev)
    else:
        dw_router, dbias = None, None
    if want_dlogits or dlogits is not None:
        dlogits = _out(dlogits, "dlogits", (T, E), f32, dev)
    ws = _given_ws(ws, dev, LAEP_CALL_ROUTE_BWD, T, k, E, d)
    check(lib().moe_route_bwd_balance(
        _ptr(dgate), _ptr(topk_idx), _ptr(topk_gate), _ptr(logits), _ptr(alive), _ptr(x),
        _ptr(w_router), _ptr(grad_coef), _ptr(seq_offsets), S, _ptr(dloss), _dtype_code(x), T, d,
        E, k, int(renorm), _ptr(dlogits), _ptr(dw_router), _ptr(dbias), _ptr(dx),
        int(accumulate_dx), _ptr(ws), ws.numel() * ws.element_size(), _stream(dev)))
    return dx, dw_router, dbias, dlogits


def moe_act8_save(act: torch.Tensor, *, q=None, scale=None):
    """act [R, C] (C a multiple of 32) in 8 bits with one power-of-two scale per
    32 columns of a row.  Returns (q [R, C] int8, scale [R, C/32] uint8, the
    scale's biased exponent)."""
    _dev(act, "act")
    R, C = act.shape
    q = _out(q, "q", (R, C), torch.int8, act.device)
    scale = _out(scale, "scale", (R, C // LAEP_ACT8_BLOCK), torch.uint8, act.device)
    check(lib().moe_act8_save(_ptr(act), _dtype_code(act), R, C, _ptr(q), _ptr(scale),
                              _stream(act.device)))
    return q, scale


def moe_act8_load(q: torch.Tensor, scale: torch.Tensor, dtype: torch.dtype = torch.bfloat16, *,
                  out=None):
    """The values an 8-bit checkpoint stands for, in dtype (exact in bfloat16)."""
    _dev(q, "q")
    R, C = q.shape
    _want(q, "q", (R, C), torch.int8)
    _want(scale, "scale", (R, C // LAEP_ACT8_BLOCK), torch.uint8)
    if dtype not in _DT:
        raise LaepError(2, f"unsupported dtype {dtype}")
    out = _out(out, "out", (R, C), dtype, q.device)
    check(lib().moe_act8_load(_ptr(q), _ptr(scale), _DT[dtype], R, C, _ptr(out),
                              _stream(q.device)))
    return out


def moe_swiglu_bwd_act8(q: torch.Tensor, scale: torch.Tensor, dh: torch.Tensor, *, da=None,
                        h=None):
    """SwiGLU backward at pre-activations kept in 8 bits (q [R, 2f], scale
    [R, 2f/32]) from dh [R, f].  Returns (da [R, 2f], h [R, f]); h is the
    recomputed input of the down projection and may be dh's buffer."""
    _dev(dh, "dh")
    R, f = dh.shape
    _want(q, "q", (R, 2 * f), torch.int8)
    _want(scale, "scale", (R, 2 * f // LAEP_ACT8_BLOCK), torch.uint8)
    da = _out(da, "da", (R, 2 * f), dh.dtype, dh.device)
    h = _out(h, "h", (R, f), dh.dtype, dh.device)
    check(lib().moe_swiglu_bwd_act8(_ptr(q), _ptr(scale), _ptr(dh), _dtype_code(dh), R, f,
                                    _ptr(da), _ptr(h), _stream(dh.device)))
    return da, h


def moe_grouped_ffn_bwd_gather_act8(dy_perm, x, row_src, k: int, act_q, act_scale, w_gate_up,
                                    w_down, offsets, *, dout=None, topk_gate=None,
                                    expert_map=None, dw_gate_up=None, dw_down=None,
                                    accumulate=False, ws=None, dx_perm=None,
                                    return_ws: bool = False):
    """moe_grouped_ffn_bwd_gather at pre-activations kept in 8 bits (act_q [R, 2f],
    act_scale [R, 2f/32]); dW_d takes the H recomputed there.  Returns as
    moe_grouped_ffn_bwd."""
    _dev(x, "x")
    T, d = x.shape
    R = row_src.shape[0]
    n, _, f = w_down.shape
    E = offsets.shape[0] - 1
    dev = x.device
    f32, i32 = torch.float32, torch.int32
    if dy_perm is None:
        if dout is None or topk_gate is None:
            raise ValueError("without dy_perm, dout and topk_gate are needed")
        _want(dout, "dout", (T, d), x.dtype), _want(topk_gate, "topk_gate", (T, k), f32)
    else:
        _want(dy_perm, "dy_perm", (R, d), x.dtype)
    _want(row_src, "row_src", (R,), i32), _want(offsets, "offsets", (E + 1,), i32)
    _want(expert_map, "expert_map", (E,), i32)
    _want(w_gate_up, "w_gate_up", (n, 2 * f, d), x.dtype)
    _want(w_down, "w_down", (n, d, f), x.dtype)
    _want(act_q, "act_q", (R, 2 * f), torch.int8)
    _want(act_scale, "act_scale", (R, 2 * f // LAEP_ACT8_BLOCK), torch.uint8)
    dx_perm = _out(dx_perm, "dx_perm", (R, d), x.dtype, dev)
    dw_gate_up = _out(dw_gate_up, "dw_gate_up", w_gate_up.shape, f32, dev)
    dw_down = _out(dw_down, "dw_down", w_down.shape, f32, dev)
    ws = _given_ws(ws, dev, LAEP_CALL_FFN_BWD, R, 1, E, d, f)
    check(lib().moe_grouped_ffn_bwd_gather_act8(
        _ptr(dy_perm), _ptr(dout), _ptr(topk_gate), _ptr(x), _ptr(row_src), T, k, _ptr(act_q),
        _ptr(act_scale), _ptr(w_gate_up), _ptr(w_down), _ptr(offsets), _ptr(expert_map),
        _dtype_code(x), E, d, f, R, _ptr(dx_perm), _ptr(dw_gate_up), _ptr(dw_down),
        int(accumulate), _ptr(ws), ws.numel() * ws.element_size(), _stream(dev)))
    out = (dx_perm, dw_gate_up, dw_down)
    return out + (ws,) if return_ws else out


# ---- experts in microscaled 4 bits (laep_mx4.h) ----------------------------------------
class Mx4(NamedTuple):
    """A matrix [..., R, C] in microscaled 4 bits, as moe_mx4_quantize writes it: codes
    uint8 [..., R, C / 2], scale uint8 [..., ceil(C / 256), R, 8]."""
    codes: torch.Tensor
    scale: torch.Tensor


# (The checks of a small call cost as much as its kernels, so the code below makes one pass
# over the attributes while all is well, and calls little: 0.6 us of a product's 8.6.)
def _need(t, name: str, shape, dtype, device):
    """A given tensor of this shape, dtype and device."""
    if not (t.shape == shape and t.dtype is dtype and t.get_device() == device.index
            and t.is_contiguous()):
        _want(t, name, shape, dtype)
        raise ValueError(f"{name} is on {t.device}, not {device}")


def _need_out(t, name: str, shape, dtype, device):
    """The given output buffer, checked, or a new one."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not (t.shape == shape and t.dtype is dtype and t.get_device() == device.index
            and t.is_contiguous()):
        _need(t, name, shape, dtype, device)
    return t


def _need_ws(ws, device, which, *sizes):
    """The given workspace (its size is the C call's to check) or a new one."""
    if ws is None:
        return _given_ws(None, device, which, *sizes)
    if ws.get_device() != device.index or not ws.is_contiguous():
        _dev(ws, "ws")
        raise ValueError(f"ws is on {ws.device}, not {device}")
    return ws


def _need_mx4(w, name: str, lead, R: int, C: int, device):
    """A given Mx4 [*lead, R, C]."""
    if not isinstance(w, Mx4):
        raise ValueError(f"{name} must be an Mx4 (moe_mx4_quantize's codes and scale)")
    codes, scale = w
    u8, index = torch.uint8, device.index
    if not (codes.shape == lead + (R, C // 2) and codes.dtype is u8
            and scale.shape == lead + (-(-C // LAEP_MX4_GROUP), R, 8) and scale.dtype is u8
            and codes.get_device() == index and scale.get_device() == index
            and codes.is_contiguous() and scale.is_contiguous()):
        _need(codes, f"{name}.codes", lead + (R, C // 2), u8, device)
        _need(scale, f"{name}.scale", lead + (-(-C // LAEP_MX4_GROUP), R, 8), u8, device)


_INT_MAX = 0x7FFFFFFF   # (ctypes passes a larger number's low 32 bits as a C int)


def _too_large(**sizes):
    name, n = max(sizes.items(), key=lambda kv: kv[1])
    raise ValueError(f"{name}={n} is past the C calls' 2^31 - 1")


def _on_device(device, fn, *args):
    """check(fn(*args, stream)) with the tensors' device current: the C calls launch there."""
    index = device.index
    if torch._C._cuda_getDevice() == index:
        check(fn(*args, torch._C._cuda_getCurrentRawStream(index)))
    else:
        with torch.cuda.device(device):
            check(fn(*args, torch._C._cuda_getCurrentRawStream(index)))


def moe_mx4_quantize(src: torch.Tensor, *, codes=None, scale=None) -> Mx4:
    """The matrices src [..., R, C] (bf16 or float32, C a multiple of 32) in
    microscaled 4 bits: every 32 columns of a row share a power-of-two scale."""
    _dev(src, "src")
    shape = tuple(src.shape)
    if len(shape) < 2:
        raise ValueError("src must have rows and columns")
    lead, R, C = shape[:-2], shape[-2], shape[-1]
    n = math.prod(lead)
    if n > _INT_MAX or C > _INT_MAX:
        _too_large(matrices=n, columns=C)
    dev = src.device
    code = _dtype_code(src)
    codes = _need_out(codes, "codes", lead + (R, C // 2), torch.uint8, dev)
    scale = _need_out(scale, "scale", lead + (-(-C // LAEP_MX4_GROUP), R, 8), torch.uint8, dev)
    _on_device(dev, lib().moe_mx4_quantize, src.data_ptr(), code, n, R, C,
               codes.data_ptr(), scale.data_ptr())
    return Mx4(codes, scale)


def moe_mx4_dequantize(codes: torch.Tensor, scale: torch.Tensor,
                       dtype: torch.dtype = torch.bfloat16, *, out=None):
    """The values [..., R, C] that codes and scale stand for, in dtype (exact, if they are
    moe_mx4_quantize's; infinities where a larger scale leaves float32's range)."""
    _dev(codes, "codes")
    shape = tuple(codes.shape)
    if len(shape) < 2:
        raise ValueError("codes must have rows and columns")
    lead, R, C = shape[:-2], shape[-2], 2 * shape[-1]
    n = math.prod(lead)
    if n > _INT_MAX or C > _INT_MAX:
        _too_large(matrices=n, columns=C)
    dev = codes.device
    if dtype not in _DT:
        raise LaepError(2, f"unsupported dtype {dtype}")
    _need(codes, "codes", shape, torch.uint8, dev)
    _need(scale, "scale", lead + (-(-C // LAEP_MX4_GROUP), R, 8), torch.uint8, dev)
    out = _need_out(out, "out", lead + (R, C), dtype, dev)
    _on_device(dev, lib().moe_mx4_dequantize, codes.data_ptr(), scale.data_ptr(), _DT[dtype],
               n, R, C, out.data_ptr())
    return out


def _mx4_routing(dev, T: int, k: int, offsets, row_src, expert_map, slots: int):
    """Checks of the routing's tensors.  Returns (E, R, k as the C calls take it)."""
    i32, index = torch.int32, dev.index
    E = offsets.numel() - 1
    if E < 1 or offsets.dim() != 1:
        raise ValueError("offsets must be an int32 tensor [E + 1]")
    if not (offsets.dtype is i32 and offsets.get_device() == index and offsets.is_contiguous()):
        _need(offsets, "offsets", (E + 1,), i32, dev)
    if expert_map is not None:
        _need(expert_map, "expert_map", (E,), torch.int32, dev)
    elif slots != E:
        raise ValueError(f"{slots} weight slots for {E} experts need an expert_map")
    if row_src is None:
        return E, T, 1
    R = row_src.numel()
    if not (row_src.dim() == 1 and row_src.dtype is i32 and row_src.get_device() == index
            and row_src.is_contiguous()):
        _need(row_src, "row_src", (R,), i32, dev)
    return E, R, k


def moe_mx4_grouped_product(x, w: Mx4, offsets: torch.Tensor, *, row_src=None, k: int = 1,
                            expert_map=None, dtype: torch.dtype = torch.bfloat16, out=None,
                            ws=None):
    """Routed rows times their expert's matrix: out [R, N] in dtype, out[r] =
    x[row_src[r] // k] @ W[slot].T.  x [T, K] is an Mx4 or bf16; w an Mx4 of [slots, N,
    K] (N, K multiples of 64); without row_src x's rows are already in the experts'
    order.  Rows of experts with a negative expert_map entry are left as they were."""
    mx4 = isinstance(x, Mx4)
    rows = x[0] if mx4 else x
    _dev(rows, "x")
    if rows.dim() != 2 or not isinstance(w, Mx4) or w[0].dim() != 3:
        raise ValueError("x must be a matrix [T, K], w an Mx4 of [slots, N, K]")
    dev = rows.device
    T, K = rows.shape
    slots, N, _ = w[0].shape
    if mx4:
        K *= 2
    if T > _INT_MAX or K > _INT_MAX or N > _INT_MAX or k > _INT_MAX:
        _too_large(T=T, K=K, N=N, k=k)
    if mx4:
        _need_mx4(x, "x", (), T, K, dev)
    else:
        _need(x, "x", (T, K), torch.bfloat16, dev)
    _need_mx4(w, "w", (slots,), N, K, dev)
    if dtype not in _DT:
        raise LaepError(2, f"unsupported dtype {dtype}")
    E, R, k = _mx4_routing(dev, T, k, offsets, row_src, expert_map, slots)
    out = _need_out(out, "out", (R, N), dtype, dev)
    ws = _need_ws(ws, dev, LAEP_CALL_MX4_PRODUCT, T, k, E, K, N)
    _on_device(dev, lib().moe_mx4_grouped_product, rows.data_ptr(),
               x[1].data_ptr() if mx4 else None, _ptr(row_src), T, k, w[0].data_ptr(),
               w[1].data_ptr(), offsets.data_ptr(), _ptr(expert_map), _DT[dtype], E, N, K, R,
               out.data_ptr(), ws.data_ptr(), ws.nbytes)
    return out


def moe_grouped_ffn_fwd_mx4(x: torch.Tensor, w_gate_up: Mx4, w_down: Mx4,
                            offsets: torch.Tensor, *, row_src=None, k: int = 1,
                            act_bits: int = 16, expert_map=None, save_act: bool = False,
                            act_save=None, y_perm=None, ws=None):
    """The grouped SwiGLU FFN at weights in microscaled 4 bits (Mx4 of [slots, 2f, d] and
    [slots, d, f]) over the bf16 tokens x [T, d], routed row r reading token
    row_src[r] // k (without row_src: row r).  ``act_bits`` 16 keeps X and H in bf16, 4
    rounds both to MX4.  ``save_act`` (act_bits 16) keeps the pre-activations for
    moe_grouped_ffn_bwd_gather at moe_mx4_dequantize of the weights.  Returns (y_perm
    [R, d], act_save [R, 2f] or None)."""
    _dev(x, "x")
    if x.dim() != 2 or not isinstance(w_gate_up, Mx4) or not isinstance(w_down, Mx4) or \
            w_down[0].dim() != 3:
        raise ValueError("x must be a matrix [T, d], the weights Mx4 of [slots, ., .]")
    dev = x.device
    T, d = x.shape
    slots, _, f = w_down[0].shape
    f *= 2
    if T > _INT_MAX or d > _INT_MAX or f > _INT_MAX or k > _INT_MAX:
        _too_large(T=T, d=d, f=f, k=k)
    _need(x, "x", (T, d), torch.bfloat16, dev)
    _need_mx4(w_gate_up, "w_gate_up", (slots,), 2 * f, d, dev)
    _need_mx4(w_down, "w_down", (slots,), d, f, dev)
    E, R, k = _mx4_routing(dev, T, k, offsets, row_src, expert_map, slots)
    y_perm = _need_out(y_perm, "y_perm", (R, d), torch.bfloat16, dev)
    if save_act or act_save is not None:
        act_save = _need_out(act_save, "act_save", (R, 2 * f), torch.bfloat16, dev)
    ws = _need_ws(ws, dev, LAEP_CALL_MX4_FFN, T, k, E, d, f)
    _on_device(dev, lib().moe_grouped_ffn_fwd_mx4, x.data_ptr(), _ptr(row_src), T, k,
               w_gate_up[0].data_ptr(), w_gate_up[1].data_ptr(), w_down[0].data_ptr(),
               w_down[1].data_ptr(), offsets.data_ptr(), _ptr(expert_map), int(act_bits), E, d, f,
               R, y_perm.data_ptr(), _ptr(act_save), ws.data_ptr(), ws.nbytes)
    return y_perm, act_save


# ---- measurement calls (laep_calib.h) -------------------------------------------------
def laep_calib_copy(src: torch.Tensor, dst: torch.Tensor):
    """dst <- src (raw bytes) with the library's streaming copy kernel."""
    _dev(src, "src")
    _dev(dst, "dst")
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() < nbytes:
        raise ValueError("dst is smaller than src")
    check(lib().laep_calib_copy(_ptr(src), _ptr(dst), nbytes, _stream(src.device)))


def laep_calib_read(src: torch.Tensor, block_bytes: int, out: torch.Tensor):
    """Blocked streaming read of src (laep_calib_read): one 512-thread
    workgroup per block_bytes, out float32 [n_blocks * 512]."""
    _dev(src, "src")
    _dev(out, "out")
    nbytes = src.numel() * src.element_size()
    if block_bytes <= 0 or out.dtype != torch.float32 or \
            out.numel() < (nbytes // block_bytes) * 512:
        raise ValueError("out must be float32 with (src bytes / block_bytes) * 512 elements")
    check(lib().laep_calib_read(_ptr(src), nbytes, int(block_bytes), _ptr(out),
                                _stream(src.device)))


def laep_calib_mfma(n_workgroups: int, iters: int, out: torch.Tensor):
    """bf16 MFMA loop: n_workgroups x 8 waves x iters x 8 MFMA 32x32x16."""
    _dev(out, "out")
    if out.dtype != torch.float32 or out.numel() < n_workgroups * 512:
        raise ValueError("out must be float32 with n_workgroups * 512 elements")
    check(lib().laep_calib_mfma(n_workgroups, iters, _ptr(out), _stream(out.device)))


def laep_ffn_fwd_row_tile(R: int, E: int, d_model: int, d_ff: int) -> int:
    """Rows per tile (32, 64, 128 or 256) of the bf16 forward FFN at these sizes."""
    return int(lib().laep_ffn_fwd_row_tile(int(R), int(E), int(d_model), int(d_ff)))


def laep_mx4_product_tile(R: int, E: int, N: int, K: int, act_bits: int = 16) -> tuple:
    """(rows, columns) of the tiles of moe_mx4_grouped_product for R = T k rows (T without
    row_src); (0, 0) for sizes that it refuses."""
    cols = ctypes.c_int(0)
    rows = lib().laep_mx4_product_tile(int(R), int(E), int(N), int(K), int(act_bits),
                                       ctypes.byref(cols))
    return int(rows), cols.value


def laep_mx4_ffn_tile(R: int, E: int, d_model: int, d_ff: int, act_bits: int = 16,
                      down: bool = False) -> tuple:
    """(rows, columns) of the tiles of moe_grouped_ffn_fwd_mx4's gate/up or down product,
    likewise."""
    cols = ctypes.c_int(0)
    rows = lib().laep_mx4_ffn_tile(int(R), int(E), int(d_model), int(d_ff), int(act_bits),
                                   int(down), ctypes.byref(cols))
    return int(rows), cols.value

"""One MoE layer pass as a fixed chain of C-ABI calls on preallocated buffers.

Forward (router path):
    moe_route -> moe_expert_counts
      [-> laep_prune_mask -> moe_route(alive) -> moe_expert_counts]   (pruning)
    -> moe_permute -> moe_grouped_ffn_fwd -> moe_combine
Forward (given routing, one device's expert shard with k = 1):
    moe_expert_counts -> moe_permute -> moe_grouped_ffn_fwd -> moe_combine
With fused dispatch (bf16, the default), moe_permute + moe_grouped_ffn_fwd
become one moe_grouped_ffn_fwd_gather call that reads the token rows through
row_src, and the backward reads them the same way
(moe_grouped_ffn_bwd_gather), so a training step never writes x_perm.
dY = g * dout is written once by moe_combine_bwd, into a buffer of the plan's
own: every column block of two products reads it, and scaling it again in each
of them costs more than the one pass.  A forward that keeps its activations
for inspection (save_act without a backward) still writes x_perm.
With one slot per token (k = 1) the combine folds in as well
(moe_grouped_ffn_fwd_gather_combine): the down projection writes each row,
times its gate, to its token row; y_perm is written only for a backward pass.
Backward:
    moe_combine_bwd -> moe_grouped_ffn_bwd[_gather] -> moe_permute_bwd
      [-> moe_route_bwd, accumulating the router's dx]   (router path)
In a training step the router's weight gradients need only the gate gradient:
backward(router=...) runs them on a side stream beside the expert backward and
takes the router's dx after moe_permute_bwd.
With act_bits=8 the pre-activations that a training step keeps are stored in 8
bits (moe_act8_save) and the backward reads those
(moe_grouped_ffn_bwd_gather_act8): 2.06 d_ff bytes a routed row are kept instead
of the 6 d_ff of act_save and H, which become scratch that plans run one after
the other can share (``scratch``).
With mx4_act=4 or 16 the expert weights are in microscaled 4 bits (api.Mx4, serving):
moe_grouped_ffn_fwd_mx4, with activations in 4 or 16 bits, then moe_combine.

All buffers are allocated once, so a pass makes no allocation and no host
synchronisation; every step runs in the library's kernels on the current
stream.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import api
from ._lib import (LAEP_ACT8_BLOCK, LAEP_CALL_COUNTS, LAEP_CALL_FFN_BWD, LAEP_CALL_FFN_FWD,
                   LAEP_CALL_MX4_FFN, LAEP_CALL_ROUTE_BWD)


class MoELayerPlan:
    def __init__(self, T: int, d_model: int, E: int, k: int, d_ff: int,
                 dtype: torch.dtype = torch.bfloat16, device="cuda", backward: bool = False,
                 save_act: Optional[bool] = None, fused_dispatch: Optional[bool] = None,
                 act_bits: int = 16, scratch: Optional["MoELayerPlan"] = None,
                 mx4_act: Optional[int] = None):
        """``act_bits`` 8: a training plan (bf16, fused dispatch) keeps its
        pre-activations in 8 bits.  ``mx4_act`` 4 or 16: a plan without a backward (bf16,
        fused dispatch) whose expert weights are api.Mx4, with activations in that many
        bits.  ``scratch``: a plan of the same sizes and kind
        whose transient buffers this one uses too; their forward and backward
        passes must not overlap."""
        self.T, self.d, self.E, self.k, self.f = T, d_model, E, k, d_ff
        self.R = T * k
        self.dtype = dtype
        dev = torch.device(device)
        self.device = dev
        i32 = torch.int32
        R = self.R
        self.topk_idx = torch.empty((T, k), dtype=i32, device=dev)
        self.topk_gate = torch.empty((T, k), dtype=torch.float32, device=dev)
        self.counts = torch.empty(E, dtype=i32, device=dev)
        self.offsets = torch.empty(E + 1, dtype=i32, device=dev)
        self.dest_row = torch.empty(R, dtype=i32, device=dev)
        self.alive = torch.empty(E, dtype=torch.uint8, device=dev)
        self.n_pruned = torch.empty(1, dtype=i32, device=dev)
        # pre-activations are kept when a backward pass will read them (or on request)
        save_act = backward if save_act is None else save_act
        # the dispatch folds into the FFN's operand loads (bf16), forward and
        # backward; x_perm is kept only unfused, or for a forward that keeps its
        # activations without a backward (inspection)
        if fused_dispatch is None:
            fused_dispatch = dtype == torch.bfloat16
        self.fused = bool(fused_dispatch)
        if act_bits not in (8, 16):
            raise ValueError(f"act_bits={act_bits} is neither 8 nor 16")
        if act_bits == 8 and not (backward and save_act and self.fused):
            raise ValueError("act_bits=8 needs a training plan with the fused dispatch (bf16)")
        self.act_bits = act_bits
        if mx4_act not in (None, 4, 16):
            raise ValueError(f"mx4_act={mx4_act} is neither 4 nor 16")
        if mx4_act is not None and (backward or save_act or not self.fused):
            raise ValueError("mx4_act needs a plan without a backward pass or kept "
                             "activations, with the fused dispatch (bf16)")
        self.mx4_act = mx4_act
        kind = (T, d_model, E, k, d_ff, dtype, dev, backward, self.fused, act_bits, mx4_act)
        if scratch is not None and scratch.kind != kind:
            raise ValueError("scratch must be a plan of the same sizes and kind")
        self.kind = kind
        self.x_perm = (None if self.fused and (backward or not save_act) else
                       torch.empty((R, d_model), dtype=dtype, device=dev))
        self.x_in = None   # the token rows of the last forward (the gathered backward reads them)
        # the dispatch order is kept when the FFN gathers through it or the
        # router backward sums dW_r over it
        self.row_src = (torch.empty(R, dtype=i32, device=dev) if self.fused or backward
                        else None)
        # one slot per token (bf16): the combine folds into the down projection's
        # epilogue; y_perm is then written only for the backward (combine_bwd) or
        # when the caller keeps the activations (save_act)
        self.fused_combine = k == 1 and self.fused and mx4_act is None
        self.y_perm = (None if self.fused_combine and not (backward or save_act) else
                       torch.empty((R, d_model), dtype=dtype, device=dev))
        if scratch is not None and act_bits == 8:   # transient: decoded into 8 bits at once
            self.act_save = scratch.act_save
        else:
            self.act_save = (torch.empty((R, 2 * d_ff), dtype=dtype, device=dev) if save_act
                             else None)
        if act_bits == 8:
            self.act_q = torch.empty((R, 2 * d_ff), dtype=torch.int8, device=dev)
            self.act_scale = torch.empty((R, 2 * d_ff // LAEP_ACT8_BLOCK), dtype=torch.uint8,
                                         device=dev)
        self.out = torch.empty((T, d_model), dtype=dtype, device=dev)
        if scratch is not None:
            self.ws_counts = scratch.ws_counts
        else:
            self.ws_counts = torch.empty(max(1, api.workspace_bytes(LAEP_CALL_COUNTS, T, k, E)),
                                         dtype=torch.uint8, device=dev)
        # (a 16-bit training plan's H stays in ws_ffn for its backward)
        if scratch is not None and (act_bits == 8 or not backward):
            self.ws_ffn = scratch.ws_ffn
        else:
            self.ws_ffn = torch.empty(
                max(1, api.workspace_bytes(LAEP_CALL_MX4_FFN, T, k, E, d_model, d_ff))
                if mx4_act is not None else
                api.workspace_bytes(LAEP_CALL_FFN_FWD, R, 1, E, d_model, d_ff),
                dtype=torch.uint8, device=dev)
        if backward:
            # dY of a fused plan: written by the combine backward, read by the data
            # gradient and dW_d of the same call (formed on load by both instead,
            # each column block scaling its rows again, the training step of 8192
            # tokens, top-8, d 2048, d_ff 1024 takes 3.12 ms against 3.03, that of
            # 32768 rows, d 4096, d_ff 2048 5.29 against 5.06)
            if scratch is not None:
                self._dy, self.dx_perm, self.ws_bwd = scratch._dy, scratch.dx_perm, scratch.ws_bwd
                self.ws_route_bwd = scratch.ws_route_bwd
                self.ws_route_bwd_w = scratch.ws_route_bwd_w
            else:
                self._dy = torch.empty((R, d_model), dtype=dtype, device=dev)
                self.dx_perm = torch.empty((R, d_model), dtype=dtype, device=dev)
                self.ws_bwd = torch.empty(
                    api.workspace_bytes(LAEP_CALL_FFN_BWD, R, 1, E, d_model, d_ff),
                    dtype=torch.uint8, device=dev)
                rb = max(1, api.workspace_bytes(LAEP_CALL_ROUTE_BWD, T, k, E, d_model))
                self.ws_route_bwd = torch.empty(rb, dtype=torch.uint8, device=dev)
                # the router's weight gradients run on a side stream beside the expert
                # backward, with a workspace of their own
                self.ws_route_bwd_w = torch.empty(rb, dtype=torch.uint8, device=dev)
            self.dy_perm = None if self.fused else self._dy
            self.dgate = torch.empty((T, k), dtype=torch.float32, device=dev)
            self.dx = torch.empty((T, d_model), dtype=dtype, device=dev)
            self.dw_gate_up = None
            self.dw_down = None
            self.dw_router = None
            self.dbias = None
            self._side = None
            self._side_done = None

    # -- pieces --------------------------------------------------------------
    def route(self, x, w_router, bias=None, alive=None, renorm=True):
        api.moe_route(x, w_router, self.k, bias=bias, alive=alive, renorm=renorm,
                      topk_idx=self.topk_idx, topk_gate=self.topk_gate)

    def count(self, etn_accum=None):
        api.moe_expert_counts(self.topk_idx, self.E, ws=self.ws_counts, counts=self.counts,
                              offsets=self.offsets, dest_row=self.dest_row,
                              row_src=self.row_src, etn_accum=etn_accum)

    def route_count(self, x, w_router, bias=None, alive=None, renorm=True, etn_accum=None):
        """route + count in one call (the router also writes the count masks)."""
        api.moe_route_count(x, w_router, self.k, bias=bias, alive=alive, renorm=renorm,
                            etn_accum=etn_accum, ws=self.ws_counts, topk_idx=self.topk_idx,
                            topk_gate=self.topk_gate, counts=self.counts, offsets=self.offsets,
                            dest_row=self.dest_row, row_src=self.row_src)

    def prune(self, beta: float, alpha: float = math.inf):
        api.laep_prune_mask(self.counts, self.T * self.k, alpha, beta, alive=self.alive,
                            n_pruned=self.n_pruned)

    def experts_and_combine(self, x, w_gate_up, w_down, expert_map=None):
        for w in (w_gate_up, w_down):
            if isinstance(w, api.Mx4) != (self.mx4_act is not None):
                raise ValueError("expert weights are Mx4 where the plan has mx4_act, and only there")
        self.x_in = x
        if self.mx4_act is not None:
            api.moe_grouped_ffn_fwd_mx4(x, w_gate_up, w_down, self.offsets, row_src=self.row_src,
                                        k=self.k, act_bits=self.mx4_act, expert_map=expert_map,
                                        ws=self.ws_ffn, y_perm=self.y_perm)
            api.moe_combine(self.y_perm, self.topk_gate, self.dest_row, out=self.out)
            return self.out
        if self.fused_combine:
            api.moe_grouped_ffn_fwd_gather_combine(
                x, self.row_src, self.topk_gate, w_gate_up, w_down, self.offsets, rows=self.R,
                expert_map=expert_map, ws=self.ws_ffn, out=self.out,
                keep_y=self.y_perm is not None, y_perm=self.y_perm,
                save_act=self.act_save is not None, act_save=self.act_save,
                x_perm_out=self.x_perm)
            self._keep_act()
            return self.out
        if self.fused:
            # x_perm (kept for inspection only) by the token-major permute, which
            # reads each token row once
            if self.x_perm is not None:
                api.moe_permute(x, self.dest_row, self.k, self.R, out=self.x_perm)
            api.moe_grouped_ffn_fwd_gather(x, self.row_src, self.k, w_gate_up, w_down,
                                           self.offsets, rows=self.R, expert_map=expert_map,
                                           ws=self.ws_ffn, y_perm=self.y_perm,
                                           save_act=self.act_save is not None,
                                           act_save=self.act_save)
        else:
            api.moe_permute(x, self.dest_row, self.k, self.R, out=self.x_perm)
            api.moe_grouped_ffn_fwd(self.x_perm, w_gate_up, w_down, self.offsets,
                                    expert_map=expert_map, ws=self.ws_ffn, y_perm=self.y_perm,
                                    save_act=self.act_save is not None, act_save=self.act_save)
        self._keep_act()
        api.moe_combine(self.y_perm, self.topk_gate, self.dest_row, out=self.out)
        return self.out

    def _keep_act(self):
        if self.act_bits == 8:
            api.moe_act8_save(self.act_save, q=self.act_q, scale=self.act_scale)

    # -- whole passes ----------------------------------------------------------
    def forward(self, x, w_router, w_gate_up, w_down, bias=None, renorm=True,
                prune_beta: Optional[float] = None, prune_alpha: float = math.inf):
        self.route_count(x, w_router, bias=bias, renorm=renorm)
        if prune_beta is not None:
            self.prune(prune_beta, prune_alpha)
            self.route_count(x, w_router, bias=bias, alive=self.alive, renorm=renorm)
        return self.experts_and_combine(x, w_gate_up, w_down)

    def forward_given_routing(self, x, topk_idx, topk_gate, w_gate_up, w_down):
        self.topk_idx.copy_(topk_idx)
        self.topk_gate.copy_(topk_gate)
        self.count()
        return self.experts_and_combine(x, w_gate_up, w_down)

    def route_backward(self, x, w_router, renorm=True, want_dbias=False):
        """Router / gate backward from self.dgate (the combine's gate gradient),
        accumulated onto self.dx.  Renormalised gates only (the full-softmax
        form needs the logits, which the plan does not keep)."""
        if not renorm:
            raise NotImplementedError("the plan keeps no logits; call moe_route_bwd directly")
        if self.dw_router is None:
            self.dw_router = torch.empty(w_router.shape, dtype=torch.float32, device=self.device)
            self.dbias = torch.empty(self.E, dtype=torch.float32, device=self.device)
        api.moe_route_bwd(self.dgate, self.topk_idx, self.topk_gate, x, w_router, renorm=True,
                          offsets=self.offsets, row_src=self.row_src, dx=self.dx,
                          accumulate_dx=True, dw_router=self.dw_router,
                          dbias=self.dbias if want_dbias else None, ws=self.ws_route_bwd)
        return self.dx, self.dw_router

    def _route_bwd(self, x, w_router, balance, **kw):
        """moe_route_bwd, or with ``balance`` (moe_route_bwd_balance's logits,
        grad_coef and options) that call."""
        if balance is None:
            api.moe_route_bwd(self.dgate, self.topk_idx, self.topk_gate, x, w_router, renorm=True,
                              offsets=self.offsets, row_src=self.row_src, **kw)
        else:
            b = dict(balance)
            api.moe_route_bwd_balance(self.dgate, self.topk_idx, self.topk_gate, b.pop("logits"),
                                      x, w_router, b.pop("grad_coef"), **b, **kw)

    def route_backward_weights_async(self, x, w_router, want_dbias=False, balance=None):
        """dw_router (and dbias) from self.dgate on a side stream, started now:
        they need only the gate gradient, so they can run beside the expert
        backward.  route_backward_data waits for them."""
        if self.dw_router is None:
            self.dw_router = torch.empty(w_router.shape, dtype=torch.float32, device=self.device)
            self.dbias = torch.empty(self.E, dtype=torch.float32, device=self.device)
        if self._side is None:
            self._side = torch.cuda.Stream(device=self.device)   # default priority
            self._side_done = torch.cuda.Event()
        main = torch.cuda.current_stream(self.device)
        self._side.wait_stream(main)
        with torch.cuda.stream(self._side):
            self._route_bwd(x, w_router, balance, data=False, dw_router=self.dw_router,
                            want_dbias=want_dbias, dbias=self.dbias if want_dbias else None,
                            ws=self.ws_route_bwd_w)
            self._side_done.record(self._side)

    def route_backward_data(self, x, w_router, balance=None):
        """The router's dx, accumulated onto self.dx; then the current stream
        waits for route_backward_weights_async."""
        self._route_bwd(x, w_router, balance, dx=self.dx, accumulate_dx=True, weights=False,
                        ws=self.ws_route_bwd)
        torch.cuda.current_stream(self.device).wait_event(self._side_done)
        return self.dx, self.dw_router

    def backward(self, dout, w_gate_up, w_down, expert_map=None, accumulate=False,
                 router=None, want_dbias=False, balance=None):
        """Expert backward; with router=(x, w_router) (renormalised gates) also
        the router's, its weight gradients beside the expert backward.
        ``balance``: the router was trained with a balance loss; a dict of
        moe_route_bwd_balance's logits, grad_coef and options (either gates)."""
        api.moe_combine_bwd(dout, self.y_perm, self.topk_gate, self.dest_row,
                            dy_perm=self._dy, dgate=self.dgate)
        if router is not None:
            self.route_backward_weights_async(router[0], router[1], want_dbias=want_dbias,
                                              balance=balance)
        if self.dw_gate_up is None:
            self.dw_gate_up = torch.empty(w_gate_up.shape, dtype=torch.float32,
                                          device=self.device)
            self.dw_down = torch.empty(w_down.shape, dtype=torch.float32, device=self.device)
        # dW_d from the H the forward computed (left in its workspace); at 8-bit
        # pre-activations from the H recomputed there
        h_fwd = (None if self.act_bits == 8 else
                 api.ffn_fwd_h_view(self.ws_ffn, self.R, self.f, self.dtype))
        if self.act_bits == 8:
            api.moe_grouped_ffn_bwd_gather_act8(self._dy, self.x_in, self.row_src, self.k,
                                                self.act_q, self.act_scale, w_gate_up, w_down,
                                                self.offsets, expert_map=expert_map,
                                                dw_gate_up=self.dw_gate_up, dw_down=self.dw_down,
                                                accumulate=accumulate, ws=self.ws_bwd,
                                                dx_perm=self.dx_perm)
        elif self.fused:   # X gathered from the forward's token rows
            api.moe_grouped_ffn_bwd_gather(self._dy, self.x_in, self.row_src, self.k,
                                           self.act_save, w_gate_up, w_down, self.offsets,
                                           h_fwd=h_fwd, expert_map=expert_map,
                                           dw_gate_up=self.dw_gate_up, dw_down=self.dw_down,
                                           accumulate=accumulate, ws=self.ws_bwd,
                                           dx_perm=self.dx_perm)
        else:
            api.moe_grouped_ffn_bwd(self.dy_perm, self.x_perm, self.act_save, w_gate_up,
                                    w_down, self.offsets, h_fwd=h_fwd, expert_map=expert_map,
                                    dw_gate_up=self.dw_gate_up, dw_down=self.dw_down,
                                    accumulate=accumulate, ws=self.ws_bwd, dx_perm=self.dx_perm)
        api.moe_permute_bwd(self.dx_perm, self.dest_row, self.T, self.k, out=self.dx)
        if router is not None:
            self.route_backward_data(router[0], router[1], balance=balance)
        return self.dx, self.dgate, self.dw_gate_up, self.dw_down


def layer_forward(x, w_router, w_gate_up, w_down, k, bias=None, renorm=True,
                  prune_beta=None, prune_alpha=math.inf):
    """One forward pass with freshly allocated buffers; returns the plan."""
    T, d = x.shape
    E = w_router.shape[0]
    f = w_down.shape[2]
    plan = MoELayerPlan(T, d, E, k, f, dtype=x.dtype, device=x.device)
    plan.forward(x, w_router, w_gate_up, w_down, bias=bias, renorm=renorm,
                 prune_beta=prune_beta, prune_alpha=prune_alpha)
    return plan

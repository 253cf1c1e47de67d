"""One pre-norm MoE block on preallocated buffers: layer norm, the MoE layer, and
in training the router's balance loss and 8-bit activation checkpoints.

Forward (x: what the block before added to the residual stream, residual: the
stream it was added to):
    moe_layer_norm      s = x + residual, y = norm(s)
    moe_route_count     routing of y, with the logits
    moe_balance_loss    loss, counts per expert, gradient coefficients (training)
    gathered expert FFN over y, moe_act8_save (training), moe_combine
The block's output goes to the next block's x, and s to its residual, whose norm
adds them; after the last block the stream is out + s.
Backward (dout: the gradient of out + s):
    MoELayerPlan.backward, the router's through moe_route_bwd_balance
    moe_layer_norm_bwd  dx = the norm's gradient + dout, dgamma, dbeta
dx is the gradient of x and of the residual alike: the dout of the block before.

Between a block's forward and its backward pass a training plan keeps s, y, the
row statistics, the routing and logits, y_perm, and the pre-activations in 8 bits
(act_bits=16: in bf16, and H); everything else is scratch, which the blocks of one
model can share (``scratch``), since their passes run one after the other.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Union

import torch

from . import api
from ._lib import LAEP_CALL_BALANCE, LAEP_CALL_LAYER_NORM_BWD
from .layer import MoELayerPlan


class BlockWeights(NamedTuple):
    """gamma, beta float32 [d] (beta may be None); w_router [E, d], w_gate_up
    [E, 2f, d] and w_down [E, d, f] in the plan's dtype (the last two api.Mx4 where it
    has mx4_act)."""
    gamma: torch.Tensor
    beta: Optional[torch.Tensor]
    w_router: torch.Tensor
    w_gate_up: Union[torch.Tensor, api.Mx4]
    w_down: Union[torch.Tensor, api.Mx4]


class MoEBlockPlan:
    def __init__(self, T: int, d_model: int, E: int, k: int, d_ff: int, *, n_seq: int = 1,
                 coef: float = 0.01, eps: float = 1e-5, renorm: bool = True,
                 training: bool = True, act_bits: int = 8, device="cuda",
                 scratch: Optional["MoEBlockPlan"] = None, mx4_act: Optional[int] = None):
        """``coef`` weighs the balance loss, over the batch (n_seq = 1) or per
        sequence; ``training`` False keeps nothing for a backward pass;
        ``act_bits``: how a training block keeps its pre-activations.  8 (the default)
        takes a third of the memory of 16 and 4 % more time a step, and the expert
        backward then sees them rounded to 1/128 of the largest of 32 neighbours; 16
        keeps them, and H, as the forward computed them.
        ``scratch``: a block of the same sizes whose transient buffers to use.
        ``mx4_act`` 4 or 16 (``training`` False): the expert weights are in microscaled 4
        bits, the experts' activations in that many."""
        if scratch is not None and scratch.n_seq != n_seq:
            raise ValueError("scratch must be a block of the same sizes and kind")
        bf16, f32 = torch.bfloat16, torch.float32
        self.n_seq, self.coef, self.eps, self.renorm = n_seq, coef, eps, renorm
        self.training = training
        self.layer = MoELayerPlan(T, d_model, E, k, d_ff, dtype=bf16, device=device,
                                  backward=training, act_bits=act_bits if training else 16,
                                  scratch=None if scratch is None else scratch.layer,
                                  mx4_act=mx4_act)
        dev = self.layer.device

        def new(*shape, dtype=f32):
            return torch.empty(shape, dtype=dtype, device=dev)

        self.y, self.sum = new(T, d_model, dtype=bf16), new(T, d_model, dtype=bf16)
        self.mean, self.rstd = new(T), new(T)
        if not training:
            return
        self.logits = new(T, E)
        self.loss = new(1)
        self.seq_counts = new(n_seq, E, dtype=torch.int32)
        self.prob_mean, self.grad_coef = new(n_seq, E), new(n_seq, E)
        self.dx = new(T, d_model, dtype=bf16)
        self.dgamma, self.dbeta = new(d_model), new(d_model)
        if scratch is not None:
            self.ws_balance, self.ws_norm = scratch.ws_balance, scratch.ws_norm
        else:
            self.ws_balance = new(api.workspace_bytes(LAEP_CALL_BALANCE, T, n_seq, E),
                                  dtype=torch.uint8)
            self.ws_norm = new(max(1, api.workspace_bytes(LAEP_CALL_LAYER_NORM_BWD, T, 1, 1,
                                                          d_model)), dtype=torch.uint8)

    def _check(self, weights: BlockWeights):
        """The matrices' shapes are the plan's (any number of expert slots: expert_map
        says which); the layer's calls read them by the plan's sizes."""
        p, bf16 = self.layer, torch.bfloat16
        api._want(weights.w_router, "w_router", (p.E, p.d), bf16)
        if p.mx4_act is not None:   # the layer's call checks the matrices against each other
            for w, n, shape in ((weights.w_gate_up, "w_gate_up", (2 * p.f, p.d)),
                                (weights.w_down, "w_down", (p.d, p.f))):
                slots = w.codes.shape[0] if isinstance(w, api.Mx4) else 0
                api._need_mx4(w, n, (slots,), *shape, p.out.device)
            return
        slots = weights.w_down.shape[0]
        api._want(weights.w_gate_up, "w_gate_up", (slots, 2 * p.f, p.d), bf16)
        api._want(weights.w_down, "w_down", (slots, p.d, p.f), bf16)

    def forward(self, x, weights: BlockWeights, residual=None, *, bias=None, alive=None,
                seq_offsets=None, expert_map=None, etn_accum=None):
        """Returns (out, s); without a residual s is x, which must then keep its values
        until the backward pass.  ``alive``: the router's mask of unpruned experts;
        ``seq_offsets``: int32 [n_seq + 1] on the device, with n_seq > 1."""
        p = self.layer
        self._check(weights)
        y, s, _, _ = api.moe_layer_norm(x, weights.gamma, weights.beta, residual=residual,
                                        eps=self.eps, out=self.y, mean=self.mean, rstd=self.rstd,
                                        sum_out=None if residual is None else self.sum)
        self._s, self._alive, self._seq_offsets = s, alive, seq_offsets
        api.moe_route_count(y, weights.w_router, p.k, bias=bias, alive=alive, renorm=self.renorm,
                            want_logits=self.training, etn_accum=etn_accum, ws=p.ws_counts,
                            topk_idx=p.topk_idx, topk_gate=p.topk_gate, counts=p.counts,
                            offsets=p.offsets, dest_row=p.dest_row, row_src=p.row_src,
                            logits=self.logits if self.training else None)
        if self.training:
            api.moe_balance_loss(self.logits, p.topk_idx, coef=self.coef, alive=alive,
                                 seq_offsets=seq_offsets, loss=self.loss, counts=self.seq_counts,
                                 prob_mean=self.prob_mean, grad_coef=self.grad_coef,
                                 ws=self.ws_balance)
        out = p.experts_and_combine(y, weights.w_gate_up, weights.w_down, expert_map=expert_map)
        return out, s

    def backward(self, dout, weights: BlockWeights, *, dloss=None, expert_map=None,
                 want_dbias: bool = False, accumulate: bool = False):
        """dx from the gradient of out + s; ``dloss`` (float32 device scalar, None:
        1) is the balance loss's.  The weight gradients are dgamma, dbeta and the
        layer's dw_router, dbias, dw_gate_up and dw_down (``accumulate`` adds to the
        last two)."""
        p = self.layer
        self._check(weights)
        api._want(dout, "dout", (p.T, p.d), torch.bfloat16)
        balance = dict(logits=self.logits, grad_coef=self.grad_coef, alive=self._alive,
                       seq_offsets=self._seq_offsets, dloss=dloss, renorm=self.renorm)
        p.backward(dout, weights.w_gate_up, weights.w_down, expert_map=expert_map,
                   accumulate=accumulate, router=(self.y, weights.w_router),
                   want_dbias=want_dbias, balance=balance)
        api.moe_layer_norm_bwd(p.dx, self._s, weights.gamma, self.mean, self.rstd, dres=dout,
                               want_dbeta=weights.beta is not None, dx=self.dx,
                               dgamma=self.dgamma,
                               dbeta=self.dbeta if weights.beta is not None else None,
                               ws=self.ws_norm)
        return self.dx

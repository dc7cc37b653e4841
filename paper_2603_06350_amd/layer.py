"""Device buffers for one MoE layer and the four-call forward.

PyTorch is used for device memory and the stream handle only; the arithmetic is
in libmoe_gfx950.so.  `MoeBuffers` owns every output and scratch tensor of the
layer so that repeated forwards allocate nothing.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import binding as B


def to_device(a: np.ndarray, device="cuda"):
    """Host array from synth_inputs -> device tensor (uint16 bf16 bits become torch.bfloat16)."""
    if a is None:
        return None
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(a).to(device)


def to_host(t: torch.Tensor) -> np.ndarray:
    """Device tensor -> host array (torch.bfloat16 comes back as uint16 bit patterns)."""
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    return t.cpu().numpy()


class MoeBuffers:
    def __init__(self, T, d, E, k, F, dtype, renorm, device="cuda", split_tiles=False):
        self.shape = B.make_shape(T, d, E, k, F, dtype, renorm)
        self.T, self.d, self.E, self.k, self.F = T, d, E, k, F
        tdt = torch.float32 if dtype == B.MOE_F32 else torch.bfloat16
        A = T * k
        kw = dict(device=device)
        self.topk_idx = torch.empty((T, k), dtype=torch.int32, **kw)
        self.topk_w = torch.empty((T, k), dtype=torch.float32, **kw)
        self.scores = torch.empty((T, E), dtype=torch.float32, **kw)
        self.counts = torch.empty((E,), dtype=torch.int32, **kw)
        self.offsets = torch.empty((E + 1,), dtype=torch.int32, **kw)
        self.dst_row = torch.empty((A,), dtype=torch.int32, **kw)
        self.src_assign = torch.empty((A,), dtype=torch.int32, **kw)
        self.x_perm = torch.empty((A, d), dtype=tdt, **kw)
        self.h = torch.empty((A, F), dtype=tdt, **kw)
        self.y_perm = torch.empty((A, d), dtype=tdt, **kw)
        self.y = torch.empty((T, d), dtype=tdt, **kw)
        self.ws_bytes = B.moe_workspace_bytes(self.shape)
        self.workspace = torch.empty((self.ws_bytes,), dtype=torch.uint8, **kw)
        # optional: the workspace that lets the grouped FFN cut the tiles of an under-filled last
        # round along K (moe_grouped_ffn_ws)
        self.ffn_ws_bytes = B.moe_ffn_workspace_bytes(self.shape) if split_tiles else 0
        self.ffn_ws = torch.empty((self.ffn_ws_bytes,), dtype=torch.uint8, **kw) if split_tiles else None

    def forward(self, x, w_gate, w1, w3, w2, gate_bias=None, stream=None, export_scores=False,
                gather_in_ffn=False, combine_in_ffn=False):
        """The whole hot path: route -> count+permute -> grouped FFN -> combine.
        gather_in_ffn: the up-projection reads x through the permutation map and x_perm is not
        materialised (same results, bit for bit).
        combine_in_ffn (k = 1 layers): the down-projection stores the weighted rows straight to y
        (moe_grouped_ffn_combine_k1); x_perm, y_perm and moe_combine are not used."""
        s = torch.cuda.current_stream() if stream is None else stream
        B.moe_route_ws(self.shape, x, w_gate, gate_bias, self.topk_idx, self.topk_w,
                       self.scores if export_scores else None, self.workspace, self.ws_bytes, s)
        B.moe_count_and_permute(self.shape, x, self.topk_idx, self.counts, self.offsets,
                                self.dst_row, self.src_assign,
                                None if (gather_in_ffn or combine_in_ffn) else self.x_perm,
                                self.workspace, self.ws_bytes, s)
        if combine_in_ffn:
            B.moe_grouped_ffn_combine_k1(self.shape, x, self.src_assign, self.offsets, w1, w3, w2,
                                         self.topk_w, self.h, self.y, s)
            return self.y
        if self.ffn_ws is not None:
            B.moe_grouped_ffn_ws(self.shape, x if gather_in_ffn else self.x_perm,
                                 self.src_assign if gather_in_ffn else None, self.offsets, w1, w3, w2,
                                 self.h, self.y_perm, 3, self.ffn_ws, self.ffn_ws_bytes, s)
        elif gather_in_ffn:
            B.moe_grouped_ffn_gather(self.shape, x, self.src_assign, self.offsets, w1, w3, w2,
                                     self.h, self.y_perm, s)
        else:
            B.moe_grouped_ffn(self.shape, self.x_perm, self.offsets, w1, w3, w2, self.h,
                              self.y_perm, s)
        B.moe_combine(self.shape, self.y_perm, self.dst_row, self.topk_w, self.y, s)
        return self.y


class LoadPredictor:
    """Speculative expert-load prediction for a later layer (paper, Section 4.1): the hidden states
    that enter layer l go through the gate of layer l+d (a replica of that gate, fine-tuned or
    not) to estimate that layer's per-expert token counts ahead of time, and Algorithm 1 turns the
    estimate into replica counts.  Everything is enqueued on one stream, meant to be a side stream
    next to the layer's own forward (Section 5: predictors run asynchronously on dedicated
    streams); nothing is read back to the host.

    enqueue() = moe_route (predictor weights) -> moe_count_and_permute without the row gather ->
    moe_scale_replicas -> moe_replica_segments.  Outputs stay in `counts`, `offsets`, `replicas`,
    `cv` ([before, after]), `seg_offsets`, `seg_expert`, `n_segments`."""

    def __init__(self, T, d, E, k, dtype, renorm, max_extra_replicas, n_gpus=0, device="cuda"):
        # F does not enter any of the calls used here; 8 keeps the shape valid for both dtypes
        self.shape = B.make_shape(T, d, E, k, 8, dtype, renorm)
        self.E = E
        self.max_extra = int(max_extra_replicas)
        A = T * k
        kw = dict(device=device)
        self.topk_idx = torch.empty((T, k), dtype=torch.int32, **kw)
        self.topk_w = torch.empty((T, k), dtype=torch.float32, **kw)
        self.counts = torch.empty((E,), dtype=torch.int32, **kw)
        self.offsets = torch.empty((E + 1,), dtype=torch.int32, **kw)
        self.dst_row = torch.empty((A,), dtype=torch.int32, **kw)
        self.src_assign = torch.empty((A,), dtype=torch.int32, **kw)
        self.ws_bytes = B.moe_workspace_bytes(self.shape)
        self.workspace = torch.empty((self.ws_bytes,), dtype=torch.uint8, **kw)
        self.replicas = torch.empty((E,), dtype=torch.int32, **kw)
        self.cv = torch.empty((2,), dtype=torch.float64, **kw)
        self.max_segments = E + self.max_extra
        self.seg_offsets = torch.empty((self.max_segments + 1,), dtype=torch.int32, **kw)
        self.seg_expert = torch.empty((self.max_segments,), dtype=torch.int32, **kw)
        self.n_segments = torch.empty((1,), dtype=torch.int32, **kw)
        # Algorithm 2 (optional): two sets of placement buffers, the previous round's is the warm set
        self.n_gpus = int(n_gpus)
        self.round = 0
        if self.n_gpus > 0:
            self.gpu_of = [torch.full((self.max_segments,), -1, dtype=torch.int32, **kw) for _ in range(2)]
            self.placed_replicas = [torch.zeros((E,), dtype=torch.int32, **kw) for _ in range(2)]
            self.gpu_load = torch.empty((self.n_gpus,), dtype=torch.float64, **kw)
            self.gpu_count = torch.empty((self.n_gpus,), dtype=torch.int32, **kw)
            self.n_warm = torch.empty((1,), dtype=torch.int32, **kw)

    def enqueue(self, x, w_pred, gate_bias=None, cv_threshold=0.2, stream=None):
        s = torch.cuda.current_stream() if stream is None else stream
        B.moe_route_ws(self.shape, x, w_pred, gate_bias, self.topk_idx, self.topk_w, None,
                       self.workspace, self.ws_bytes, s)
        B.moe_count_and_permute(self.shape, None, self.topk_idx, self.counts, self.offsets,
                                self.dst_row, self.src_assign, None, self.workspace, self.ws_bytes, s)
        # memory in units of one expert: the cap is the number of additional replicas
        B.moe_scale_replicas(self.E, self.counts, 1, self.max_extra, cv_threshold, self.replicas,
                             self.cv, s)
        B.moe_replica_segments(self.E, self.offsets, self.replicas, self.max_segments,
                               self.seg_offsets, self.seg_expert, self.n_segments, s)
        if self.n_gpus > 0:
            cur, prev = self.round & 1, (self.round & 1) ^ 1
            with torch.cuda.stream(s):          # keep these replica counts: the next call's warm set
                self.placed_replicas[cur].copy_(self.replicas, non_blocking=True)
            B.moe_place_replicas(self.E, self.counts, self.replicas, self.n_gpus,
                                 self.placed_replicas[prev] if self.round > 0 else None,
                                 self.gpu_of[prev] if self.round > 0 else None, None,
                                 self.max_segments, self.gpu_of[cur], self.gpu_load, self.gpu_count,
                                 self.n_warm, s)
            self.round += 1


class GateTrainer:
    """Gradients of gates, for fine-tuning load predictors (paper, Section 4.1: a predictor is a copy of a later layer's
    gate, trained on stored hidden states and that gate's outputs) or for the load balance of routers.  One step:

        for i in range(n_gates):
            trainer.enqueue(i, x[i], w_gate[i], target_scores[i])     # loss and gradients of gate i
        trainer.clip()                                               # over the gradients of all gates
        ...                                                           # the caller's optimizer, on d_w_gate and d_gate_bias

    enqueue() = moe_route_ws (scores of the gate) -> moe_gate_distill -> moe_balance_loss -> moe_route_backward (with a
    balance_coef) -> moe_gate_backward.  Everything is enqueued on one stream; nothing is read back to the host, and
    nothing is allocated.  Outputs: `loss`, `balance` [n_gates] (the distillation and the balance loss), `counts`
    [n_gates, E], `d_w_gate` [n_gates, E, d] and `d_gate_bias` [n_gates, E] in fp32, and `norm` [1] of clip().  All gates
    share the trainer's workspace: use one stream at a time."""

    def __init__(self, T, d, E, k, n_gates, dtype, renorm, max_norm=1.0, balance_coef=0.0, device="cuda"):
        # F does not enter any of the calls used here; 8 keeps the shape valid for both dtypes
        self.shape = B.make_shape(T, d, E, k, 8, dtype, renorm)
        self.n_gates = int(n_gates)
        self.max_norm, self.balance_coef = float(max_norm), float(balance_coef)
        kw = dict(device=device)
        self.topk_idx = torch.empty((T, k), dtype=torch.int32, **kw)
        self.topk_w = torch.empty((T, k), dtype=torch.float32, **kw)
        self.scores = torch.empty((T, E), dtype=torch.float32, **kw)
        self.d_scores = torch.empty((T, E), dtype=torch.float32, **kw)
        self.prob_sum = torch.empty((E,), dtype=torch.float32, **kw)
        self.counts = torch.zeros((n_gates, E), dtype=torch.int32, **kw)
        self.loss = torch.zeros((n_gates,), dtype=torch.float32, **kw)
        self.balance = torch.zeros((n_gates,), dtype=torch.float32, **kw)
        self.d_w_gate = torch.zeros((n_gates, E, d), dtype=torch.float32, **kw)
        self.d_gate_bias = torch.zeros((n_gates, E), dtype=torch.float32, **kw)
        self.grads = B.GradList([t for i in range(n_gates) for t in (self.d_w_gate[i], self.d_gate_bias[i])])
        self.weight_grads = B.GradList([self.d_w_gate[i] for i in range(n_gates)])
        self.norm = torch.zeros((1,), dtype=torch.float32, **kw)
        # one buffer: the calls of a step follow each other on a stream
        self.ws_bytes = max(B.moe_workspace_bytes(self.shape), B.moe_train_workspace_bytes(self.shape),
                            B.moe_grad_workspace_bytes(self.grads), B.moe_grad_workspace_bytes(self.weight_grads))
        self.workspace = torch.empty((self.ws_bytes,), dtype=torch.uint8, **kw)

    def score(self, x, w_gate, scores, gate_bias=None, stream=None):
        """The scores [T, E] of a gate on x: targets for the gates that predict it."""
        s = torch.cuda.current_stream() if stream is None else stream
        sh = self.shape
        B.check_tensors("GateTrainer.score", ("x", x, sh.dtype, sh.T * sh.d), ("w_gate", w_gate, sh.dtype, sh.E * sh.d),
                        ("scores", scores, B.F32, sh.T * sh.E), ("gate_bias", gate_bias, B.F32, sh.E))
        B.moe_route_ws(sh, x, w_gate, gate_bias, self.topk_idx, self.topk_w, scores, self.workspace, self.ws_bytes, s)

    def enqueue(self, i, x, w_gate, target_scores, gate_bias=None, token_mask=None, accumulate=False, d_x=None,
                stream=None, coef=1.0):
        """Losses and gradients of gate i.  token_mask: 0 for padded tokens.  accumulate: the gradients are added to
        those of earlier micro-batches (before clip()).  coef: what the gradients of this call are multiplied by; micro-batches
        add up to the gradient of the mean over all their tokens if each has its share of the tokens that count.  d_x: an
        output for the hidden states' gradient, or None."""
        s = torch.cuda.current_stream() if stream is None else stream
        ws, nb = self.workspace, self.ws_bytes
        self.score(x, w_gate, self.scores, gate_bias, s)
        B.moe_gate_distill(self.shape, self.scores, target_scores, token_mask, coef, self.loss[i:i + 1], self.d_scores, 0,
                           ws, nb, s)
        B.moe_balance_loss(self.shape, self.scores, self.topk_idx, token_mask, self.counts[i], self.prob_sum,
                           self.balance[i:i + 1], ws, nb, s)
        if self.balance_coef != 0.0:
            B.moe_route_backward(self.shape, self.scores, None, None, self.counts[i], coef * self.balance_coef, token_mask,
                                 self.d_scores, 1, s)
        B.moe_gate_backward(self.shape, x, None if d_x is None else w_gate, self.d_scores, token_mask, self.d_w_gate[i],
                            self.d_gate_bias[i], d_x, B.MOE_ACCUMULATE_WEIGHTS if accumulate else 0, ws, nb, s)

    def clip(self, stream=None, bias=True):
        """Scales the gradients of all gates, in place, to a norm of at most max_norm; returns `norm` (on the device).
        bias=False: of gates without a trained bias; d_gate_bias has no part in the norm and is left as it is."""
        s = torch.cuda.current_stream() if stream is None else stream
        B.moe_clip_grads(self.grads if bias else self.weight_grads, self.max_norm, self.norm, self.workspace, self.ws_bytes, s)
        return self.norm


def finetune_predictor(trainer: GateTrainer, x_now, target_scores, w_gate, steps, lr, token_mask=None, gate_bias=None):
    """Fine-tunes the gate of `trainer` (which has one), starting from w_gate: predictor of `target_scores` from x_now.
    gate_bias: of a gate that has one; a copy of it is trained as well.  Returns the new weights in w_gate's type, the losses
    of the steps and, with a gate_bias, the new bias.  The optimizer is PyTorch's Adam on fp32 copies.  ValueError if the
    gradients of a step are not finite (an infinity or NaN in x_now or target_scores, or weights that grew out of range)."""
    if trainer.n_gates != 1:      # clip() goes over the gradients of all gates, also those that no step here writes
        raise ValueError(f"finetune_predictor: a trainer of one gate, not of {trainer.n_gates}")
    w_gate = w_gate.detach()
    master = w_gate.float().clone().requires_grad_(True)
    bias = None if gate_bias is None else gate_bias.detach().clone().requires_grad_(True)      # fp32: its own copy
    opt = torch.optim.Adam([master] if bias is None else [master, bias], lr=lr)
    w, losses, norms = w_gate.clone(), [], []
    for _ in range(steps):
        trainer.enqueue(0, x_now, w, target_scores, gate_bias=bias, token_mask=token_mask)
        norms.append(trainer.clip(bias=bias is not None).clone())
        losses.append(trainer.loss[0].clone())
        master.grad = trainer.d_w_gate[0]
        if bias is not None:
            bias.grad = trainer.d_gate_bias[0]
        opt.step()
        with torch.no_grad():
            w.copy_(master)
    losses = [float(v) for v in losses]
    for i, norm in enumerate(norms):
        if not math.isfinite(float(norm)):
            raise ValueError(f"finetune_predictor: the gradients of step {i} are not finite (norm {float(norm)}, loss {losses[i]})")
    return (w, losses) if bias is None else (w, losses, bias.detach())


def predicted_vs_actual_loads(pred: LoadPredictor, x_now, x_later, w_pred, gate_bias=None, stream=None, w_later=None,
                              bias_later=None):
    """How well the loads predicted from the current hidden states match those the same gate (or w_later and bias_later,
    the gate that w_pred and gate_bias were fine-tuned to predict; each is the predictor's where it is None) sees one
    layer later (paper, Section 4.1 and its accuracy study): both passes are the library's routing and counting; the
    comparison of the two small count vectors is host arithmetic.
    Returns (predicted counts, actual counts, fraction of (token, slot) choices that the later
    routing also makes for that token)."""
    s = torch.cuda.current_stream() if stream is None else stream
    pred.enqueue(x_now, w_pred, gate_bias, stream=s)
    with torch.cuda.stream(s):
        c_pred = pred.counts.clone()
        idx_pred = pred.topk_idx.clone()
    pred.enqueue(x_later, w_pred if w_later is None else w_later,
                 gate_bias if bias_later is None else bias_later, stream=s)
    with torch.cuda.stream(s):
        same = (idx_pred.unsqueeze(2) == pred.topk_idx.unsqueeze(1)).any(dim=2).float().mean()
    s.synchronize()
    return c_pred.cpu().numpy(), pred.counts.cpu().numpy(), float(same.item())

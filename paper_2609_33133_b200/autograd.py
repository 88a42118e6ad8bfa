"""torch.autograd wrappers around the entry points (argument marshalling only): tree attention, embedding, vocabulary loss, block ends.

`tree_attention(plan, q_p, k_p, v_p, q_r, k_r, v_r)` returns `(o_p, o_r)` for the packed prompt and
response tokens of a plan's groups; backward fills the gradients of all six inputs.  The order inside
backward is the one the method requires (Sec. 3.2): the replay backward first, which seeds the shared
prompt-KV gradient with the sum over every branch (Eq. 2), then the prefill backward, which adds the
prompt's own contribution and pushes the total through the prefill pass.  Inputs and outputs are bf16
`[tokens, heads, head_dim]`; the prompt-KV gradients are accumulated in fp32 and cast once at the end
(autograd hands a gradient back in its input's dtype).  The fp32 accumulators of the latest backward stay
available as `plan.prompt_grad_fp32 = (dK_P, dV_P)` for callers that want them unrounded.

`embed(lm, table, ids)` and `lm_loss(lm, hidden, weight, targets)` are the two vocabulary ends of a model around it: a
`binding.LM` handle carries the sizes and scales.  Negative ids are padding in both.

`block(blk, x, o, ..)`, `norm(blk, x, w)` and `glu(blk, g, u)` are what lies between a decoder layer's products; a `binding.Block` handle
carries the width, the scales and the form of the gate.  With `ckpt=True` what their backward passes need is kept in 8 bits, and `linear` and
`glu_linear` take their weight gradients from the same checkpoints, so that neither the residual stream, nor the norms' outputs, nor the MLP's
inner activations outlive the forward pass in full.
"""
from __future__ import annotations

import torch
import torch.nn.functional as F

from . import binding as B


class _TreeAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, q_p, k_p, v_p, q_r, k_r, v_r):
        for t in (q_p, k_p, v_p, q_r, k_r, v_r):
            if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
                raise ValueError("tree_attention takes contiguous bf16 CUDA tensors")
        dev = q_p.device
        hq, d = plan.h_q, plan.head_dim
        o_p = torch.empty((plan.total_p, hq, d), device=dev, dtype=torch.bfloat16)
        o_r = torch.empty((plan.total_r, hq, d), device=dev, dtype=torch.bfloat16)
        lse_p = torch.empty((hq, plan.total_p), device=dev, dtype=torch.float32)
        lse_r = torch.empty((hq, plan.total_r), device=dev, dtype=torch.float32)
        ws = torch.empty(max(plan.ws_fwd_bytes, plan.ws_bwd_bytes, 256), device=dev, dtype=torch.uint8)
        plan.prefill_fwd(q_p, k_p, v_p, o_p, lse_p, ws)
        plan.replay_fwd(q_r, k_r, v_r, k_p, v_p, o_r, lse_r, ws)
        ctx.plan, ctx.ws = plan, ws
        ctx.save_for_backward(q_p, k_p, v_p, q_r, k_r, v_r, o_p, lse_p, o_r, lse_r)
        return o_p, o_r

    @staticmethod
    def backward(ctx, do_p, do_r):
        plan, ws = ctx.plan, ctx.ws
        q_p, k_p, v_p, q_r, k_r, v_r, o_p, lse_p, o_r, lse_r = ctx.saved_tensors
        dev = q_p.device
        hq, hkv, d = plan.h_q, plan.h_kv, plan.head_dim
        bf = torch.bfloat16
        do_p = torch.zeros_like(o_p) if do_p is None else do_p.to(bf).contiguous()
        do_r = torch.zeros_like(o_r) if do_r is None else do_r.to(bf).contiguous()
        dq_p = torch.empty((plan.total_p, hq, d), device=dev, dtype=bf)
        dq_r = torch.empty((plan.total_r, hq, d), device=dev, dtype=bf)
        dk_r = torch.empty((plan.total_r, hkv, d), device=dev, dtype=bf)
        dv_r = torch.empty((plan.total_r, hkv, d), device=dev, dtype=bf)
        dk_acc = torch.zeros((plan.total_p, hkv, d), device=dev, dtype=torch.float32)
        dv_acc = torch.zeros((plan.total_p, hkv, d), device=dev, dtype=torch.float32)
        dk_p = torch.empty((plan.total_p, hkv, d), device=dev, dtype=bf)
        dv_p = torch.empty((plan.total_p, hkv, d), device=dev, dtype=bf)
        plan.replay_bwd(q_r, k_r, v_r, k_p, v_p, o_r, lse_r, do_r, dq_r, dk_r, dv_r, dk_acc, dv_acc, ws)
        plan.prefill_bwd(q_p, k_p, v_p, o_p, lse_p, do_p, dk_acc, dv_acc, dq_p, dk_p, dv_p, ws)
        plan.prompt_grad_fp32 = (dk_acc, dv_acc)
        return None, dq_p, dk_p, dv_p, dq_r, dk_r, dv_r


def tree_attention(plan: B.Plan, q_p, k_p, v_p, q_r, k_r, v_r):
    """Prompt-sharing tree attention of a plan's groups; differentiable in all six tensors."""
    return _TreeAttention.apply(plan, q_p, k_p, v_p, q_r, k_r, v_r)


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, lm, table, ids, out_dtype):
        out = torch.empty((ids.shape[0], lm.hidden), device=table.device, dtype=out_dtype or table.dtype)
        lm.embed_fwd(table, ids, out)
        ctx.lm, ctx.dtype = lm, table.dtype
        ctx.save_for_backward(ids)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_out):
        lm, (ids,) = ctx.lm, ctx.saved_tensors
        d_table = torch.empty((lm.vocab, lm.hidden), device=d_out.device, dtype=ctx.dtype)
        ws = torch.empty(lm.workspace_parts(ids.shape[0])[2], device=d_out.device, dtype=torch.uint8)
        lm.embed_bwd(d_out.contiguous(), ids, d_table, ws)
        return None, d_table, None, None


def embed(lm: B.LM, table, ids, out_dtype=None):
    """lm.embed_scale * table[ids] in fp32, rounded to out_dtype (default: the table's); zeros for negative ids.  Differentiable in
    table (fp32, bf16 or fp16), whose gradient is dense and in its type."""
    return _Embed.apply(lm, table, ids, out_dtype)


class _LmLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, lm, hidden, weight, targets):
        n, dev = targets.shape[0], hidden.device
        loss = torch.empty(n, device=dev, dtype=torch.float32)
        lse = torch.empty(n, device=dev, dtype=torch.float32)
        ws = torch.empty(lm.workspace_parts(n)[0], device=dev, dtype=torch.uint8)
        lm.loss_fwd(hidden, weight, targets, loss, lse, ws)
        ctx.lm = lm
        ctx.save_for_backward(hidden, weight, targets, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_loss):
        lm, (hidden, weight, targets, lse) = ctx.lm, ctx.saved_tensors
        d_hidden = torch.empty_like(hidden) if ctx.needs_input_grad[1] else None
        d_weight = torch.empty_like(weight) if ctx.needs_input_grad[2] else None
        ws = torch.empty(lm.workspace_parts(targets.shape[0])[1], device=hidden.device, dtype=torch.uint8)
        lm.loss_bwd(hidden, weight, targets, lse, d_loss.contiguous(), d_hidden, d_weight, ws)
        return None, d_hidden, d_weight, None


def lm_loss(lm: B.LM, hidden, weight, targets):
    """Cross entropy of every token (fp32; zero for a negative target) under the logits lm.logit_scale * hidden @ weight.T, which
    are never held: hidden [tokens, hidden] and weight [vocab, hidden] bf16.  Differentiable in both; a gradient that nobody
    asks for is not computed.  The negative of it is the log-probability of the target."""
    return _LmLoss.apply(lm, hidden, weight, targets)


class Kept:
    """A tensor in 8 bits, as a norm's output: what `ckpt` [tokens, pitch] stands for times row[t] and col[c]."""

    def __init__(self, ckpt, row, col):
        self.ckpt, self.row, self.col = ckpt, row, col


def _like(t, shape=None, dtype=None):
    return None if t is None else torch.empty(t.shape if shape is None else shape, device=t.device, dtype=dtype or t.dtype)


class _Block(torch.autograd.Function):
    @staticmethod
    def forward(ctx, blk, x, o, gate, w_out, w_in, h_dtype, ckpt):
        n, dev = x.shape[0], x.device
        f32 = lambda: torch.empty(n, device=dev, dtype=torch.float32)
        box = lambda: torch.empty((n, B.ckpt_pitch(blk.hidden)), device=dev, dtype=torch.uint8)
        y = None if o is None else torch.empty_like(x)
        h = None if w_in is None else torch.empty((n, blk.hidden), device=dev, dtype=h_dtype)
        r_out, r_in = None if w_out is None else f32(), None if w_in is None else f32()
        kept_y, kept_o = (box() if w_in is not None else None, None if o is None else box()) if ckpt else (None, None)
        blk.fwd(x, o, gate, w_out, w_in, y, h, r_out, r_in, kept_y, kept_o)
        ctx.set_materialize_grads(False)
        ctx.blk, ctx.like = blk, (x.dtype, None if o is None else o.dtype)
        # (all of it as saved tensors: an attribute would outlive the backward pass as long as somebody holds the loss)
        ctx.save_for_backward(gate, w_out, w_in, r_out, r_in, *((kept_y, kept_o) if ckpt else (x if o is None else y, o)))
        kept = Kept(kept_y, r_in, w_in.detach()) if kept_y is not None else None
        return y, h, kept

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dh, _):
        blk = ctx.blk
        gate, w_out, w_in, r_out, r_in, y, o = ctx.saved_tensors
        x_dtype, o_dtype = ctx.like
        if dy is None and dh is None:
            return (None,) * 8
        lead = dh if dy is None else dy
        dy, dh = (None if t is None else t.contiguous() for t in (dy, dh))
        if dh is None:
            y = r_in = w_in = None
        need = ctx.needs_input_grad
        dx = _like(lead, dtype=x_dtype) if need[1] else None
        d_o = _like(lead, dtype=o_dtype) if need[2] else None
        d_gate, dw_out, dw_in = (_like(t) if wanted else None for t, wanted in zip((gate, w_out, w_in), need[3:6]))
        ws = torch.empty(blk.workspace_bytes(lead.shape[0]), device=lead.device, dtype=torch.uint8)
        try:
            blk.bwd(dy, dh, y, o, gate, w_out, w_in, r_out, r_in, dx, d_o, d_gate, dw_out, dw_in, ws)
        except B.AugtreeError as err:
            if err.code != B.ERR_UNSUPPORTED or o is None or dh is None:
                raise
            # A row of all inputs does not fit a CTA: about 8192 channels, everything in fp32 and a gate.  In two calls then, the norm before the next block
            # and what lies before it.  What passes between them is the gradient of y in fp32, which one call would have held as well.
            dx = _like(lead, dtype=x_dtype) if dx is None else dx
            blk.bwd(dy, dh, y, None, None, None, w_in, None, r_in, dx, None, None, None, dw_in, ws)
            blk.bwd(dx, None, None, o, gate, w_out, None, r_out, None, None, d_o, d_gate, dw_out, None, ws)
            dx = dx if need[1] else None
        return None, dx, d_o, d_gate, dw_out, dw_in, None, None


def block(blk: B.Block, x, o, gate=None, w_out=None, w_in=None, *, h_dtype=torch.bfloat16, ckpt=False):
    """End of a block: y = x + s a(gate) norm(o, w_out) (o itself without w_out) and, with w_in, h = norm(y, w_in) in h_dtype.  Returns
    (y, h or None, Kept or None): the last with ckpt=True, where y and o are kept in 8 bits for the backward pass.  Differentiable in all tensors."""
    return _Block.apply(blk, x, o, gate, w_out, w_in, h_dtype, ckpt)


def norm(blk: B.Block, x, w, *, h_dtype=torch.bfloat16, ckpt=False):
    """h = x / rms(x) * w in h_dtype; returns (h, Kept or None)."""
    return _Block.apply(blk, x, None, None, None, w, h_dtype, ckpt)[1:]


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, blk, h, weight, kept):
        ctx.blk = blk
        ctx.save_for_backward(weight, kept.ckpt, kept.row, kept.col)     # (what is changed before the backward pass is an error, as everywhere)
        return F.linear(h, weight)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d):
        blk, (weight, ckpt, row, col) = ctx.blk, ctx.saved_tensors
        d = d.contiguous()
        dw = None
        if ctx.needs_input_grad[2]:
            dw = _like(weight)      # (contiguous, whatever the weight's strides)
            ws = torch.empty(blk.wgrad_workspace_bytes(d.shape[0], *weight.shape), device=d.device, dtype=torch.uint8)
            blk.wgrad(d, ckpt, dw, ws, row, col)
        return None, d @ weight if ctx.needs_input_grad[1] else None, dw, None


def linear(blk: B.Block, h, weight, kept=None):
    """h @ weight.T in bf16.  With `kept` (of the same h) the weight's gradient comes from the checkpoint and h is not saved; what that gradient's product does
    not take (other types, more dimensions, a number of features that is no multiple of 8) is refused here and not in the backward pass."""
    if kept is None:
        return F.linear(h, weight)
    y = _Linear.apply(blk, h, weight, kept)
    if weight.requires_grad and torch.is_grad_enabled():
        got = lambda t: f"{tuple(t.shape)} {t.dtype}"
        if h.dim() != 2 or y.dtype is not torch.bfloat16 or weight.dtype not in (torch.bfloat16, torch.float32) or weight.shape[0] % 8:
            raise ValueError("linear with a checkpoint: expected a bf16 product of h [tokens, columns] with a bf16 or fp32 weight [a multiple of 8, columns], got "
                             f"{got(h)} and {got(weight)}, product {y.dtype}")
        if kept.ckpt.shape != (h.shape[0], B.ckpt_pitch(h.shape[1])):
            raise ValueError(f"linear: h is {got(h)}, the checkpoint is of another tensor: {got(kept.ckpt)}")
        blk.wgrad_workspace_bytes(h.shape[0], *weight.shape)      # (raises for sizes beyond the product's limits)
    return y


class _Glu(torch.autograd.Function):
    @staticmethod
    def forward(ctx, blk, g, u, weight, ckpt):
        n, cols = g.shape
        a = torch.empty((n, cols), device=g.device, dtype=g.dtype)
        box = lambda: torch.empty((n, B.ckpt_pitch(cols)), device=g.device, dtype=torch.uint8) if ckpt else None
        kept = (box(), box())
        blk.glu_fwd(g, u, a, *kept)
        ctx.blk = blk
        ctx.save_for_backward(weight, *(kept if ckpt else (g, u)))
        return a if weight is None else F.linear(a, weight)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d):
        weight, g, u = ctx.saved_tensors
        da = (d if weight is None else d @ weight).contiguous()
        dg, du = torch.empty_like(da), torch.empty_like(da)
        a = torch.empty_like(da) if weight is not None and ctx.needs_input_grad[3] else None
        ctx.blk.glu_bwd(da, g, u, dg, du, a)
        return None, dg, du, None if a is None else d.t() @ a, None


def glu(blk: B.Block, g, u, *, ckpt=False):
    """g / (1 + exp(-g)) u (rows contiguous, one type); with ckpt=True g and u are kept in 8 bits for the backward pass."""
    return _Glu.apply(blk, g, u, None, ckpt)


def glu_linear(blk: B.Block, g, u, weight, *, ckpt=False):
    """glu(g, u) @ weight.T: the product behind a gated MLP, whose weight gradient takes the activation made again in the backward pass, so that it is
    never saved."""
    return _Glu.apply(blk, g, u, weight, ckpt)

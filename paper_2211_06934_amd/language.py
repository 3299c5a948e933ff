"""torch.autograd over the operators of a language model (``operators``).

An inner step of Listing 1 takes the gradient of its loss with
``create_graph=True`` and the outer loss differentiates through that gradient,
so each Function here has a backward that is a Function itself:

* ``linear_attention``: the operator is linear in q and in its initial state
  and bilinear in (k, v), its gradients are the same sum on permuted operands,
  and the derivative of a gradient is made of the operator's own calls.  Any
  order of differentiation works.
* ``qknorm_rope`` and ``distillation_loss``: differentiable twice, by kernels
  for the backward and for the backward's backward.  Asking for a third order
  raises an error.

Tensors are brought into a shape that the kernels read (whole heads, whole
rows) before a Function is applied, so that what it saves are its inputs.

``linear_attention_step`` is the single-token form for generation: no graph,
the state updated in place.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import operators as _o


def _dense(x: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """x with contiguous elements along its last axis (a cotangent may be an expanded scalar)."""
    return x if x is None or x.shape[-1] <= 1 or x.stride(-1) == 1 else x.contiguous()


def _whole(x: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    return None if x is None else x.contiguous()


def _plus(*terms):
    """The sum of the terms that are there."""
    terms = [t for t in terms if t is not None]
    if not terms:
        return None
    total = terms[0]
    for t in terms[1:]:
        total = total + t
    return total


# ---- linear attention -------------------------------------------------------


class LinearAttentionFn(torch.autograd.Function):
    """(q, k, v, state) -> (out, state_out); state may be None."""

    @staticmethod
    def forward(ctx, q, k, v, state, log_decay, lengths, scale: float, want_state: bool):
        out = torch.empty(*q.shape[:3], v.shape[3], dtype=q.dtype, device=q.device)
        s1 = torch.empty(k.shape[0], k.shape[2], k.shape[3], v.shape[3], device=q.device) if want_state else None
        _o.linattn_fwd(q, k, v, log_decay, out, state, s1, lengths, scale)
        ctx.save_for_backward(q, k, v, state, log_decay, lengths)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return out, s1

    @staticmethod
    def backward(ctx, dout, ds1):
        q, k, v, state, log_decay, lengths = ctx.saved_tensors
        need = ctx.needs_input_grad
        if dout is None and ds1 is None:
            return (None,) * 8
        dout = torch.zeros(*q.shape[:3], v.shape[3], dtype=q.dtype, device=q.device) if dout is None else _dense(dout)
        want = (need[0], need[1], need[2], need[3] and state is not None)
        grads = LinearAttentionGradFn.apply(dout, _whole(ds1), q, k, v, state, log_decay, lengths, ctx.scale, want)
        return (*grads, None, None, None, None)


class LinearAttentionGradFn(torch.autograd.Function):
    """(dout, dstate_out, q, k, v, state) -> (dq, dk, dv, dstate), those that `want` names."""

    @staticmethod
    def forward(ctx, dout, ds1, q, k, v, state, log_decay, lengths, scale: float, want):
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) if w else None for x, w in zip((q, k, v), want))
        ds = torch.empty(k.shape[0], k.shape[2], k.shape[3], v.shape[3], device=q.device) if want[3] else None
        _o.linattn_bwd(dout, q, k, v, log_decay, dq, dk, dv, state, ds1, ds, lengths, scale)
        ctx.save_for_backward(dout, ds1, q, k, v, state, log_decay, lengths)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return dq, dk, dv, ds

    # Of <a, dq> + <b, dk> + <c, dv> + <e, dstate> = <dout, F> + <ds1, S> with
    #   F = out(a, k, v; state) + out(q, b, v; e) + out(q, k, c; 0)
    #   S = state_out(b, v; e) + state_out(k, c; 0)
    # each term is the operator on other operands, and its gradients are the
    # operator's own.
    @staticmethod
    def backward(ctx, a, b, c, e):
        do, ds1, q, k, v, state, lg, ln = ctx.saved_tensors
        need = ctx.needs_input_grad
        end = ds1 is not None and need[1]
        a, b, c, e = _dense(a), _dense(b), _dense(c), _whole(e)

        def out(q, k, v, s0, want_state):
            return LinearAttentionFn.apply(q, k, v, s0, lg, ln, ctx.scale, want_state)

        def grads(ds1, q, k, v, s0, want):
            return LinearAttentionGradFn.apply(do, ds1, q, k, v, s0, lg, ln, ctx.scale, want) if any(want) else (None,) * 4

        g_do, g_s1, g_q, g_k, g_v, g_s0 = ([] for _ in range(6))
        if a is not None:
            if need[0]:
                g_do.append(out(a, k, v, state, False)[0])
            _, dk, dv, ds = grads(None, a, k, v, state, (False, need[3], need[4], need[5] and state is not None))
            g_k.append(dk), g_v.append(dv), g_s0.append(ds)
        if b is not None or e is not None:
            b = torch.zeros_like(k) if b is None else b
            if need[0] or end:
                o, s = out(q, b, v, e, end)
                g_do.append(o), g_s1.append(s)
            dq, _, dv, _ = grads(ds1, q, b, v, e, (need[2], False, need[4], False))
            g_q.append(dq), g_v.append(dv)
        if c is not None:
            if need[0] or end:
                o, s = out(q, k, c, None, end)
                g_do.append(o), g_s1.append(s)
            dq, dk, _, _ = grads(ds1, q, k, c, None, (need[2], need[3], False, False))
            g_q.append(dq), g_k.append(dk)
        return (_plus(*g_do) if need[0] else None, _plus(*g_s1), _plus(*g_q), _plus(*g_k), _plus(*g_v), _plus(*g_s0),
                None, None, None, None)


def linear_attention(q, k, v, log_decay, state=None, lengths=None, scale: float = 1.0,
                     return_state: bool = False):
    """out_t = scale S_t^T q_t with S_t = exp(log_decay) S_{t-1} + k_t v_t^T, over sequences.

    q [B, T, H, Dk], k [B, T, Hk, Dk], v [B, T, Hk, Dv], all fp32 or all bf16 (H a multiple of Hk: query heads share k/v
    heads); log_decay fp32 [Hk], a constant: it has no gradient, and one that asks for it is refused.  state: fp32
    [B, Hk, Dk, Dv] before the first token (None: zeros).  lengths: int32 [B]; tokens from there on give zeros.  Returns
    out [B, T, H, Dv], with return_state also the state after the last token.  Differentiable in q, k, v and state, any
    number of times."""
    if isinstance(log_decay, torch.Tensor) and log_decay.requires_grad:
        raise ValueError("linear_attention: log_decay has no gradient: pass a tensor that does not require one")
    _o._dims(q, k, v, 4)
    out, s1 = LinearAttentionFn.apply(_dense(q), _dense(k), _dense(v), _whole(state), log_decay, lengths, float(scale), bool(return_state))
    return (out, s1) if return_state else out


def linear_attention_step(q, k, v, log_decay, state, scale: float = 1.0) -> torch.Tensor:
    """One token of every sequence for generation: q [B, H, Dk], k [B, Hk, Dk], v [B, Hk, Dv] -> out [B, H, Dv]; `state` is
    updated in place.  Not differentiable: an operand that asks for a gradient is refused, but under torch.no_grad()."""
    if torch.is_grad_enabled():
        for x, what in ((q, "q"), (k, "k"), (v, "v"), (log_decay, "log_decay"), (state, "state")):
            if isinstance(x, torch.Tensor) and x.requires_grad:
                raise ValueError("linear_attention_step: %s asks for a gradient, and single tokens have none: detach it, or step "
                                 "under torch.no_grad()" % what)
    _o._dims(q, k, v, 3)
    with torch.no_grad():
        q, k, v = _dense(q), _dense(k), _dense(v)
        out = torch.empty(*q.shape[:2], v.shape[2], dtype=q.dtype, device=q.device)
        _o.linattn_step(q, k, v, log_decay, state, out, scale)
    if not state.is_inference():  # the kernel wrote past torch: a graph that saved the state has to notice
        torch.autograd.graph.increment_version(state)
    return out


# ---- norms of queries and keys, rotation ------------------------------------


class QkNormRopeFn(torch.autograd.Function):
    """(q, k, q_weight, k_weight) -> (q_out, k_out); k and the weights may be None."""

    @staticmethod
    def forward(ctx, q, k, qw, kw, cos, sin, positions, how):
        yq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        yk = None if k is None else torch.empty(k.shape, dtype=k.dtype, device=k.device)
        _o.qknorm_rope_fwd(q, k, qw, kw, cos, sin, yq, yk, positions, *how)
        ctx.save_for_backward(q, k, qw, kw, cos, sin, positions)
        ctx.how = how
        return yq, yk

    @staticmethod
    def backward(ctx, dyq, dyk):
        q, k, qw, kw, cos, sin, positions = ctx.saved_tensors
        want = (ctx.needs_input_grad[2] and qw is not None, ctx.needs_input_grad[3] and kw is not None)
        return (*QkNormRopeGradFn.apply(_dense(dyq), _dense(dyk) if k is not None else None, q, k, qw, kw, cos, sin, positions, ctx.how, want),
                None, None, None, None)


class QkNormRopeGradFn(torch.autograd.Function):
    """(dq_out, dk_out, q, k, q_weight, k_weight) -> (dq, dk, dq_weight, dk_weight)."""

    @staticmethod
    def forward(ctx, dyq, dyk, q, k, qw, kw, cos, sin, positions, how, want):
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        dk = None if k is None else torch.empty(k.shape, dtype=k.dtype, device=k.device)
        dw = [torch.empty_like(w) if yes else None for w, yes in zip((qw, kw), want)]
        _o.qknorm_rope_bwd(dyq, dyk, q, k, qw, kw, cos, sin, dq, dk, *dw, positions, *how)
        ctx.save_for_backward(dyq, dyk, q, k, qw, kw, cos, sin, positions)
        ctx.how = how
        ctx.set_materialize_grads(False)
        return (dq, dk, *dw)

    @staticmethod
    @once_differentiable
    def backward(ctx, a, ak, b, bk):
        dyq, dyk, q, k, qw, kw, cos, sin, positions = ctx.saved_tensors
        new = lambda x: None if x is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        oy, oyk, ox, oxk = new(dyq), new(dyk), new(q), new(k)
        ow = [torch.empty_like(w) if need and w is not None else None for w, need in zip((qw, kw), ctx.needs_input_grad[4:6])]
        _o.qknorm_rope_bwd_bwd(_dense(a), _dense(ak), _whole(b), _whole(bk), dyq, dyk, q, k, qw, kw, cos, sin, oy, oyk, ox, oxk, *ow,
                               positions, *ctx.how)
        return (oy, oyk, ox, oxk, *ow, None, None, None, None, None)


def qknorm_rope(q, k, q_weight=None, k_weight=None, cos=None, sin=None, positions=None, first: int = 0, eps: float = 1e-6,
                interleaved: bool = False) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """RMS norms of queries [B, T, H, D] and keys [B, T, Hk, D] for each head, scaled by fp32 weights [D] (None: ones), and
    the rotation by row positions[b, t] (None: first + t) of the fp32 tables cos and sin [rows, rot/2] (None: no rotation);
    pairs are (i, i + rot/2), or (2i, 2i + 1) with `interleaved`.  k may be None.  Returns (q_out, k_out).  Differentiable
    twice in q, k and the weights; the tables are constants."""
    for x, what in ((cos, "cos"), (sin, "sin")):
        if isinstance(x, torch.Tensor) and x.requires_grad:
            raise ValueError("qknorm_rope: %s has no gradient: pass a tensor that does not require one" % what)
    return QkNormRopeFn.apply(_dense(q), _dense(k), _whole(q_weight), _whole(k_weight), cos, sin, positions, (int(first), float(eps), bool(interleaved)))


# ---- distillation -----------------------------------------------------------


class DistillationFn(torch.autograd.Function):
    """(logits, teacher) -> the loss of every row."""

    @staticmethod
    def forward(ctx, logits, teacher, ids, temperature: float):
        loss, stats = (torch.empty(n, device=logits.device) for n in ((logits.shape[0],), (logits.shape[0], 2)))
        _o.distill_fwd(logits, ids, teacher, loss, stats, temperature)
        ctx.save_for_backward(logits, teacher, ids, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    def backward(ctx, dloss):
        logits, teacher, ids, stats = ctx.saved_tensors
        return (*DistillationGradFn.apply(dloss.contiguous(), logits, teacher, ids, stats, ctx.temperature, ctx.needs_input_grad[1]), None, None)


class DistillationGradFn(torch.autograd.Function):
    """(dloss, logits, teacher) -> (dlogits, dteacher)."""

    @staticmethod
    def forward(ctx, dloss, logits, teacher, ids, stats, temperature: float, want_teacher: bool):
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        dteacher = torch.empty_like(teacher) if want_teacher else None
        _o.distill_bwd(dloss, logits, ids, teacher, stats, dlogits, dteacher, temperature)
        ctx.save_for_backward(dloss, logits, teacher, ids, stats)
        ctx.temperature = temperature
        ctx.set_materialize_grads(False)
        return dlogits, dteacher

    @staticmethod
    @once_differentiable
    def backward(ctx, a, c):
        dloss, logits, teacher, ids, stats = ctx.saved_tensors
        need = ctx.needs_input_grad
        od = torch.empty_like(dloss) if need[0] else None
        ot = torch.empty_like(teacher) if need[2] else None
        ol = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        _o.distill_bwd_bwd(_dense(a), _whole(c), dloss, logits, ids, teacher, stats, od, ol, ot, ctx.temperature)
        return od, ol, ot, None, None, None, None


def distillation_loss(logits, ids, teacher, temperature: float = 1.0) -> torch.Tensor:
    """Loss [N] of the student's logits [N, V] (fp32 or bf16) against a teacher's fp32 logits [N, K] at tokens ids [N, K]
    (int32 or int64): T^2 KL(softmax(teacher / T) || softmax(logits / T)) over the row's entries.  A negative id or a
    teacher logit of -inf is no entry; a row without entries has loss 0.  Differentiable twice in logits and teacher."""
    return DistillationFn.apply(_dense(logits), _whole(teacher), _whole(ids), float(temperature))

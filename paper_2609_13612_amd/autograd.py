"""torch.autograd functions over the C ABI: the fused attention (and its
block-sparse and bias / relu forms) and the norm and rotation of queries and
keys as differentiable operations for training code.

``attention`` runs attnfuse_fwd, keeps Q, K, V, O and the row statistic LSE
(Section 4.4: the forward saves one scalar per row), and its backward runs
attnfuse_bwd on the incoming gradient of O.  Argument marshalling only: every
step of the computation runs in the HIP kernels, and the gradients are exactly
those attnfuse_bwd returns.  ALiBi slopes, theta, the window and the scale get
no gradient.

A backward that is captured into a graph needs leaves of its own: torch keeps a
leaf's accumulation on the stream that first used it for as long as any eager
graph of that leaf lives, and work on that stream ends the capture.

There are no second derivatives: under create_graph the gradients are the same,
and a derivative of them raises a RuntimeError.
"""
import functools

import torch

from . import api


class _Once(torch.autograd.Function):
    """The first n tensors, as functions of the others that have no derivative."""
    @staticmethod
    def forward(ctx, n, *tensors):
        return tuple(t.data for t in tensors[:n])

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the gradients of these operations cannot be differentiated twice")


def _once(backward):
    """A Function's backward whose gradients come from kernels: under create_graph they depend on what they were formed
    from through _Once.  (torch's once_differentiable ties them to leaves of its own, and not at all where the incoming
    gradient is a constant: a gradient penalty's term would be lost without a word.)"""
    @functools.wraps(backward)
    def run(ctx, *grads):
        if not torch.is_grad_enabled():
            return backward(ctx, *grads)
        with torch.no_grad():
            out = backward(ctx, *grads)
        of = [t for t in (*grads, *ctx.saved_tensors) if t is not None and t.requires_grad]
        given = [x for x in out if x is not None]
        tied = iter(_Once.apply(len(given), *given, *of))
        return tuple(None if x is None else next(tied) for x in out)
    return run


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, alibi_slopes, rope, theta, mask, window, scale, sinks):
        o, lse = api.attnfuse_fwd(q, k, v, rope=rope, theta=theta, mask=mask, window=window,
                                  alibi_slopes=alibi_slopes, scale=scale, sinks=sinks)
        ctx.save_for_backward(q, k, v, o, lse, alibi_slopes)
        ctx.cfg = dict(rope=rope, theta=theta, mask=mask, window=window, scale=scale, sinks=sinks)
        ctx.mark_non_differentiable(lse)
        return o, lse

    @staticmethod
    @_once
    def backward(ctx, do, _dlse):
        q, k, v, o, lse, slopes = ctx.saved_tensors
        dq, dk, dv = api.attnfuse_bwd(q, k, v, o, do.contiguous(), lse, alibi_slopes=slopes, **ctx.cfg)
        return dq, dk, dv, None, None, None, None, None, None, None


class _BlockSparseAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, alibi_slopes, block_mask, rope, theta, mask, window, scale):
        o, lse = api.attnfuse_fwd_blocksparse(q, k, v, block_mask, rope=rope, theta=theta, mask=mask, window=window,
                                              alibi_slopes=alibi_slopes, scale=scale)
        ctx.save_for_backward(q, k, v, o, lse, alibi_slopes)
        ctx.block_mask = block_mask
        ctx.cfg = dict(rope=rope, theta=theta, mask=mask, window=window, scale=scale)
        ctx.mark_non_differentiable(lse)
        return o, lse

    @staticmethod
    @_once
    def backward(ctx, do, _dlse):
        q, k, v, o, lse, slopes = ctx.saved_tensors
        dq, dk, dv = api.attnfuse_bwd_blocksparse(q, k, v, o, do.contiguous(), lse, ctx.block_mask,
                                                  alibi_slopes=slopes, **ctx.cfg)
        return dq, dk, dv, None, None, None, None, None, None, None


class _BiasNormAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, bias, norm, rope, theta, mask, window, scale):
        o, lse = api.attnfuse_fwd_bias_norm(q, k, v, bias=bias, norm=norm, rope=rope, theta=theta, mask=mask,
                                            window=window, scale=scale)
        ctx.save_for_backward(q, k, v, o, lse, bias)
        ctx.cfg = dict(norm=norm, rope=rope, theta=theta, mask=mask, window=window, scale=scale)
        if lse is not None:
            ctx.mark_non_differentiable(lse)
        return o, lse

    @staticmethod
    @_once
    def backward(ctx, do, _dlse):
        q, k, v, o, lse, bias = ctx.saved_tensors
        dq, dk, dv = api.attnfuse_bwd_bias_norm(q, k, v, o, do.contiguous(), lse, bias=bias, **ctx.cfg)
        return dq, dk, dv, None, None, None, None, None, None, None


class _QkNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, rope_table, eps, rope, theta, max_positions):
        ctx.cfg = dict(eps=eps, rope=rope, theta=theta, max_positions=max_positions)
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, rope_table)
        return api.attnfuse_qknorm_rope(q, k, q_weight, k_weight, positions=positions, rope_table=rope_table, **ctx.cfg)

    @staticmethod
    @_once
    def backward(ctx, dqr, dkr):
        q, k, qw, kw, positions, table = ctx.saved_tensors
        want = ctx.needs_input_grad
        dq, dk, dqw, dkw = api.attnfuse_qknorm_rope_bwd(
            q, k, dqr.contiguous(), None if k is None else dkr.contiguous(), qw, kw, positions=positions, rope_table=table,
            weight_grads=want[2] or want[3], **ctx.cfg)
        return dq, dk, dqw if want[2] else None, dkw if want[3] else None, None, None, None, None, None, None


def qknorm_rope(q, k=None, q_weight=None, k_weight=None, *, eps=1e-6, rope="neox", theta=10000.0, positions=None,
                max_positions=None, rope_table=None):
    """Differentiable norm and rotation of query and key rows: (Qr, Kr), or Qr without k; gradients for q, k and the
    weights.  Arguments as api.attnfuse_qknorm_rope."""
    if api._native is not None:   # the same function, its backward in C++
        r = api._native.qknorm_grad(q, k, q_weight, k_weight, positions, rope_table, api._TABLES, eps, api.ROPE.get(rope, -1),
                                    theta, max_positions)
        if r is not None:
            qr, kr = api._result(r, "attnfuse_qknorm_rope")
            return qr if k is None else (qr, kr)
    qr, kr = _QkNormRope.apply(q, k, q_weight, k_weight, positions, rope_table, eps, rope, theta, max_positions)
    return qr if k is None else (qr, kr)


def attention(q, k, v, *, rope="none", theta=10000.0, mask="causal", window=None, alibi_slopes=None, scale=None,
              return_lse=False, sinks=0):
    """Differentiable fused attention: O [B, H, S, D] (and the non-differentiable
    LSE [B, H, S] with ``return_lse``); arguments as api.attnfuse_fwd."""
    if sinks and api._native is not None:   # the same function, its backward in C++
        window, sinks = api._need_sinks(sinks, mask, window, alibi_slopes)
        r = api._native.sinks_grad(q, k, v, None, api._TABLES, api.ROPE.get(rope, -1), theta, window, sinks, scale)
        if r is not None:
            o, lse = api._result(r, "attnfuse_fwd_sinks")
            return (o, lse) if return_lse else o
    o, lse = _Attention.apply(q, k, v, alibi_slopes, rope, theta, mask, window, scale, sinks)
    return (o, lse) if return_lse else o


def blocksparse_attention(q, k, v, block_mask, *, rope="none", theta=10000.0, mask="none", window=None,
                          alibi_slopes=None, scale=None, return_lse=False):
    """Differentiable block-sparse attention over a blockmask.BlockMask;
    arguments as api.attnfuse_fwd_blocksparse."""
    o, lse = _BlockSparseAttention.apply(q, k, v, alibi_slopes, block_mask, rope, theta, mask, window, scale)
    return (o, lse) if return_lse else o


def attention_bias_norm(q, k, v, *, bias=None, norm="softmax", rope="none", theta=10000.0, mask="causal",
                        window=None, scale=None, return_lse=False):
    """Differentiable attention with a dense additive bias tensor and softmax or
    relu normalisation; arguments as api.attnfuse_fwd_bias_norm (the bias gets
    no gradient; under relu attention LSE is None)."""
    o, lse = _BiasNormAttention.apply(q, k, v, bias, norm, rope, theta, mask, window, scale)
    return (o, lse) if return_lse else o

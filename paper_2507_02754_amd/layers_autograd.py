"""torch.autograd wrappers of the entry points of include/simplicial_layers.h.

No arithmetic of their own: forwards and backwards are the library's, through
`layers_binding`. Inputs whose strides the kernels do not take (rows that are not
16-byte aligned, a last dimension that is not contiguous) are copied first.
"""

import collections

import torch

from .layers_binding import (simplicial_dot_attn_bwd, simplicial_dot_attn_fwd, simplicial_logprobs_bwd,
                             simplicial_logprobs_fwd, simplicial_norm_rotate_bwd, simplicial_norm_rotate_fwd)

__all__ = ["norm_rotate", "dot_attention", "token_logprobs", "TokenLogprobs", "NormRotateFunction", "DotAttentionFunction",
           "TokenLogprobsFunction"]


def _rows(t):
    """`t`, or a contiguous copy where its rows are not 16-byte aligned."""
    unit = 16 // t.element_size()
    if t.dim() == 4 and (t.stride(3) != 1 or t.data_ptr() % 16 or
                         any(s % unit for s, n in zip(t.stride()[:3], t.shape) if n > 1)):
        return t.contiguous() if not t.is_contiguous() else t.clone()
    return t


def _needs_grad(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


class NormRotateFunction(torch.autograd.Function):
    """ys = norm and rotation of the first `count` of `tensors`, with the rest as their weights."""

    @staticmethod
    def forward(ctx, options, count, *tensors):
        xs, weights = [_rows(x) for x in tensors[:count]], tensors[count:] or None
        ys = simplicial_norm_rotate_fwd(xs, weights, **options)
        ctx.save_for_backward(*xs, *(weights or ()))
        ctx.options, ctx.count = options, count
        return tuple(ys)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *dys):
        tensors = ctx.saved_tensors
        xs, weights = tensors[:ctx.count], tensors[ctx.count:] or None
        dys = [torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else _dense(dy, x.dtype)
               for x, dy in zip(xs, dys)]
        dxs, dws = simplicial_norm_rotate_bwd(xs, dys, weights, weight_grads=any(ctx.needs_input_grad[2 + ctx.count:]),
                                              **ctx.options)
        return (None, None, *dxs, *(dws if weights else ()))


def _dense(g, dtype):
    """An upstream gradient as the kernels take it: contiguous and aligned, of the output's type."""
    g = g.to(dtype).contiguous()
    return g if g.data_ptr() % 16 == 0 else g.clone()


def norm_rotate(xs, weights=None, eps=1e-6, freqs=None, layout="half", positions=None, start=0):
    """RMS norm of each head and position rotation of one to three tensors (queries,
    keys, K'), with autograd support for them and for the weights.

    xs[t] is [B, N, heads_t, D]; arguments as simplicial_norm_rotate_fwd, whose results
    are returned as a tuple. eps = 0 without weights is the L2 norm scaled by sqrt(D). A
    weight is given for every tensor or for none."""
    options = dict(eps=eps, freqs=freqs, layout=layout, positions=positions, start=start)
    xs = list(xs)
    if weights is not None and any(w is None for w in weights):
        raise ValueError("a weight for every tensor, or weights=None")
    if _needs_grad(*xs, *(weights or ())):
        return NormRotateFunction.apply(options, len(xs), *xs, *(weights or ()))
    return tuple(simplicial_norm_rotate_fwd([_rows(x) for x in xs], weights, **options))


class DotAttentionFunction(torch.autograd.Function):
    """(O, LSE) of dot-product attention; LSE is returned without a gradient."""

    @staticmethod
    def forward(ctx, q, k, v, options):
        q, k, v = _rows(q), _rows(k), _rows(v)
        out, lse = simplicial_dot_attn_fwd(q, k, v, **options)
        ctx.save_for_backward(q, k, v, out, lse)
        ctx.options = options
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, _dlse):
        q, k, v, out, lse = ctx.saved_tensors
        if dout is None:
            dout = torch.zeros_like(out)
        return (*simplicial_dot_attn_bwd(q, k, v, out, _dense(dout, out.dtype), lse, **ctx.options), None)


def dot_attention(q, k, v, scale=None, causal=True, window=0, softcap=0.0, slopes=None, documents=None, prefix=None,
                  k_lens=None):
    """O = dot-product attention(Q, K, V) with autograd support for Q, K and V.

    Arguments as simplicial_dot_attn_fwd: q [B, Nq, H, D], k and v [B, Nk, Hkv, D], the
    queries the last Nq of the keys' positions; score cap, distance bias, and causal,
    window, prefix and document masks. The options are not differentiated."""
    options = dict(scale=scale, causal=causal, window=window, softcap=softcap, slopes=slopes, documents=documents,
                   prefix=prefix, k_lens=k_lens)
    if slopes is not None and slopes.requires_grad:
        raise ValueError("the slopes of the distance bias get no gradient")
    if _needs_grad(q, k, v):
        return DotAttentionFunction.apply(q, k, v, options)[0]
    return simplicial_dot_attn_fwd(_rows(q), _rows(k), _rows(v), **options)[0]


TokenLogprobs = collections.namedtuple("TokenLogprobs", "logprob entropy lse top_logprobs top_tokens")


class TokenLogprobsFunction(torch.autograd.Function):
    """The results of simplicial_logprobs_fwd; the top tokens and their log
    probabilities are returned without a gradient."""

    @staticmethod
    def forward(ctx, logits, targets, top):
        results = simplicial_logprobs_fwd(logits, targets, top)
        ctx.save_for_backward(logits, targets, results[2], results[1])
        ctx.mark_non_differentiable(*results[3:])
        ctx.set_materialize_grads(False)
        return results

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_logprob, d_entropy, d_lse, _dtop, _dindex):
        logits, targets, lse, entropy = ctx.saved_tensors
        grads = [None if g is None else g.contiguous() for g in (d_logprob, d_entropy, d_lse)]
        return simplicial_logprobs_bwd(logits, targets, lse, entropy, *grads), None, None


def token_logprobs(logits, targets, top=0):
    """Log probabilities of given tokens, with entropy and top alternatives, and with
    autograd support (logprob, entropy and lse).

    logits [..., V], targets [...] int64 (negative: left out, logprob 0). Returns a
    TokenLogprobs of logprob, entropy, lse ([...] float32), top_logprobs and top_tokens
    ([..., top]), as simplicial_logprobs_fwd."""
    lead, V = logits.shape[:-1], logits.shape[-1]
    if targets.shape != lead:
        raise ValueError(f"targets have shape {tuple(targets.shape)}, expected {tuple(lead)}")
    rows, flat = logits.reshape(-1, V), targets.reshape(-1)
    if V > 1 and rows.stride(1) != 1 or (rows.shape[0] > 1 and rows.stride(0) < V):
        rows = rows.contiguous()
    if not flat.is_contiguous():
        flat = flat.contiguous()
    if _needs_grad(rows):
        r = TokenLogprobsFunction.apply(rows, flat, int(top))
    else:
        r = simplicial_logprobs_fwd(rows, flat, top)
    if len(lead) == 1:
        return TokenLogprobs(*r)
    return TokenLogprobs(*(t.view(lead) for t in r[:3]), *(t.view(*lead, int(top)) for t in r[3:]))

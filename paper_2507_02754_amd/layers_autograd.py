"""torch.autograd wrappers of the entry points of include/simplicial_layers.h.

No arithmetic of their own: forwards and backwards are the library's, through
`layers_binding`. Inputs whose strides the kernels do not take (rows that are not
16-byte aligned, a last dimension that is not contiguous) are copied first.
"""

import collections

import torch
from torch.autograd import forward_ad

from .layers_binding import _DotCall, _RotateCall, rotary_angles, simplicial_logprobs_bwd, simplicial_logprobs_fwd

__all__ = ["norm_rotate", "dot_attention", "token_logprobs", "TokenLogprobs", "NormRotateFunction", "DotAttentionFunction",
           "TokenLogprobsFunction"]


def _rows(t):
    """`t`, or a contiguous copy where its rows are not 16-byte aligned."""
    if t.dim() != 4 or (t.is_contiguous() and t.data_ptr() % 16 == 0):
        return t
    unit = 16 // t.element_size()
    if t.stride(3) != 1 or t.data_ptr() % 16 or any(s % unit for s, n in zip(t.stride()[:3], t.shape) if n > 1):
        return t.contiguous() if not t.is_contiguous() else t.clone()
    return t


def _needs_grad(*tensors):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


# Without gradients the calls below go past their Functions, which would refuse a tensor of
# forward-mode differentiation; its values alone would give a result without a tangent, read as a
# derivative of zero.
def _refuse_tangents(name, *tensors):
    if forward_ad._current_level < 0:  # (none has a tangent: a microsecond of a token's call)
        return
    for t in tensors:
        if isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None:
            raise NotImplementedError(f"{name} has no forward-mode derivative")


# Options enter the kernels as numbers: one that asks for a gradient would stay as it is in training.
def _refuse_gradients(name, *options):
    if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in options):
        raise ValueError(f"{name}: no gradient; pass what does not require one")


# A Function keeps the tensors of its call with save_for_backward alone, which notices
# changes in place and lets hooks put them elsewhere meanwhile; the checked arguments serve the
# backward where the tensors come back to the same places.
def _save(ctx, call, options, tensors):
    ctx.save_for_backward(*[t for t in tensors if t is not None])
    ctx.present = [t is not None for t in tensors]
    ctx.call, ctx.options, ctx.places = call, options, call.places()
    call.kept = None


def _saved(ctx):
    tensors = iter(ctx.saved_tensors)
    return [next(tensors) if there else None for there in ctx.present]


class NormRotateFunction(torch.autograd.Function):
    """ys = norm and rotation of the first `count` of `tensors`, with the rest as their weights."""

    @staticmethod
    def forward(ctx, options, count, *tensors):
        xs, weights = [_rows(x) for x in tensors[:count]], tensors[count:] or None
        call = _RotateCall(xs, weights, *options)
        ys = call.forward()
        _save(ctx, call, options, [*xs, *(weights or ()), options[3]])
        ctx.count = count
        return tuple(ys)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *dys):
        call, count, options = ctx.call, ctx.count, ctx.options
        *tensors, positions = _saved(ctx)
        xs, weights = tensors[:count], tensors[count:] or None
        call.kept = (xs, weights, positions)
        if call.places() != ctx.places:
            call = _RotateCall(xs, weights, *options[:3], positions, *options[4:])
        dys = [torch.zeros(s, dtype=call.dtype, device=call.device) if dy is None else _dense(dy, call.dtype)
               for s, dy in zip(call.shapes, dys)]
        dxs, dws = call.backward(dys, weight_grads=any(ctx.needs_input_grad[2 + count:]))
        ctx.call.kept = None
        return (None, None, *dxs, *(dws if weights else ()))


def _dense(g, dtype):
    """An upstream gradient as the kernels take it: contiguous and aligned, of the output's type."""
    if g.dtype != dtype or not g.is_contiguous():
        g = g.to(dtype).contiguous()
    return g if g.data_ptr() % 16 == 0 else g.clone()


def norm_rotate(xs, weights=None, eps=1e-6, freqs=None, layout="half", positions=None, start=0):
    """RMS norm of each head and position rotation of one to three tensors (queries,
    keys, K'), with autograd support for them and for the weights.

    xs[t] is [B, N, heads_t, D]; arguments as simplicial_norm_rotate_fwd, whose results
    are returned as a tuple. eps = 0 without weights is the L2 norm scaled by sqrt(D). A
    weight is given for every tensor or for none. eps and freqs are not differentiated (refused
    where they ask for a gradient)."""
    xs, weights = list(xs), None if weights is None else list(weights)
    _refuse_tangents("norm_rotate", *xs, *(weights or ()))

    def check(*given):
        _refuse_tangents("norm_rotate", *given)
        _refuse_gradients("eps and freqs", *given)

    check(eps)
    options = (eps, rotary_angles(freqs, check), layout, positions, start)
    if weights is not None and (len(weights) != len(xs) or any(w is None for w in weights)):
        raise ValueError("a weight for every tensor, or weights=None")
    if _needs_grad(*xs, *(weights or ())):
        return NormRotateFunction.apply(options, len(xs), *xs, *(weights or ()))
    return tuple(_RotateCall([_rows(x) for x in xs], weights, *options).forward())


class DotAttentionFunction(torch.autograd.Function):
    """(O, LSE) of dot-product attention; LSE is returned without a gradient."""

    @staticmethod
    def forward(ctx, q, k, v, options):
        q, k, v = _rows(q), _rows(k), _rows(v)
        call = _DotCall(q, k, v, *options)
        lo = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q.dtype == torch.bfloat16 else None
        out, lse = call.forward(out_lo=lo)
        _save(ctx, call, options, [q, k, v, out, lse, lo, *options[4:]])
        call.q = call.k = call.v = None
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, _dlse):
        call = ctx.call
        q, k, v, out, lse, lo, *masks = _saved(ctx)
        call.q, call.k, call.v, call.kept = q, k, v, masks
        if call.places() != ctx.places:
            call = _DotCall(q, k, v, *ctx.options[:4], *masks)
        dout = torch.zeros_like(out) if dout is None else _dense(dout, out.dtype)
        grads = call.backward(out, dout, lse, lo)
        ctx.call.q = ctx.call.k = ctx.call.v = ctx.call.kept = None
        return (*grads, None)


def dot_attention(q, k, v, scale=None, causal=True, window=0, softcap=0.0, slopes=None, documents=None, prefix=None,
                  k_lens=None):
    """O = dot-product attention(Q, K, V) with autograd support for Q, K and V.

    Arguments as simplicial_dot_attn_fwd: q [B, Nq, H, D], k and v [B, Nk, Hkv, D], the
    queries the last Nq of the keys' positions; score cap, distance bias, and causal,
    window, prefix and document masks. The options are not differentiated (those that ask for
    a gradient are refused). bfloat16 tensors have their probabilities rounded to bfloat16 for
    the products, float32 ones do not."""
    options = (scale, causal, window, softcap, slopes, documents, prefix, k_lens)
    _refuse_tangents("dot_attention", q, k, v, scale, softcap, slopes)
    _refuse_gradients("scale, softcap and slopes", scale, softcap, slopes)
    if _needs_grad(q, k, v):
        return DotAttentionFunction.apply(q, k, v, options)[0]
    return _DotCall(_rows(q), _rows(k), _rows(v), *options).forward()[0]


TokenLogprobs = collections.namedtuple("TokenLogprobs", "logprob entropy lse top_logprobs top_tokens")


class TokenLogprobsFunction(torch.autograd.Function):
    """The results of simplicial_logprobs_fwd; the top tokens and their log
    probabilities are returned without a gradient."""

    @staticmethod
    def forward(ctx, logits, targets, top):
        logprob, entropy, both, *best = simplicial_logprobs_fwd(logits, targets, top, lse_lo=True)
        lse = both[0].data  # (a tensor of its own: results may not be views; saved for the check of changes in place)
        results = (logprob, entropy, lse, *best)
        ctx.save_for_backward(logits, targets, both, entropy, lse)
        ctx.mark_non_differentiable(*results[3:])
        ctx.set_materialize_grads(False)
        return results

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_logprob, d_entropy, d_lse, _dtop, _dindex):
        logits, targets, lse, entropy, _ = ctx.saved_tensors
        grads = [None if g is None else g.contiguous() for g in (d_logprob, d_entropy, d_lse)]
        return simplicial_logprobs_bwd(logits, targets, lse, entropy, *grads), None, None


def token_logprobs(logits, targets, top=0):
    """Log probabilities of given tokens, with entropy and top alternatives, and with
    autograd support (logprob, entropy and lse).

    logits [..., V], targets [...] int64 (negative: left out, logprob 0). Returns a
    TokenLogprobs of logprob, entropy, lse ([...] float32), top_logprobs and top_tokens
    ([..., top]), as simplicial_logprobs_fwd."""
    _refuse_tangents("token_logprobs", logits)
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

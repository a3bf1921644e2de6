"""Plain float64 implementations of the operators of include/simplicial_layers.h, with
bounds of what rounding may add, element by element. Test infrastructure: they share
no code with the library.

Bounds count roundings: one to a type of b mantissa bits is off by at most
torch.finfo(type).eps / 2 relative to the value (bf16 2^-8, float32 2^-24).
"""

import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24  # float32


def close(got, want, bound, what):
    """|got - want| <= bound element by element, infinities and NaN in the same places."""
    got, want, bound = (t.detach().double().cpu() for t in (got, want, bound))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), f"{what}: infinities differ"
    assert torch.isfinite(got[fine]).all(), f"{what}: not finite"
    over = (got - want).abs()[fine] - bound[fine]
    assert over.numel() == 0 or over.max() <= 0, \
        f"{what}: {int((over > 0).sum())} of {over.numel()} values beyond their bound, by up to {over.max():.3g}"


# ---- norm and rotation ----


def rotate_pairs(layout, n):
    i = torch.arange(n)
    return {"half": (i, n + i), "pairs": (2 * i, 2 * i + 1), "axis": (3 * i, 3 * i + 1)}[layout]


def turn(t, positions, freqs, layout, sign=1.0):
    """t [B, N, H, D] float64, positions [B, N]."""
    n = len(freqs)
    if n == 0:
        return t.clone()
    angle = sign * positions.double()[..., None] * torch.tensor(freqs, dtype=torch.float64, device=t.device)
    c, s = angle.cos()[:, :, None], angle.sin()[:, :, None]
    first, second = (x.to(t.device) for x in rotate_pairs(layout, n))
    out = t.clone()
    a, b = t[..., first], t[..., second]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    return out


def norm_rotate(x, weight, eps, freqs, layout, positions, dy=None):
    """(y, its bound), and with dy also ((dx, bound), (dweight, bound) or None)."""
    half = HALF[x.dtype]
    D = x.shape[-1]
    xd = x.double()
    ms = xd.square().mean(-1, keepdim=True)
    r = torch.ones_like(ms)
    if eps is not None:
        r = torch.where(ms + eps > 0, (ms + eps).clamp(min=1e-300) ** -0.5, 0.0)
    w = torch.ones(D, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    u = xd * r * w
    y = turn(u, positions, freqs, layout)
    # float32 before the rounding: r is off by (D / 16 + 8) U, every product by U, sine and
    # cosine by 4 U (a fraction of a turn rounded to 24 bits, times 2 pi), a sum by U.
    big = u.abs().amax(-1, keepdim=True)
    f32 = (D / 16 + 24) * U
    yb = half * y.abs() + 2 * f32 * big
    if dy is None:
        return y, yb
    g = turn(dy.double(), positions, freqs, layout, -1.0)
    gb = 16 * U * dy.double().abs().amax(-1, keepdim=True) + 0 * g
    dw = None
    if weight is not None:
        t = g * xd * r
        # each term off by (f32 + 16 U); sums of at most (B N H) terms in chains of a few
        # hundred, each addition off by U of the absolute sum
        terms = (t.abs() * f32 + gb * (xd * r).abs()).sum((0, 1, 2))
        dw = ((t.sum((0, 1, 2))), HALF[weight.dtype] * t.sum((0, 1, 2)).abs() + terms + 600 * U * t.abs().sum((0, 1, 2)))
    gw = g * w
    if eps is None:
        dx, db = gw, gb * w.abs()
    else:
        dot = (gw * xd).mean(-1, keepdim=True)
        dx = r * (gw - xd * r * r * dot)
        size = (gw * xd).abs().mean(-1, keepdim=True)
        db = r * (gb * w.abs() + f32 * gw.abs() + xd.abs() * r * r * (gb * w.abs() * xd.abs()).mean(-1, keepdim=True)
                  + 3 * f32 * xd.abs() * r * r * size) + f32 * dx.abs()
    return y, yb, (dx, half * dx.abs() + db), dw


# ---- dot-product attention ----


def visible(B, Nq, Nk, causal=True, window=0, documents=None, prefix=None, k_lens=None, device="cpu"):
    """bool [B, Nq, Nk] by the definition, and |p - j|."""
    j = torch.arange(Nk, device=device)[None, None]
    L = torch.full((B,), Nk, device=device) if k_lens is None else k_lens.to(device).long().clamp(0, Nk)
    p = (L[:, None] - Nq + torch.arange(Nq, device=device))[:, :, None]
    near = torch.ones((B, Nq, Nk), dtype=torch.bool, device=device)
    if causal:
        near = near & (j <= p)
    if window:
        near = near & ((p - j).abs() < window)
    if prefix is not None:
        near = near | (j < prefix.to(device).long()[:, None, None])
    see = near & (p >= 0) & (j < L[:, None, None])
    if documents is not None:
        ids = documents.to(device).long()
        mine = ids.gather(1, p[..., 0].clamp(0, Nk - 1))
        see = see & (mine[:, :, None] == ids[:, None, :]) & (ids >= 0)[:, None, :]
    return see, (p - j).abs().double()


def dot_attention(q, k, v, scale=None, causal=True, window=0, softcap=0.0, slopes=None, documents=None, prefix=None,
                  k_lens=None, dout=None):
    """{name: (value, bound)} of out, lse and, with dout, dq, dk, dv. Masked pairs do not
    enter (their values may be anything)."""
    dt, dev = q.dtype, q.device
    B, Nq, H, D = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    see, distance = visible(B, Nq, Nk, causal, window, documents, prefix, k_lens, dev)
    see, distance = see[:, None], distance[:, None]
    qd = q.double().transpose(1, 2)
    kd, vd = (t.double().transpose(1, 2).repeat_interleave(H // Hkv, 1) for t in (k, v))
    # a key or query that nothing sees may hold anything
    kseen, qseen = see.any(2)[..., None], see.any(3)[..., None]
    kd, vd, qd = torch.where(kseen, kd, 0.0), torch.where(kseen, vd, 0.0), torch.where(qseen, qd, 0.0)
    s = qd @ kd.transpose(2, 3) * scale
    mag = qd.abs() @ kd.abs().transpose(2, 3) * abs(scale)
    a, dcap = s, torch.ones_like(s)
    if softcap:
        t = torch.tanh(s / softcap)
        a, dcap = softcap * t, 1 - t * t
    if slopes is not None:
        a = a - slopes.double()[None, :, None, None] * distance
    lse = torch.logsumexp(torch.where(see, a, -math.inf), 3)
    p = torch.where(see, torch.exp(a - torch.where(torch.isinf(lse), 0.0, lse)[..., None]), 0.0)
    out = p @ vd
    # A score is off by (D / 2 + 8) U of its terms' absolute sum, the cap by 16 U softcap, the
    # distance's product by 2 U of itself: da. A probability by twice that and the exponent's 4 U (1 + |a - lse|).
    half = HALF[dt]
    low = half if dt == torch.bfloat16 else 0.0  # P and dS are rounded to bf16 for their products
    da = (D / 2 + 8) * U * mag + 16 * U * softcap + 4 * U * (1 + a.abs())
    if slopes is not None:
        da = da + 4 * U * slopes.double()[None, :, None, None].abs() * distance
    da = torch.where(see, da, 0.0)
    rp = 2 * da.amax(3, keepdim=True) + 8 * U * torch.where(see, 1 + (a - lse[..., None]).abs(), 0.0)
    rp = torch.where(see, rp, 0.0)
    chain = (Nk / 32 + 64) * U  # sums of blocks of 32
    sums = (p * (rp + low + chain)) @ vd.abs()
    res = {"out": (out.transpose(1, 2), (half * out.abs() + 1.01 * sums).transpose(1, 2)),
           "lse": (lse, torch.where(torch.isinf(lse), 0.0, da.amax(3) + chain + 4 * U * (1 + lse.abs())))}
    if dout is None:
        return res
    do = torch.where(qseen, dout.double().transpose(1, 2), 0.0)
    dp = do @ vd.transpose(2, 3)
    dpm = do.abs() @ vd.abs().transpose(2, 3)
    delta = (do * out).sum(-1, keepdim=True)
    # Delta from the rounded output
    ddelta = (do.abs() * (half * out.abs() + 1.01 * sums)).sum(-1, keepdim=True) + D * U * (do * out).abs().sum(-1, keepdim=True)
    ds = p * (dp - delta) * dcap * scale
    ddcap = 32 * U + 2 * da / softcap if softcap else 0.0
    dds = abs(scale) * p * ((dp - delta).abs() * (dcap * (rp + 8 * U) + ddcap) + dcap * ((D / 2 + 8) * U * dpm + ddelta)) + low * ds.abs()
    chq = (H // Hkv * Nq / 32 + 64) * U

    def group(t):
        return t.view(B, Hkv, H // Hkv, Nk, D).sum(2).transpose(1, 2)

    dq, dqb = ds @ kd, (dds + chain * ds.abs()) @ kd.abs()
    dst, ddst, pt = ds.transpose(2, 3), (dds + chq * ds.abs()).transpose(2, 3), p.transpose(2, 3)
    dk, dkb = group(dst @ qd), group(ddst @ qd.abs())
    dv, dvb = group(pt @ do), group((p * (rp + low + chq)).transpose(2, 3) @ do.abs())
    dq, dqb = dq.transpose(1, 2), dqb.transpose(1, 2)
    for name, x, b in (("dq", dq, dqb), ("dk", dk, dkb), ("dv", dv, dvb)):
        res[name] = (x, half * x.abs() + 1.01 * b + 1e-30)
    return res


# ---- log probabilities ----


def logprobs(x, targets, top=0, grads=None):
    """{name: (value, bound)}: logprob, entropy, lse, top_logprob, top_index (exact), and with
    grads (d_logprob, d_entropy, d_lse; [R] each) dx."""
    R, V = x.shape
    xd = x.double()
    lse = torch.logsumexp(xd, 1)
    none = torch.isinf(lse) & (lse < 0)
    logp = torch.where(none[:, None], -math.inf, xd - torch.where(none, 0.0, lse)[:, None])
    p = torch.exp(logp)
    plogp = torch.where(p > 0, p * logp, torch.where(torch.isnan(p), p, 0.0))
    entropy = torch.where(none, 0.0, -plogp.sum(1))
    at = targets.clamp(0, V - 1)
    lp = logp.gather(1, at[:, None])[:, 0]
    lp = torch.where(targets < 0, 0.0, torch.where(targets >= V, math.nan, lp))
    # An exponential is off by 4 U (1 + |log p|), sums of V terms in chains of 128 and a tree by 160 U.
    size = torch.where(p > 0, p * logp.abs(), 0.0).sum(1)
    rel = 164 * U + 4 * U * (1 + size)
    top_x = torch.where(torch.isinf(xd), 0.0, xd).abs().amax(1)
    lse_b = rel + 2 * U * (top_x + lse.abs().nan_to_num(0, 0, 0))
    spread = torch.where(p > 0, p * logp * logp, 0.0).sum(1)
    ent_b = 2 * rel * (1 + size) + 4 * U * spread + 4 * U * (1 + lse.abs().nan_to_num(0, 0, 0))
    zero = torch.zeros_like(lse)
    res = {"lse": (lse, lse_b), "entropy": (entropy, ent_b),
           "logprob": (lp, lse_b + 2 * U * lp.abs().nan_to_num(0, 0, 0))}
    if top:
        # NaN first, then descending, equal ones by ascending token
        key = torch.where(torch.isnan(xd), math.inf, xd)
        order = torch.sort(key + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
        res["top_index"] = order
        tl = logp.gather(1, order)
        res["top_logprob"] = (tl, lse_b[:, None] + 2 * U * tl.abs().nan_to_num(0, 0, 0))
    if grads is not None:
        glp, gh, gl = (zero if g is None else g.double() for g in grads)
        glp = torch.where(targets < 0, 0.0, glp)
        dx = torch.where(p > 0, p * ((gl - glp)[:, None] - gh[:, None] * (logp + entropy[:, None])), 0.0)
        dx = torch.where(torch.isnan(p), p, dx)
        hit = torch.zeros_like(dx).scatter_(1, at[:, None], torch.where((targets >= 0) & (targets < V), glp, 0.0)[:, None])
        size = p * ((gl - glp).abs()[:, None] + gh.abs()[:, None] * (torch.where(p > 0, logp.abs(), 0.0) + entropy.abs()[:, None]))
        err = (lse_b + ent_b)[:, None] + 8 * U * (1 + torch.where(p > 0, logp.abs(), 0.0))
        dx = dx + hit
        dx = torch.where(none[:, None], 0.0, torch.where((targets >= V)[:, None], math.nan, dx))
        res["dx"] = (dx, HALF[x.dtype] * dx.abs() + 2 * err * size + (lse_b + ent_b)[:, None] * gh.abs()[:, None] * p + 4 * U * hit.abs() + 2.0 ** -126)
    return res

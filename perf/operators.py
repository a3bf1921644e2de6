"""The operators of the layers around 2-simplicial attention, as a program calls them.

  norm_rotate      RMS norm of each head's queries and keys and their position rotation
  dot_attention    attention with capped scores, distance bias, document / prefix / window masks
  token_logprobs   log probabilities of given tokens, entropy and top alternatives

`run` computes a case in plain torch operations (`own` false) or through the
package (`own` true):

  listed()             the named cases
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  what a program holds before the call
  run(state)           one pass; returns every output
  work(case)           bytes and FLOPs the pass cannot do without
  exact(case, seed)    the outputs in float64

Fields of a case: `op` ("rotate", "attn", "logprobs"), `train` (forward and
backward, else the forward alone), `dtype`, and the sizes of the operator:
  rotate    B, N, heads of q, k and k' (H, Hk, Hp; Hp 0: no k'), D, layout, freqs
            (angles per position), norm, weight, far (largest first position),
            fused (q, k, k' are slices of one projection's output)
  attn      B, Nq, Nk, H, Hk, D, causal, window, cap, alibi, docs (documents per
            row, with padding behind the last; 0: none), prefix (largest prefix
            length), lens (rows of a cache filled to different lengths)
  logprobs  R rows, V tokens, top
"""

import math

import torch

own = False


def _rotate(name, B, N, H, Hk, D, Hp=0, train=True, dtype="bf16", layout="half", freqs=None, norm=True, weight=True,
            far=0, fused=False):
    c = dict(op="rotate", B=B, N=N, H=H, Hk=Hk, Hp=Hp, D=D, train=train, dtype=dtype, layout=layout,
             freqs=freqs or (D // 3 if layout == "axis" else D // 2), norm=norm, weight=weight, far=far, fused=fused)
    return dict(c, name=name) if name else c


def _attn(name, B, Nq, Nk, H, Hk, D, train=True, dtype="bf16", causal=True, window=0, cap=0.0, alibi=False, docs=0,
          prefix=0, lens=False):
    c = dict(op="attn", B=B, Nq=Nq, Nk=Nk, H=H, Hk=Hk, D=D, train=train, dtype=dtype, causal=causal, window=window,
             cap=cap, alibi=alibi, docs=docs, prefix=prefix, lens=lens)
    return dict(c, name=name) if name else c


def _logprobs(name, R, V, train=True, dtype="bf16", top=0):
    c = dict(op="logprobs", R=R, V=V, train=train, dtype=dtype, top=top)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token of four sequences, far into their contexts: latency.
        _rotate("rotate_token", 4, 1, 16, 4, 128, train=False, far=120000),
        # The training step of the 8k workload: q and k normed with learned weights.
        _rotate("rotate_train_8k", 2, 8192, 8, 8, 128, fused=True),
        # q, k and k' of the determinant logits, rotated about an axis of each
        # 3-component chunk, without weights; a ragged length, grouped heads.
        _rotate("rotate_axis", 1, 6001, 16, 4, 128, Hp=4, layout="axis", weight=False),
        # One new token of eight sequences over a cache filled to different lengths.
        _attn("attn_token", 8, 1, 16384, 16, 4, 128, train=False, cap=30.0, lens=True),
        # A prompt of 4096 tokens whose first part all positions see.
        _attn("attn_prompt_4k", 1, 4096, 4096, 8, 8, 128, train=False, prefix=1024),
        # The training step on packed documents, grouped heads: the largest.
        _attn("attn_train_docs", 1, 8192, 8192, 16, 4, 128, docs=3, cap=50.0),
        # The training step of a window with a distance bias, short heads.
        _attn("attn_train_window", 2, 4093, 4093, 16, 16, 64, window=512, alibi=True),
        # A training step in float32 (a layer whose attention runs in float32).
        _attn("attn_train_fp32", 1, 2000, 2000, 4, 4, 64, dtype="fp32", prefix=200),
        # Sampling: the next token's distribution of eight sequences.
        _logprobs("logprobs_token", 8, 50001, train=False, top=8),
        # Scoring a text of 2048 tokens with its alternatives.
        _logprobs("logprobs_score", 2047, 32000, train=False, top=5),
        # The loss of a training step over 8192 tokens, with the entropy.
        _logprobs("logprobs_train", 8192, 65536),
        # The loss of the small interleaved stack: vocabulary 512, float32.
        _logprobs("logprobs_small", 510, 512, dtype="fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_FLOPS = 4.5e11  # of a drawn attention case: the largest listed one's
MOST_SCORES = 1 << 30  # of one, over all heads, seen or not: likewise (the plain form holds them several times)
MOST_LOGITS = 1 << 30  # bytes of the logits: likewise


def draw(rng):
    op = rng.choice(["rotate", "attn", "attn", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "rotate":
        D, layout = rng.choice([16, 32, 64, 128, 128]), rng.choice(["half", "half", "pairs", "axis"])
        train = rng.random() < 0.7
        B, N = rng.choice([1, 2, 3]), _log(rng, 1, 9000)
        H = rng.choice([4, 8, 16])
        Hk = H // rng.choice([1, 2, 4])
        full = D // 3 if layout == "axis" else D // 2
        freqs = rng.choice([full, full, 8 * rng.randint(1, D // 16) if layout == "half" else rng.randint(1, full)])
        norm = rng.random() < 0.85
        return _rotate("", B, N, H, Hk, D, Hp=rng.choice([0, 0, Hk]), train=train, dtype=dtype, layout=layout, freqs=freqs,
                       norm=norm, weight=norm and rng.random() < 0.6, far=rng.choice([0, 0, 5000, 1000000]),
                       fused=rng.random() < 0.5)
    if op == "logprobs":
        V = _log(rng, 2, 120000)
        train = rng.random() < 0.6
        R = min(_log(rng, 1, 8192 if train else 4096), MOST_LOGITS // (V * (4 if dtype == "fp32" else 2)))
        return _logprobs("", R, V, train=train, dtype=dtype, top=0 if train else min(V, rng.choice([0, 1, 5, 20, 32])))
    D, H = rng.choice([16, 32, 64, 64, 128, 128, 128]), rng.choice([4, 8, 16])
    Hk = H // rng.choice([1, 2, 4])
    cap, alibi = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.25
    if rng.random() < 0.3:  # new tokens over a cache
        return _attn("", rng.choice([1, 2, 8, rng.randint(3, 16)]), rng.choice([1, 1, rng.randint(2, 9)]), _log(rng, 16, 16384),
                     H, Hk, D, train=False, dtype=dtype, cap=cap, alibi=alibi, window=rng.choice([0, 0, rng.randint(64, 2000)]),
                     lens=rng.random() < 0.8)
    B, N = rng.choice([1, 1, 2]), _log(rng, 1, 8192)
    mask = rng.choice(["causal", "docs", "prefix", "window", "all"])
    N = min(N, int((MOST_SCORES / (B * H)) ** 0.5))
    c = _attn("", B, N, N, H, Hk, D, train=rng.random() < 0.7, dtype=dtype, causal=mask != "all", cap=cap, alibi=alibi,
              docs=rng.randint(1, 6) if mask == "docs" else 0, prefix=rng.randint(1, max(2, N // 2)) if mask == "prefix" else 0,
              window=rng.randint(1, 1024) if mask == "window" else 0)
    if dtype == "fp32":  # an eighth of the bf16 rate or less
        c = dict(c, Nq=min(N, 3000), Nk=min(N, 3000))
    flops = work(c)["flops"]
    if flops > MOST_FLOPS:
        less = (MOST_FLOPS / flops) ** (0.5 if not c["window"] else 1.0)
        N = int(c["Nk"] * less)
        c = dict(c, Nq=N, Nk=N, prefix=int(c["prefix"] * less))
    return c


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _freqs(case):
    n = case["freqs"]
    return tuple(10000.0 ** (-i / n) for i in range(n))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def integers(lo, hi, shape, dtype=torch.int64):
        return torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=dtype)

    state = dict(case)
    if case["op"] == "rotate":
        B, N, D = case["B"], case["N"], case["D"]
        heads = [h for h in (case["H"], case["Hk"], case["Hp"]) if h]
        x = normal(B, N, sum(heads), D).mul_(3.0).to(dt)
        state["x"] = [t if case["fused"] else t.contiguous() for t in x.split(heads, dim=2)]
        state["w"] = [(1.0 + 0.2 * normal(D)).to(dt) for _ in heads] if case["weight"] else None
        state["g"] = [normal(B, N, h, D).to(dt) for h in heads]
        # Every sequence of a batch has its own first position.
        state["positions"] = integers(0, case["far"] + 1, (B, 1)) + torch.arange(N, device="cuda")
        state["angles"] = _freqs(case)
        state["eps"] = 1e-6 if case["norm"] else None
        if case["train"]:
            state["leaves"] = [t.detach().requires_grad_(True) for t in state["x"] + (state["w"] or [])]
        return state
    if case["op"] == "logprobs":
        R, V = case["R"], case["V"]
        state["targets"] = integers(0, V, (R,))
        x = normal(R, V).mul_(2.0)
        x[torch.arange(R, device="cuda"), state["targets"]] += 4.0  # the model knows something
        state["logits"] = x.to(dt)
        del x
        if case["train"]:
            state["logits"].requires_grad_(True)
            state["g"] = [normal(R) / R, normal(R) * (0.01 / R)]
        return state
    B, Nq, Nk, H, Hk, D = (case[n] for n in ("B", "Nq", "Nk", "H", "Hk", "D"))
    state["q"], state["k"], state["v"] = normal(B, Nq, H, D).to(dt), normal(B, Nk, Hk, D).to(dt), normal(B, Nk, Hk, D).to(dt)
    state["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H) if case["alibi"] else None
    state["documents"] = state["prefix"] = state["k_lens"] = None
    if case["docs"]:
        # `docs` documents cut at random places, padding (-1) behind the last.
        cuts = integers(0, Nk, (B, case["docs"] - 1)).sort(1).values if case["docs"] > 1 else integers(0, 1, (B, 0))
        at = torch.arange(Nk, device="cuda")
        ids = (at[None, :, None] >= cuts[:, None, :]).sum(2)
        end = integers(Nk - Nk // 16, Nk + 1, (B, 1))
        state["documents"] = torch.where(at < end, ids, -1).to(torch.int32)
    if case["prefix"]:
        state["prefix"] = integers(0, case["prefix"] + 1, (B,), torch.int32)
    if case["lens"]:
        state["k_lens"] = integers(Nk // 4, Nk + 1, (B,), torch.int32)
    if case["train"]:
        state["leaves"] = [state[n].requires_grad_(True) for n in ("q", "k", "v")]
        state["g"] = normal(B, Nq, H, D).to(dt)
    return state


def run(state):
    return _OWN[state["op"]](state) if own else _PLAIN[state["op"]](state)


# ---- the package's operators ----


def _own_rotate(s):
    from paper_2507_02754_amd import norm_rotate

    n = len(s["x"])
    x, w = (s["leaves"][:n], s["leaves"][n:] or None) if s["train"] else (s["x"], s["w"])
    y = norm_rotate(x, weights=w, eps=s["eps"], freqs=s["angles"], layout=s["layout"], positions=s["positions"])
    return [*y, *torch.autograd.grad(y, s["leaves"], s["g"])] if s["train"] else list(y)


def _own_attn(s):
    from paper_2507_02754_amd import dot_attention, simplicial_dot_attn_fwd

    opts = dict(causal=s["causal"], window=s["window"], softcap=s["cap"], slopes=s["slopes"], documents=s["documents"],
                prefix=s["prefix"], k_lens=s["k_lens"])
    if not s["train"]:
        return list(simplicial_dot_attn_fwd(s["q"], s["k"], s["v"], **opts))
    out = dot_attention(*s["leaves"], **opts)
    return [out, *torch.autograd.grad(out, s["leaves"], s["g"])]


def _own_logprobs(s):
    from paper_2507_02754_amd import token_logprobs

    r = token_logprobs(s["logits"], s["targets"], top=s["top"])
    out = [r.logprob, r.entropy]
    if s["train"]:
        out += torch.autograd.grad(out, [s["logits"]], s["g"])
    return out + ([r.top_logprobs, r.top_tokens] if s["top"] else [])


_OWN = {"rotate": _own_rotate, "attn": _own_attn, "logprobs": _own_logprobs}


# ---- the plain forms: float32, rounded once at the end ----


def _plain_rotate(s):
    n, D, m = len(s["x"]), s["D"], s["freqs"]
    x, w = (s["leaves"][:n], s["leaves"][n:] or None) if s["train"] else (s["x"], s["w"])
    # Angles in 64 bits: a far position times a frequency loses the fraction of a turn in 32.
    angle = s["positions"].double()[..., None] * torch.tensor(s["angles"], dtype=torch.float64, device="cuda")
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]

    def turn(t):
        if s["layout"] == "half":
            a, b, rest = t[..., :m], t[..., m:2 * m], t[..., 2 * m:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
        step = 3 if s["layout"] == "axis" else 2
        a, b, rest = t[..., 0:step * m:step], t[..., 1:step * m:step], t[..., step * m:]
        other = [t[..., 2:step * m:step]] if step == 3 else []
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin, *other], -1).flatten(-2), rest], -1)

    def one(t, weight):
        f = t.float()
        if s["norm"]:
            f = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + s["eps"])
        if weight is not None:
            f = f * weight.float()
        return turn(f).to(t.dtype)

    y = list(map(one, x, w or [None] * n))
    return [*y, *torch.autograd.grad(y, s["leaves"], s["g"])] if s["train"] else y


def _visible(s):
    """Which keys each query sees, [B, Nq, Nk], and their distance |p - j|, [B, Nq, Nk] or [1, Nq, Nk]."""
    Nq, Nk = s["Nq"], s["Nk"]
    j = torch.arange(Nk, device="cuda")
    lens = s["k_lens"].long()[:, None, None] if s["k_lens"] is not None else torch.full((1, 1, 1), Nk, device="cuda")
    p = lens - Nq + torch.arange(Nq, device="cuda")[None, :, None]  # the queries are the last Nq positions
    see = torch.ones((1, Nq, Nk), dtype=torch.bool, device="cuda")
    if s["causal"]:
        see = j <= p
    if s["window"]:
        see = see & ((p - j).abs() < s["window"])
    if s["prefix"] is not None:
        see = see | (j < s["prefix"][:, None, None])
    see = see & (p >= 0) & (j < lens)
    if s["documents"] is not None:
        ids = s["documents"]
        mine = ids.gather(1, p[..., 0].clamp(min=0).expand(ids.shape[0], Nq))
        see = see & (mine[:, :, None] == ids[:, None]) & (ids >= 0)[:, None]
    return see, (p - j).abs()


def _plain_attn(s):
    B, Nq, Nk, H, Hk, D = (s[n] for n in ("B", "Nq", "Nk", "H", "Hk", "D"))
    q, k, v = s["leaves"] if s["train"] else (s["q"], s["k"], s["v"])
    see, distance = _visible(s)
    see = see[:, None, None]
    qf = q.float().view(B, Nq, Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    kf, vf = k.float().permute(0, 2, 3, 1).contiguous(), v.float().transpose(1, 2).contiguous()
    a = (torch.matmul(qf, kf) * D ** -0.5).view(B, Hk, H // Hk, Nq, Nk)
    if s["cap"]:
        a = s["cap"] * torch.tanh(a / s["cap"])
    if s["slopes"] is not None:
        a = a - s["slopes"].view(Hk, H // Hk, 1, 1) * distance[:, None, None]
    a = a.masked_fill(~see, -math.inf)
    top = a.detach().amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(a - top)
    total = e.sum(-1, keepdim=True)
    weights = (e / torch.where(total == 0, 1.0, total)).view(B, Hk, -1, Nk)
    out = torch.matmul(weights, vf).view(B, Hk, H // Hk, Nq, D).permute(0, 3, 1, 2, 4).reshape(B, Nq, H, D).to(q.dtype)
    if s["train"]:
        return [out, *torch.autograd.grad(out, s["leaves"], s["g"])]
    return [out, (top + total.log()).view(B, H, Nq)]


def _plain_logprobs(s):
    x = s["logits"].float()
    top = x.detach().amax(-1, keepdim=True)
    lse = top + torch.exp(x - top).sum(-1, keepdim=True).log()
    logp = x - lse
    lp = logp.gather(1, s["targets"][:, None])[:, 0]
    entropy = -(torch.exp(logp) * logp).sum(-1)
    if s["train"]:
        return [lp, entropy, *torch.autograd.grad([lp, entropy], [s["logits"]], s["g"])]
    if not s["top"]:
        return [lp, entropy]
    # Equal values go to the lowest token: the value in the upper bits of one
    # whole number, the token in the lower.
    bits = (x + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + ((1 << 32) - 1 - torch.arange(s["V"], device="cuda"))
    tokens = (1 << 32) - 1 - (key.topk(s["top"], -1).values & ((1 << 32) - 1))
    return [lp, entropy, logp.gather(1, tokens), tokens]


_PLAIN = {"rotate": _plain_rotate, "attn": _plain_attn, "logprobs": _plain_logprobs}


def _pairs(case):
    """(query, key) pairs one head sees over all sequences, expected where cuts and lengths are drawn."""
    Nq, Nk = case["Nq"], case["Nk"]
    if case["lens"]:
        Nk = 0.625 * Nk
    each = Nq * Nk - (Nq * (Nq - 1) / 2 if case["causal"] else 0)
    if case["window"]:
        w = min(case["window"], Nk)
        each = min(each, Nq * w - (w * (w - 1) / 2 if Nq == Nk else 0)) if case["causal"] else min(each, Nq * (2 * w - 1))
    if case["docs"]:
        each = each * 2 / (case["docs"] + 1) * (31 / 32) ** 2
    if case["prefix"]:
        each += (case["prefix"] / 2) ** 2 / 2
    return case["B"] * max(each, Nq)


def work(case):
    el = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "rotate":
        values = case["B"] * case["N"] * (case["H"] + case["Hk"] + case["Hp"]) * case["D"]
        # forward: x read, y written; training: x and dy read, y and dx written
        return {"bytes": values * el * (4 if case["train"] else 2) + 8 * case["B"] * case["N"],
                "flops": values * (22 if case["train"] else 8)}
    if case["op"] == "logprobs":
        values = case["R"] * case["V"]
        return {"bytes": values * el * (2 if case["train"] else 1) + case["R"] * (24 + 12 * case["top"]),
                "flops": values * (14 if case["train"] else 6)}
    B, Nq, Nk, H, Hk, D = (case[n] for n in ("B", "Nq", "Nk", "H", "Hk", "D"))
    keys = min(Nk, case["window"] + Nq) if case["window"] and not case["train"] else Nk * (0.625 if case["lens"] else 1)
    qs, ks = B * Nq * H * D * el, B * keys * Hk * D * el
    # forward: Q K^T and P V; backward: Q K^T again, dP, dV, dQ, dK
    if case["train"]:
        return {"bytes": 4 * qs + 4 * ks, "flops": 14 * H * D * _pairs(case)}
    return {"bytes": 2 * qs + 2 * ks + 4 * B * H * Nq, "flops": 4 * H * D * _pairs(case)}


# ---- float64 ----


def _exact_rotate(s):
    """The rotation as a product of complex numbers, its adjoint for the gradients."""
    n = s["freqs"]
    angle = s["positions"].double()[..., None] * torch.tensor(s["angles"], dtype=torch.float64, device="cuda")
    z = torch.complex(angle.cos(), angle.sin())[:, :, None]
    at = torch.arange(n, device="cuda")
    first = {"half": at, "pairs": 2 * at, "axis": 3 * at}[s["layout"]]
    second = first + (n if s["layout"] == "half" else 1)

    def turn(t, z):
        r = torch.complex(t[..., first], t[..., second]) * z
        t = t.clone()
        t[..., first], t[..., second] = r.real, r.imag
        return t

    ys, dxs, dws = [], [], []
    for i, x in enumerate(s["x"]):
        x = x.detach().double()
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"]) if s["norm"] else torch.ones_like(x[..., :1])
        w = s["w"][i].detach().double() if s["w"] else torch.ones(s["D"], dtype=torch.float64, device="cuda")
        ys.append(turn(x * r * w, z))
        if s["train"]:
            d = turn(s["g"][i].double(), z.conj())
            dws.append((d * x * r).sum((0, 1, 2)))
            d = d * w
            dxs.append(r * d - (x * r ** 3 * (d * x).mean(-1, keepdim=True) if s["norm"] else 0))
    return [*ys, *dxs, *(dws if s["w"] else [])]


def _exact_attn(s):
    """Head by head over blocks of queries, the gradients from their formulas."""
    B, Nq, Nk, H, Hk, D = (s[n] for n in ("B", "Nq", "Nk", "H", "Hk", "D"))
    see, distance = _visible(s)
    see, distance = see.expand(B, Nq, Nk), distance.expand(B, Nq, Nk)
    q, k, v = (s[n].detach().double() for n in ("q", "k", "v"))
    out, lse = torch.zeros_like(q), torch.zeros((B, H, Nq), dtype=q.dtype, device="cuda")
    dq, dk, dv = (torch.zeros_like(t) for t in (q, k, v))
    block = max(1, (1 << 25) // Nk)
    for b in range(B):
        for h in range(H):
            kh, vh = k[b, :, h * Hk // H].contiguous(), v[b, :, h * Hk // H].contiguous()
            for i in range(0, Nq, block):
                rows = slice(i, min(i + block, Nq))
                qh = q[b, rows, h].contiguous()
                a = qh @ kh.t() * D ** -0.5
                slope = 1.0
                if s["cap"]:
                    a = s["cap"] * torch.tanh(a / s["cap"])
                    slope = 1 - (a / s["cap"]) ** 2
                if s["slopes"] is not None:
                    a = a - s["slopes"][h].double() * distance[b, rows]
                a = torch.where(see[b, rows], a, -math.inf)
                z = torch.logsumexp(a, -1)
                p = torch.where(see[b, rows], torch.exp(a - z[:, None]), 0.0)
                o = p @ vh
                out[b, rows, h], lse[b, h, rows] = o, z
                if s["train"]:
                    do = s["g"][b, rows, h].double()
                    da = p * (do @ vh.t() - (do * o).sum(-1, keepdim=True)) * slope * D ** -0.5
                    dq[b, rows, h] = da @ kh
                    dk[b, :, h * Hk // H] += da.t() @ qh
                    dv[b, :, h * Hk // H] += p.t() @ do
    return [out, dq, dk, dv] if s["train"] else [out, lse]


def _exact_logprobs(s):
    x = s["logits"].detach().double()
    logp = torch.log_softmax(x, -1)
    del x
    lp = logp.gather(1, s["targets"][:, None])
    p = torch.exp(logp)
    entropy = -(p * logp).sum(-1, keepdim=True)
    if s["train"]:
        g, h = (t.double()[:, None] for t in s["g"])
        dx = -p * (g + h * (logp + entropy))
        dx.scatter_add_(1, s["targets"][:, None], g)
        return [lp[:, 0], entropy[:, 0], dx]
    if not s["top"]:
        return [lp[:, 0], entropy[:, 0]]
    return [lp[:, 0], entropy[:, 0], logp.topk(s["top"], -1).values, None]


def exact(case, seed):
    with torch.no_grad():
        return {"rotate": _exact_rotate, "attn": _exact_attn, "logprobs": _exact_logprobs}[case["op"]](prepare(case, seed))

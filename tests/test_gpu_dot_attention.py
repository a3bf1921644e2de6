"""Dot-product attention with capped scores, distance bias and masks on the GPU against
float64."""

import math

import pytest
import torch

import layers_reference as ref
from paper_2507_02754_amd import (dot_attention, load_library, simplicial_dot_attn_bwd, simplicial_dot_attn_fwd)

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    load_library()


def _normal(*shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def _ints(lo, hi, shape, seed):
    return torch.randint(lo, hi, shape, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()


def _slopes(H):
    return (2.0 ** (-8.0 * torch.arange(1, H + 1) / H)).cuda()


def _check(q, k, v, dout, label, **opts):
    lo = torch.empty_like(q, memory_format=torch.contiguous_format) if q.dtype == BF and dout is not None else None
    out, lse = simplicial_dot_attn_fwd(q, k, v, out_lo=lo, **opts)
    got = {"out": out, "lse": lse}
    if dout is not None:
        got.update(zip(("dq", "dk", "dv"), simplicial_dot_attn_bwd(q, k, v, out, dout, lse, out_lo=lo, **opts)))
    torch.cuda.synchronize()
    want = ref.dot_attention(q, k, v, dout=dout, **opts)
    for name, w in want.items():
        ref.close(got[name], *w, f"{label}: {name}")
    return got


def _inputs(B, Nq, Nk, H, Hkv, D, dt, seed=0, scale=1.0):
    return (_normal(B, Nq, H, D, seed=seed, dtype=dt, scale=scale), _normal(B, Nk, Hkv, D, seed=seed + 1, dtype=dt, scale=scale),
            _normal(B, Nk, Hkv, D, seed=seed + 2, dtype=dt), _normal(B, Nq, H, D, seed=seed + 3, dtype=dt))


# B, N, H, Hkv, D, causal, window, cap, alibi
SIZES = [
    (1, 1, 1, 1, 16, True, 0, 0.0, False),
    (2, 2, 2, 1, 128, True, 0, 0.0, False),
    (1, 31, 3, 1, 32, True, 0, 5.0, True),
    (1, 33, 4, 4, 64, False, 0, 0.0, False),
    (2, 64, 6, 2, 128, True, 0, 0.0, True),
    (1, 97, 5, 5, 64, False, 10, 0.0, False),
    (1, 130, 8, 2, 128, True, 1, 0.0, False),
    (2, 127, 4, 1, 16, True, 50, 2.0, False),
    (1, 257, 7, 1, 32, True, 0, 0.0, False),
    (1, 260, 2, 2, 128, False, 33, 3.0, True),
    (1, 515, 4, 2, 64, True, 64, 0.0, True),
    (1, 600, 4, 4, 128, True, 0, 20.0, False),
    (1, 1021, 4, 1, 128, True, 0, 0.0, False),
    (1, 700, 2, 2, 16, False, 0, 0.0, False),
    (1, 900, 16, 4, 64, True, 300, 30.0, False),
    (2, 1500, 2, 1, 128, True, 0, 0.0, True),
    (1, 1100, 3, 3, 64, False, 0, 0.0, False),
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_float64(size, dt):
    B, N, H, Hkv, D, causal, window, cap, alibi = size
    print(f"\n[dot] {size} {dt}", flush=True)
    q, k, v, dout = _inputs(B, N, N, H, Hkv, D, dt, seed=N)
    _check(q, k, v, dout, str(size), causal=causal, window=window, softcap=cap, slopes=_slopes(H) if alibi else None)


# Sizes that take every form of the bf16 kernels: workgroups of 128 rows and keys, with one
# group of wavefronts and two, and several workgroups a block of keys (float32 the same).
FORMS = [
    (4, 390, 64, 64, 128),   # 1024 blocks of 128 rows and of keys
    (2, 450, 40, 20, 128),   # two groups of wavefronts on both sides
    (1, 700, 16, 4, 128),    # grouped heads: several workgroups a block of keys
    (1, 2100, 3, 1, 64),     # head_dim 64, likewise
    (5, 300, 48, 48, 64),    # 128 rows at head_dim 64
    (3, 520, 48, 16, 32),
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", FORMS, ids=str)
def test_every_form(size, dt):
    """Each with a causal mask alone, documents with padding, a window with cap and bias, and
    a prefix over caches filled to different lengths (one empty, one shorter than its queries)."""
    B, N, H, Hkv, D = size
    print(f"\n[dot] form {size} {dt}", flush=True)
    q, k, v, dout = _inputs(B, N, N, H, Hkv, D, dt, seed=N)
    _check(q, k, v, dout, f"{size} causal")
    at = torch.arange(N)
    ids = torch.stack([(at >= 37 + 11 * b).int() + (at >= N // 2).int() + (at >= N - 60).int() * 5 for b in range(B)]).to(torch.int32)
    ids[0, N - 30:] = -1
    _check(q, k, v, dout, f"{size} documents", documents=ids.cuda())
    _check(q, k, v, dout, f"{size} window", window=131, softcap=3.0, slopes=_slopes(H))
    lens = torch.tensor([N, N // 2, 0, 40, N - 1][:B], dtype=torch.int32).cuda()
    prefix = torch.tensor([77, 33, 5, N, 0][:B], dtype=torch.int32).cuda()
    for b in range(B):
        k[b, int(lens[b]):] = float("nan")
        v[b, int(lens[b]):] = float("inf")
    _check(q, k, v, dout, f"{size} prefix", prefix=prefix, k_lens=lens, softcap=20.0)


@pytest.mark.parametrize("size", [s for s in FORMS if s[4] >= 64], ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("-inf")])
def test_masked_values_in_every_form(size, bad):
    """One later document of nothing but NaN or infinities: the others do not see it."""
    B, N, H, Hkv, D = size
    q, k, v, dout = _inputs(B, N, N, H, Hkv, D, BF, seed=N + 1)
    n = N // 2 + 13
    ids = (torch.arange(N) >= n).to(torch.int32).expand(B, N).contiguous().cuda()
    want = ref.dot_attention(q, k, v, documents=ids, dout=dout)
    for x in (q, k, v, dout):
        x[:, n:] = bad
    out, lse = simplicial_dot_attn_fwd(q, k, v, documents=ids)
    grads = simplicial_dot_attn_bwd(q, k, v, out, dout, lse, documents=ids)
    torch.cuda.synchronize()
    ref.close(lse[:, :, :n], *(x[:, :, :n] for x in want["lse"]), "lse")
    for name, x in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        ref.close(x[:, :n], *(y[:, :n] for y in want[name]), name)


# B, Nq, Nk, H, Hkv, D, window, cap, lens
NEW = [
    (1, 1, 1, 4, 4, 64, 0, 0.0, None),
    (3, 1, 50, 8, 2, 128, 0, 0.0, [0, 1, 50]),
    (4, 1, 3000, 16, 4, 128, 0, 30.0, [3000, 2999, 17, 64]),
    (2, 1, 5001, 8, 8, 64, 700, 0.0, [5001, 650]),
    (2, 1, 1000, 4, 1, 32, 0, 0.0, [999, 32]),
    (2, 3, 777, 6, 2, 128, 0, 0.0, [777, 2]),      # fewer keys than queries
    (2, 9, 2050, 16, 2, 64, 100, 0.0, [2050, 1025]),
    (1, 33, 1025, 4, 2, 16, 0, 0.0, None),
    (1, 200, 4000, 8, 2, 128, 0, 0.0, [3500]),
    (2, 1, 4100, 4, 4, 16, 0, 0.0, [-5, 9000]),    # clamped to [0, Nk]
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("case", NEW, ids=str)
def test_new_tokens_over_a_cache(case, dt):
    """The queries are the last positions of every sequence's filled part; what lies behind
    it (here NaN) is not looked at. Backward too: keys behind the filled part get zeros."""
    B, Nq, Nk, H, Hkv, D, window, cap, lens = case
    print(f"\n[dot] cache {case} {dt}", flush=True)
    q, k, v, dout = _inputs(B, Nq, Nk, H, Hkv, D, dt, seed=Nk)
    k_lens = None
    if lens is not None:
        k_lens = torch.tensor(lens, dtype=torch.int32).cuda()
        for b, n in enumerate(lens):
            k[b, min(max(n, 0), Nk):] = float("nan")
            v[b, min(max(n, 0), Nk):] = float("nan")
    got = _check(q, k, v, dout, str(case), window=window, softcap=cap, k_lens=k_lens)
    if lens is not None:
        for b, n in enumerate(lens):
            n = min(max(n, 0), Nk)
            assert (got["dk"][b, n:] == 0).all() and (got["dv"][b, n:] == 0).all()
            empty = max(Nq - n, 0)
            assert (got["out"][b, :empty] == 0).all() and (got["lse"][b, :, :empty] == -math.inf).all()
            assert (got["dq"][b, :empty] == 0).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("D", [32, 128])
def test_documents_and_prefix(D, dt):
    """Packed documents with padding behind them, document numbers in any order and
    interleaved, prefixes from none to all, and both with a window."""
    B, N, H, Hkv = 3, 421, 4, 2
    print(f"\n[dot] documents D={D} {dt}", flush=True)
    q, k, v, dout = _inputs(B, N, N, H, Hkv, D, dt, seed=D)
    at = torch.arange(N)
    ids = torch.stack([(at >= 100).int() + (at >= 101).int() + (at >= 300).int(), 7 - at // 64, _ints(0, 4, (N,), 5).cpu()]).to(torch.int32)
    ids[0, 400:] = -1
    ids[1, :5] = -7
    ids = ids.cuda()
    prefix = torch.tensor([0, 150, N], dtype=torch.int32).cuda()
    got = _check(q, k, v, dout, "documents", documents=ids)
    assert (got["out"][0, 400:] == 0).all() and (got["lse"][0, :, 400:] == -math.inf).all()
    assert (got["dk"][0, 400:] == 0).all() and (got["dq"][0, 400:] == 0).all()
    _check(q, k, v, dout, "documents, all keys", documents=ids, causal=False)
    _check(q, k, v, dout, "prefix", prefix=prefix)
    _check(q, k, v, dout, "prefix and window", prefix=prefix, window=40, slopes=_slopes(H))
    _check(q, k, v, dout, "documents, prefix and window", documents=ids, prefix=prefix, window=90, softcap=4.0)
    lens = torch.tensor([N, 200, 77], dtype=torch.int32).cuda()
    _check(q[:, :60].contiguous(), k, v, dout[:, :60].contiguous(), "documents of a cache", documents=ids, prefix=prefix, k_lens=lens)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_masked_values_do_not_reach_what_does_not_see_them(dt, bad):
    """NaN and infinities in a later document, in padding, in later positions and in
    empty rows leave every query and key that does not see them as they are."""
    B, N, H, Hkv, D = 1, 300, 4, 2, 64
    print(f"\n[dot] masked {bad} {dt}", flush=True)
    q, k, v, dout = _inputs(B, N, N, H, Hkv, D, dt, seed=3)
    at = torch.arange(N)
    ids = torch.where(at < 290, (at >= 141).int(), -1).to(torch.int32)[None].cuda()
    # (the value of no masked pair enters the reference: it serves the clean inputs and the others)
    want = ref.dot_attention(q, k, v, documents=ids, dout=dout)
    for where in (slice(141, 290), slice(290, N)):
        t = [x.clone() for x in (q, k, v, dout)]
        for x in t:
            x[:, where] = bad
        out, lse = simplicial_dot_attn_fwd(*t[:3], documents=ids)
        grads = simplicial_dot_attn_bwd(*t[:3], out, t[3], lse, documents=ids)
        torch.cuda.synchronize()
        n = where.start
        ref.close(lse[:, :, :n], *(x[:, :, :n] for x in want["lse"]), "lse")
        for name, x in zip(("out", "dq", "dk", "dv"), (out, *grads)):
            ref.close(x[:, :n], *(y[:, :n] for y in want[name]), name)
            assert n < 290 or bool((x[:, where] == 0).all()), name
    # causal: a later position's values do not reach earlier ones within a block either
    v2 = v.clone()
    v2[:, 45] = bad
    out, _ = simplicial_dot_attn_fwd(q, k, v2)
    want = ref.dot_attention(q, k, v)
    torch.cuda.synchronize()
    ref.close(out[:, :45], *(x[:, :45] for x in want["out"]), "before a bad value")
    assert not bool(torch.isfinite(out[:, 45:]).any())


def test_views():
    """q, k and v as slices of one projection's output, a cache longer than what is
    passed, and heads moved behind positions."""
    B, N, H, D = 2, 150, 4, 64
    qkv = _normal(B, N, 3, H, D, seed=8, dtype=BF)
    q, k, v = qkv.unbind(2)
    _check(q, k, v, _normal(B, N, H, D, seed=9, dtype=BF), "slices")
    cache = _normal(2, B, 512, H, D, seed=10, dtype=BF)
    k, v = cache[0][:, :N], cache[1][:, :N]
    _check(q[:, -1:], k, v, None, "cache")
    byhead = _normal(B, H, N, D, seed=11, dtype=F32).transpose(1, 2)
    _check(byhead, byhead, byhead, None, "heads first")
    odd = _normal(B, N, H, D + 4, seed=12, dtype=BF)[..., 4:]
    a = dot_attention(odd, odd, odd)
    b = dot_attention(*[odd.contiguous()] * 3)
    assert torch.equal(a, b)


def test_one_head_for_all_by_stride():
    """k and v expanded over the batch (stride 0): read once, same results."""
    q, k, v, _ = _inputs(3, 70, 70, 4, 2, 64, BF, seed=5)
    k1, v1 = k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)
    a = simplicial_dot_attn_fwd(q, k1, v1)
    b = simplicial_dot_attn_fwd(q, k1.contiguous(), v1.contiguous())
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("D", [16, 64, 128])
def test_one_key_alone_has_no_gradient_of_scores(dt, D):
    """Rows that see one key (a first token, a window of one): O is its value, dq and dk are 0."""
    for N, H, Hkv, B in ((1, 4, 2, 3), (70, 4, 4, 1), (390, 64, 64, 4)):
        q, k, v, dout = _inputs(B, N, N, H, Hkv, D, dt, seed=N)
        leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
        out = dot_attention(*leaves, window=1)
        dq, dk, dv = torch.autograd.grad(out, leaves, dout)
        assert torch.equal(out, v.repeat_interleave(H // Hkv, 2))
        assert (dq == 0).all() and (dk == 0).all()
        want = dout.double().view(B, N, Hkv, H // Hkv, D).sum(3)
        ref.close(dv, want, 2 * ref.HALF[dt] * dout.double().abs().view(B, N, Hkv, H // Hkv, D).sum(3) + 1e-30, "dv")


@pytest.mark.parametrize("dt", [BF, F32])
def test_large_scores(dt):
    """Scores of hundreds (one key takes all weight), a zero scale and a negative one."""
    q, k, v, dout = _inputs(1, 140, 140, 2, 2, 64, dt, seed=6, scale=8.0)
    _check(q, k, v, dout, "large")
    _check(q, k, v, dout, "zero scale", scale=0.0)
    _check(q, k, v, dout, "negative scale", scale=-0.01, softcap=1.0)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", [(1, 70, 70, 48, 1, 64), (2, 1, 500, 40, 1, 128), (1, 333, 333, 66, 2, 128), (2, 5, 161, 33, 1, 16)], ids=str)
def test_more_heads_on_one_than_a_block_has_rows(size, dt):
    B, Nq, Nk, H, Hkv, D = size
    q, k, v, dout = _inputs(*size, dt, seed=H)
    ids = (torch.arange(Nk) >= Nk - 30).to(torch.int32).expand(B, Nk).contiguous().cuda()
    lens = torch.tensor([Nk - 7, Nk][:B], dtype=torch.int32).cuda()
    _check(q, k, v, dout, f"{size} documents", documents=ids, k_lens=lens)
    _check(q, k, v, dout, f"{size} window", window=40, slopes=_slopes(H), softcap=8.0)


@pytest.mark.parametrize("dt", [BF, F32])
def test_shared_and_expanded_inputs(dt):
    """Keys and values that every head or every sequence shares by a stride of 0, and an
    upstream gradient of one number."""
    B, N, H, D = 2, 90, 4, 64
    q, k, v, _ = _inputs(B, N, N, H, 1, D, dt, seed=9)
    kb, vh = k[:1].expand(B, N, 1, D).expand(B, N, H, D), v.expand(B, N, H, D)
    dout = torch.ones_like(q)
    _check(q, kb, vh, dout, "expanded")
    leaves = [x.detach().clone().requires_grad_(True) for x in (q, k, v)]
    out = dot_attention(leaves[0], leaves[1][:1].expand(B, N, H, D), leaves[2].expand(B, N, H, D))
    grads = torch.autograd.grad(out.sum(), leaves)
    whole = simplicial_dot_attn_fwd(q, kb.contiguous(), vh.contiguous(), out_lo=(lo := torch.empty_like(q) if dt == BF else None))
    want = simplicial_dot_attn_bwd(q, kb.contiguous(), vh.contiguous(), whole[0], dout, whole[1], out_lo=lo)
    assert torch.equal(out, whole[0]) and torch.equal(grads[0], want[0])
    total = want[2].double().sum(2, keepdim=True)
    assert ((grads[2].double() - total).abs() <= 4 * ref.HALF[dt] * want[2].double().abs().sum(2, keepdim=True)).all()


def test_windows_of_any_number():
    """Windows past the keys (and past 32 bits) hide nothing; negative ones are refused."""
    q, k, v, _ = _inputs(1, 70, 70, 2, 1, 64, BF)
    want = simplicial_dot_attn_fwd(q, k, v)
    for window in (70, 1 << 31, (1 << 32) + 5):
        got = simplicial_dot_attn_fwd(q, k, v, window=window)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
    for window in (-1, -(1 << 32)):
        with pytest.raises(ValueError, match="negative"):
            simplicial_dot_attn_fwd(q, k, v, window=window)


# B, Nq, Nk, H, Hkv, D: the forms of the forward
FORWARDS = [(1, 140, 140, 2, 2, 64), (4, 390, 390, 64, 64, 128), (2, 450, 450, 40, 20, 128), (1, 700, 700, 16, 4, 128),
            (2, 1, 2900, 8, 2, 128), (5, 300, 300, 48, 48, 64)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", FORWARDS, ids=str)
def test_caps_far_above_the_scores(size, dt):
    """A cap of 10^6 takes less than 10^-9 off scores of this size: as without one, to the
    bounds of that; and one of 2000 to its own."""
    B, Nq, Nk, H, Hkv, D = size
    q, k, v, dout = _inputs(*size, dt, seed=Nk, scale=2.0)
    want = ref.dot_attention(q, k, v, dout=dout)
    lo = torch.empty_like(q) if dt == BF else None
    out, lse = simplicial_dot_attn_fwd(q, k, v, softcap=1e6, out_lo=lo)
    grads = simplicial_dot_attn_bwd(q, k, v, out, dout, lse, softcap=1e6, out_lo=lo)
    for name, x in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *grads)):
        ref.close(x, *want[name], f"{size} cap 1e6: {name}")
    _check(q, k, v, dout, f"{size} cap 2000", softcap=2000.0, slopes=_slopes(H))


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", FORWARDS, ids=str)
def test_enormous_scores(size, dt, sign):
    """Scores of 2^41 and 2^113, three values of them: a mean, with some weights, of the values
    whose keys have the largest. float32 rounds a score by up to 2^-24 of it, 2^17 and more
    here, so that the weights among equal scores are open; but keys of another score, 2^41 and
    more below, have none, and nothing overflows on the way."""
    B, Nq, Nk, H, Hkv, D = size
    see = ref.visible(B, Nq, Nk, True, 0, None, None, None, "cuda")[0][0]  # [Nq, Nk]
    kind = (1 + torch.arange(Nk) * 7 % 3).cuda()
    v = _normal(B, Nk, Hkv, D, seed=Nk, dtype=dt)
    vd = v.double().view(B, Nk, Hkv * D)
    for e in (19, 55):
        q = torch.full((B, Nq, H, D), 2.0 ** e, dtype=dt, device="cuda")
        k = (kind.view(1, Nk, 1, 1) * (sign * 2.0 ** e)).to(dt).expand(B, Nk, Hkv, D).contiguous()
        out, lse = simplicial_dot_attn_fwd(q, k, v, scale=8.0 / D)
        a = torch.where(see, sign * kind.double() * 2.0 ** (2 * e + 3), -math.inf)
        top = a.amax(1)
        for i in {0, 1, 2, 31, 32, 95, Nq // 2, Nq - 1} & set(range(Nq)):
            values = vd[:, (a[i] == top[i]).nonzero()[:, 0]]
            o = out[:, i].double().view(B, Hkv, H // Hkv, D).transpose(1, 2).reshape(B, H // Hkv, Hkv * D)
            slack = (ref.HALF[dt] + (Nk / 32 + 64) * ref.U) * values.abs().amax(1, keepdim=True)
            low, high = values.amin(1, keepdim=True) - slack, values.amax(1, keepdim=True) + slack
            assert ((o >= low) & (o <= high)).all(), f"{size} 2^{2 * e + 3} row {i}"
        top = top.view(1, 1, Nq).expand(B, H, Nq)
        ref.close(lse, top, (D / 2 + 16) * ref.U * top.abs(), "lse")


def test_far_cache_passes_32_bits():
    """One new token over a cache of more than 2^32 bytes a tensor, two of its heads."""
    Nk, Hkv, D = 1 << 21, 8, 128  # 2^31 elements
    k = torch.empty((1, Nk, Hkv, D), dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for part in k.split(1 << 18, 1):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda", dtype=torch.float32))
    v = k.flip(3)
    q = _normal(1, 1, Hkv, D, seed=2, dtype=BF)
    out, lse = simplicial_dot_attn_fwd(q, k, v)
    torch.cuda.synchronize()
    for h in (0, 7):
        want = ref.dot_attention(q[:, :, h:h + 1], k[:, :, h:h + 1], v[:, :, h:h + 1])
        ref.close(out[:, :, h:h + 1], *want["out"], "out")
        ref.close(lse[:, h:h + 1], *want["lse"], "lse")


def test_autograd_equals_the_direct_calls():
    q, k, v, dout = _inputs(2, 90, 90, 4, 2, 64, BF, seed=12)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    out = dot_attention(*leaves, softcap=9.0, window=30)
    grads = torch.autograd.grad(out, leaves, dout.float().to(BF).transpose(1, 2).contiguous().transpose(1, 2))
    lo = torch.empty_like(q)
    o, lse = simplicial_dot_attn_fwd(q, k, v, softcap=9.0, window=30, out_lo=lo)
    want = simplicial_dot_attn_bwd(q, k, v, o, dout, lse, softcap=9.0, window=30, out_lo=lo)
    assert torch.equal(out, o) and all(torch.equal(a, b) for a, b in zip(grads, want))


@pytest.mark.parametrize("size", [(1, 50, 4, 2, 128), (1, 300, 8, 8, 64), (2, 450, 40, 20, 128), (4, 390, 64, 64, 128)], ids=str)
def test_what_rounding_took(size):
    """O + out_lo is O to twice the digits, in every form of the forward and over a split key
    axis, and the gradients without it are within the rounding of O."""
    B, N, H, Hkv, D = size
    q, k, v, dout = _inputs(B, N, N, H, Hkv, D, BF, seed=13)
    lo = torch.empty_like(q)
    out, lse = simplicial_dot_attn_fwd(q, k, v, out_lo=lo)
    exact, bound = ref.dot_attention(q, k, v)["out"]
    both = out.double() + lo.double()
    assert ((both - exact).abs() <= bound - 2.0 ** -8 * exact.abs() + 2.0 ** -15 * exact.abs()).all()
    assert (lo.double().abs() <= 2.0 ** -8 * both.abs() * 1.01 + 1e-30).all()
    grads = simplicial_dot_attn_bwd(q, k, v, out, dout, lse)
    for name, x in zip(("dq", "dk", "dv"), grads):
        ref.close(x, *ref.dot_attention(q, k, v, dout=dout)[name], name)
    one = q[:, -1:].contiguous()
    lo1 = torch.empty_like(one)
    out1, _ = simplicial_dot_attn_fwd(one, k, v, out_lo=lo1)
    both1 = out1.double() + lo1.double()
    assert ((both1 - exact[:, -1:]).abs() <= bound[:, -1:] - 2.0 ** -8 * exact[:, -1:].abs() + 2.0 ** -15 * exact[:, -1:].abs()).all()


def test_gradients_against_differences():
    """float32 directional differences with a cap, a bias and a prefix."""
    q, k, v, dout = _inputs(1, 40, 40, 4, 2, 32, F32, seed=20)
    opts = dict(softcap=2.0, slopes=_slopes(4), prefix=torch.tensor([9], dtype=torch.int32).cuda(), window=17)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    grads = torch.autograd.grad(dot_attention(*leaves, **opts), leaves, dout)
    step = 2.0 ** -7
    for i in range(3):
        d = _normal(*leaves[i].shape, seed=30 + i)
        ends = []
        for sign in (1, -1):
            t = [q, k, v]
            t[i] = t[i] + sign * step * d
            ends.append((dot_attention(*t, **opts).double() * dout.double()).sum())
        slope, want = (ends[0] - ends[1]) / (2 * step), (grads[i].double() * d.double()).sum()
        assert abs(slope - want) <= 1e-3 * (grads[i].double() * d.double()).abs().sum(), i


def test_results_repeat_and_captured_graphs():
    q, k, v, dout = _inputs(2, 300, 300, 8, 2, 128, BF, seed=40)
    ids = (torch.arange(300) // 77).to(torch.int32).expand(2, 300).contiguous().cuda()
    lens = torch.tensor([300, 123], dtype=torch.int32).cuda()
    one = q[:, :1].contiguous()

    def calls():
        out, lse = simplicial_dot_attn_fwd(q, k, v, documents=ids)
        return (out, lse, *simplicial_dot_attn_bwd(q, k, v, out, dout, lse, documents=ids),
                *simplicial_dot_attn_fwd(one, k, v, k_lens=lens))

    eager, again = calls(), calls()
    assert all(torch.equal(a, b) for a, b in zip(eager, again))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for i in range(3):
        q.copy_(_normal(*q.shape, seed=50 + i, dtype=BF))
        one.copy_(q[:, :1])
        lens -= 9
        ids += 1
        eager = calls()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), i

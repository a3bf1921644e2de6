"""Infinities and NaN in dot-product attention: where they belong they come out, in every
form of the kernels, and nowhere else."""

import pytest
import torch

import layers_reference as ref
from paper_2507_02754_amd import load_library, simplicial_dot_attn_bwd, simplicial_dot_attn_fwd

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAMES = ("out", "lse", "dq", "dk", "dv")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    load_library()


def _normal(*shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _inputs(B, Nq, Nk, H, Hkv, D, dt, seed):
    """q, k, v and the upstream gradient."""
    return [_normal(B, Nq, H, D, seed=seed, dtype=dt), _normal(B, Nk, Hkv, D, seed=seed + 1, dtype=dt),
            _normal(B, Nk, Hkv, D, seed=seed + 2, dtype=dt), _normal(B, Nq, H, D, seed=seed + 3, dtype=dt)]


def _call(q, k, v, dout, **opts):
    """All results by name, the buffers filled with a finite number before."""
    B, Nq, H, D = q.shape
    lo = torch.full_like(q, 7.0) if q.dtype == BF else None
    out, lse = simplicial_dot_attn_fwd(q, k, v, out=torch.full_like(q, 7.0), lse=torch.full((B, H, Nq), 7.0, device="cuda"), out_lo=lo, **opts)
    grads = simplicial_dot_attn_bwd(q, k, v, out, dout, lse, out_lo=lo, grads=[torch.full_like(t, 7.0) for t in (q, k, v)], **opts)
    torch.cuda.synchronize()
    return dict(zip(NAMES, (out, lse, *grads)))


def _plain(q, k, v, dout):
    """The formulas in float64, every key visible, whatever the values."""
    B, Nq, H, D = q.shape
    Nk, Hkv = k.shape[1:3]
    q, do = (t.double().transpose(1, 2) for t in (q, dout))
    k, v = (t.double().transpose(1, 2).repeat_interleave(H // Hkv, 1) for t in (k, v))
    s = q @ k.transpose(2, 3) * D ** -0.5
    p = torch.softmax(s, 3)
    out = p @ v
    ds = p * (do @ v.transpose(2, 3) - (do * out).sum(3, keepdim=True)) * D ** -0.5
    dk, dv = (t.view(B, Hkv, H // Hkv, Nk, D).sum(2) for t in (ds.transpose(2, 3) @ q, p.transpose(2, 3) @ do))
    return dict(zip(NAMES, (out.transpose(1, 2), torch.logsumexp(s, 3), (ds @ k).transpose(1, 2), dk.transpose(1, 2), dv.transpose(1, 2))))


# B, N, H, Hkv, D: the forms of the backward's two sides (float32 has one)
FORMS = [
    (1, 70, 2, 2, 64),       # 32 rows and 32 keys a workgroup
    (4, 390, 64, 64, 128),   # 128 rows and 128 keys
    (2, 450, 40, 20, 128),   # two groups of wavefronts on both sides
    (1, 700, 16, 4, 128),    # several workgroups a block of keys
    (1, 2100, 3, 1, 64),
    (5, 300, 48, 48, 64),
    (3, 520, 48, 16, 32),
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", FORMS, ids=str)
def test_without_a_mask(size, dt):
    """Every query sees every key: against float64, and with one NaN or infinity in each of q, k, v
    and the upstream gradient, whose results are finite where the formula's are, and only there."""
    B, N, H, Hkv, D = size
    print(f"\n[dot] no mask {size} {dt}", flush=True)
    clean = _inputs(B, N, N, H, Hkv, D, dt, seed=N)
    q, k, v, dout = clean
    got = _call(*clean, causal=False)
    for name, w in ref.dot_attention(q, k, v, causal=False, dout=dout).items():
        ref.close(got[name], *w, name)
    for which, name in enumerate(("q", "k", "v", "dout")):
        for bad, at in ((float("nan"), N - 3), (float("inf"), N // 2), (-float("inf"), 5)):
            t = [x.clone() for x in clean]
            t[which][B - 1, at, t[which].shape[2] - 1, D // 2 + 1] = bad
            got = _call(*t, causal=False)
            for result, w in _plain(*t).items():
                assert torch.equal(torch.isfinite(got[result]), torch.isfinite(w)), f"{bad} in {name}: {result}"


# B, N, H, Hkv, D and every sequence's filled length: the first has fewer keys than queries
FILLED = [
    (2, 70, 2, 2, 64, [45, 70]),
    (2, 450, 40, 20, 128, [301, 450]),
    (4, 390, 64, 64, 128, [333, 390, 128, 390]),
    (1, 700, 16, 4, 128, [591]),
    (1, 2100, 3, 1, 64, [2017]),
    (5, 300, 48, 48, 64, [257, 300, 300, 300, 300]),
    (1, 900, 2, 1, 16, [899]),
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("size", FILLED, ids=str)
def test_keys_behind_the_filled_length(size, bad, dt):
    """They get zeros, whatever a query that sees nothing or one that sees every key before them
    holds, and of the queries the first changes no other result."""
    B, N, H, Hkv, D, lens = size
    print(f"\n[dot] filled {size} {bad} {dt}", flush=True)
    L = lens[0]
    k_lens = torch.tensor(lens, dtype=torch.int32).cuda()
    clean = _inputs(B, N, N, H, Hkv, D, dt, seed=N + 7)
    want = ref.dot_attention(*clean[:3], k_lens=k_lens, dout=clean[3])
    for which, name in ((0, "q"), (3, "dout")):
        t = [x.clone() for x in clean]
        t[which][0, 0] = bad  # (at position L - N)
        t[which][0, N - L - 1] = bad
        got = _call(*t, k_lens=k_lens)
        for result, w in want.items():
            ref.close(got[result], *w, f"{name} of queries without a key: {result}")
        t[which][0, N - 1] = bad  # (the last one sees all keys)
        got = _call(*t, k_lens=k_lens)
        for result in ("dk", "dv"):
            assert (got[result][0, L:] == 0).all(), f"{name} of the last query: {result} behind the filled length"
            assert not torch.isfinite(got[result][0, :L]).any() or (name, result) == ("dout", "dk"), result
            ref.close(got[result][1:], *(x[1:] for x in want[result]), f"{result} of the other sequences")
        assert not torch.isfinite(got["dq"][0, N - 1]).any()
        ref.close(got["dq"][0, :N - 1], *(x[0, :N - 1] for x in want["dq"]), "dq of the other queries")


@pytest.mark.parametrize("window", [0, 45])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", FORMS, ids=str)
def test_what_a_value_reaches(size, dt, window):
    """One infinity or NaN, or a column of them, in q, k, v or the upstream gradient under a
    mask: what sees it by the formulas is not finite, everything else is as without it."""
    B, N, H, Hkv, D = size
    print(f"\n[dot] reach {size} {dt} {window}", flush=True)
    G, hk = H // Hkv, Hkv - 1
    heads = slice(hk * G, H)  # the last group
    clean = _inputs(B, N, N, H, Hkv, D, dt, seed=N + 1)
    want = ref.dot_attention(*clean[:3], window=window, dout=clean[3])
    see = ref.visible(1, N, N, True, window, device="cuda")[0][0]  # [query, key]
    nan, inf = float("nan"), float("inf")

    def check(which, where, value, label, **reached):
        """`reached`: positions (bool [N]) of each result that are not finite, or ([N], column)."""
        t = [x.clone() for x in clean]
        t[which][(0, *where)] = value
        got = _call(*t, window=window)
        for name, (w, bound) in want.items():
            bad = torch.zeros(w.shape, dtype=torch.bool, device="cuda")
            if name in reached:
                at, column = reached[name] if isinstance(reached[name], tuple) else (reached[name], slice(None))
                if name == "lse":
                    bad[0, heads] = at
                else:
                    bad[0, :, slice(hk, None) if name in ("dk", "dv") else heads, column] = at[:, None, None] if isinstance(column, slice) \
                        else at[:, None]
            assert not torch.isfinite(got[name][bad]).any(), f"{label}: {name} is finite where it is reached"
            ref.close(torch.where(bad, w, got[name].double()), w, bound, f"{label}: {name}")

    everyone = torch.ones(N, dtype=torch.bool, device="cuda")
    for j, value in ((3, inf), (N // 2 + 1, nan), (N - 1, -inf)):
        rows = see[:, j]
        keys = see[rows].any(0)  # seen by a query that sees j
        check(2, (j, hk, 1), value, f"v at {j}", out=(rows, 1), dq=rows, dk=keys)
        check(1, (j, hk, 1), nan, f"k at {j}", out=rows, lse=rows, dq=rows, dk=keys, dv=keys)
    check(2, (slice(None), hk, 2), nan, "a column of v", out=(everyone, 2), dq=everyone, dk=everyone)
    if G == 1:  # (one query head of a group)
        for i, value in ((0, inf), (N // 2 + 1, nan), (N - 5, -inf)):
            row, keys = torch.arange(N, device="cuda") == i, see[i]
            check(3, (i, H - 1, 1), value, f"dout at {i}", dq=row, dk=keys, dv=(keys, 1))
            check(0, (i, H - 1, 1), nan, f"q at {i}", out=row, lse=row, dq=row, dk=keys, dv=keys)
        check(3, (slice(None), H - 1, 2), nan, "a column of dout", dq=everyone, dk=everyone, dv=(everyone, 2))

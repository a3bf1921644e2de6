"""Windows, and documents of any numbers, in every form of the backward's key side against float64."""

import pytest
import torch

import layers_reference as ref
from paper_2507_02754_amd import load_library, simplicial_dot_attn_bwd, simplicial_dot_attn_fwd

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    load_library()


def _normal(*shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


# B, N, H, Hkv, D, window: one head's keys see H / Hkv (window + 128) rows of H / Hkv N
SIZES = [
    (1, 700, 16, 1, 128, 131),   # blocks of keys shared by workgroups
    (1, 700, 16, 1, 128, 600),
    (1, 700, 40, 1, 64, 131),
    (1, 700, 16, 4, 128, 131),   # blocks of 32 keys
    (1, 1500, 12, 4, 64, 200),
    (3, 1400, 17, 17, 128, 150),  # two groups of wavefronts
    (4, 420, 64, 64, 128, 33),   # whole blocks
    (2, 900, 12, 12, 64, 1),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_float64(size, causal):
    B, N, H, Hkv, D, window = size
    print(f"\n[dot] window {size} {causal}", flush=True)
    q, dout = (_normal(B, N, H, D, seed=N + i, dtype=BF) for i in range(2))
    k, v = (_normal(B, N, Hkv, D, seed=N + 2 + i, dtype=BF) for i in range(2))
    ids = ((torch.arange(N) * 5) // (2 * N) + (torch.arange(N) >= N - 40).int() * 3).to(torch.int32).expand(B, N).contiguous().cuda()
    slopes = (2.0 ** (-8.0 * torch.arange(1, H + 1) / H)).cuda()
    prefix = torch.arange(B, dtype=torch.int32).cuda() * 50 + 20
    for opts in (dict(), dict(softcap=4.0, slopes=slopes), dict(documents=ids), dict(prefix=prefix)):
        opts.update(causal=causal, window=window)
        lo = torch.empty_like(q)
        out, lse = simplicial_dot_attn_fwd(q, k, v, out_lo=lo, **opts)
        grads = simplicial_dot_attn_bwd(q, k, v, out, dout, lse, out_lo=lo, **opts)
        torch.cuda.synchronize()
        want = ref.dot_attention(q, k, v, dout=dout, **opts)
        for name, x in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *grads)):
            ref.close(x, *want[name], f"{sorted(opts)}: {name}")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", [s[:5] for s in SIZES], ids=str)
def test_documents_of_any_number(size, dt):
    """The largest number, 0 and others in runs of any length, padding of several negative numbers
    between them, behind them, in whole blocks and alternating with a document."""
    B, N, H, Hkv, D = size
    print(f"\n[dot] documents {size} {dt}", flush=True)
    g = torch.Generator().manual_seed(N + D)
    q, dout = (_normal(B, N, H, D, seed=N + i, dtype=dt) for i in range(2))
    k, v = (_normal(B, N, Hkv, D, seed=N + 2 + i, dtype=dt) for i in range(2))
    numbers = torch.tensor([2 ** 31 - 1, 0, -(2 ** 31), 7, -1, 2 ** 31 - 2])
    runs = torch.randint(1, 120, (B, N), generator=g)
    ids = torch.stack([numbers[torch.arange(N) % 6].repeat_interleave(r)[:N] for r in runs])
    ids[0, N // 2:N // 2 + 70:2] = -5
    ids[B - 1, N - 45:] = -1
    ids = ids.to(torch.int32).cuda()
    for opts in (dict(documents=ids), dict(documents=ids, causal=False)):
        lo = torch.empty_like(q) if dt == BF else None
        out, lse = simplicial_dot_attn_fwd(q, k, v, out_lo=lo, **opts)
        grads = simplicial_dot_attn_bwd(q, k, v, out, dout, lse, out_lo=lo, **opts)
        torch.cuda.synchronize()
        want = ref.dot_attention(q, k, v, dout=dout, **opts)
        for name, x in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *grads)):
            ref.close(x, *want[name], f"{sorted(opts)}: {name}")

"""Norm and rotation of queries and keys on the GPU against float64."""

import pytest
import torch

import layers_reference as ref
from paper_2507_02754_amd import (load_library, norm_rotate, rotary_freqs, simplicial_attn_det_fwd,
                                  simplicial_norm_rotate_bwd, simplicial_norm_rotate_fwd)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    load_library()


def _normal(*shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


BF, F32 = torch.bfloat16, torch.float32
CASES = [
    # B, N, heads, D, dtype, layout, pairs, eps, weight type, first position
    (1, 1, (1,), 16, BF, "half", 8, 1e-6, None, 0),
    (4, 1, (16, 4), 128, BF, "half", 64, 1e-6, BF, 120000),
    (2, 37, (4, 2), 64, BF, "half", 32, 1e-5, F32, 7),
    (2, 37, (3, 3, 1), 64, F32, "half", 16, 1e-6, F32, 1000000),  # part of the head rotated
    (1, 65, (8, 2, 2), 128, BF, "axis", 42, 0.0, None, 3),
    (1, 130, (2, 1), 128, F32, "axis", 17, 1e-6, BF, 50),
    (3, 19, (2,), 32, F32, "axis", 10, 1e-6, F32, 0),
    (1, 50, (2, 2), 16, BF, "axis", 5, 1e-6, None, 0),
    (2, 33, (5, 1), 32, BF, "pairs", 16, 1e-6, BF, 4),
    (1, 257, (4,), 128, F32, "pairs", 5, 1e-6, F32, 9),
    (1, 40, (4, 4), 16, F32, "pairs", 8, None, None, 123456789),  # rotation alone
    (2, 21, (4, 4), 64, BF, "half", 0, 1e-6, BF, 0),  # norm alone
    (1, 3000, (8, 8), 128, BF, "half", 64, 1e-6, BF, 0),  # several rows a lane group
    (1, 9001, (16, 4, 4), 64, BF, "half", 32, 1e-6, F32, 11),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_forward_and_backward(case):
    B, N, heads, D, dt, layout, pairs, eps, wdt, start = case
    print(f"\n[norm_rotate] {case}", flush=True)
    xs = [_normal(B, N, h, D, seed=10 + i, dtype=dt, scale=2.0) for i, h in enumerate(heads)]
    dys = [_normal(B, N, h, D, seed=20 + i, dtype=dt) for i, h in enumerate(heads)]
    ws = None if wdt is None else [1 + _normal(D, seed=30 + i, dtype=wdt, scale=0.2) for i in range(len(heads))]
    freqs = rotary_freqs(pairs) if pairs else None
    opts = dict(eps=eps, freqs=freqs, layout=layout, start=start)
    ys = simplicial_norm_rotate_fwd(xs, ws, **opts)
    dxs, dws = simplicial_norm_rotate_bwd(xs, dys, ws, **opts)
    torch.cuda.synchronize()
    positions = (start + torch.arange(N, device="cuda")).expand(B, N)
    for i, x in enumerate(xs):
        y, yb, (dx, dxb), dw = ref.norm_rotate(x, ws and ws[i], eps, freqs or (), layout, positions, dys[i])
        ref.close(ys[i], y, yb, f"y[{i}]")
        ref.close(dxs[i], dx, dxb, f"dx[{i}]")
        if ws:
            ref.close(dws[i], dw[0], dw[1], f"dw[{i}]")
        else:
            assert dws[i] is None


@pytest.mark.parametrize("layout,pairs", [("half", 24), ("pairs", 31), ("axis", 20)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_views_and_positions(layout, pairs, dt):
    """q, k and k' as slices of one projection's output, positions of every sequence
    its own, out of order and negative among them, and the same through autograd."""
    B, N, D = 2, 29, 64
    print(f"\n[norm_rotate] views {layout} {dt}", flush=True)
    both = _normal(B, N, 9, D, seed=1, dtype=dt)
    xs = list(both.split([4, 2, 3], dim=2))
    assert not xs[0].is_contiguous()
    positions = torch.randint(-5000, 200000, (B, N), generator=torch.Generator().manual_seed(3)).cuda()
    ws = [1 + _normal(D, seed=5 + i, scale=0.3) for i in range(3)]
    leaves = [t.clone().requires_grad_(True) for t in ws]
    src = both.clone().requires_grad_(True)
    dys = [_normal(*x.shape, seed=50 + i, dtype=dt) for i, x in enumerate(xs)]
    freqs = rotary_freqs(pairs)
    ys = norm_rotate(src.split([4, 2, 3], dim=2), leaves, freqs=freqs, layout=layout, positions=positions)
    grads = torch.autograd.grad(ys, [src, *leaves], dys)
    torch.cuda.synchronize()
    at = 0
    for i, x in enumerate(xs):
        y, yb, (dx, dxb), dw = ref.norm_rotate(x, ws[i], 1e-6, freqs, layout, positions, dys[i])
        ref.close(ys[i], y, yb, f"y[{i}]")
        ref.close(grads[0][:, :, at:at + x.shape[2]], dx, dxb, f"dx[{i}]")
        ref.close(grads[1 + i], *dw, f"dw[{i}]")
        at += x.shape[2]
    shared = norm_rotate(xs, ws, freqs=freqs, layout=layout, positions=positions[0])
    own = norm_rotate(xs, ws, freqs=freqs, layout=layout, positions=positions[:1].expand(B, N))
    assert all(torch.equal(a, b) for a, b in zip(shared, own))


def test_unaligned_views_are_copied():
    x = _normal(1, 5, 2, 68, seed=2, dtype=BF)[..., 4:]
    y = norm_rotate([x], freqs=rotary_freqs(32))[0]
    z = norm_rotate([x.contiguous()], freqs=rotary_freqs(32))[0]
    assert torch.equal(y, z)


def test_rows_of_zeros_and_values_out_of_range():
    """A row of zeros without eps gives zeros and zero gradients; infinities and NaN stay
    in their rows and, where nothing turns them, in their components."""
    x = _normal(1, 4, 2, 64, seed=4)
    x[0, 1, 0] = 0
    x[0, 2, 1, 3] = float("nan")
    dy = _normal(1, 4, 2, 64, seed=5)
    y = simplicial_norm_rotate_fwd([x], eps=0.0, freqs=rotary_freqs(32))[0]
    dx = simplicial_norm_rotate_bwd([x], [dy], eps=0.0, freqs=rotary_freqs(32))[0][0]
    assert (y[0, 1, 0] == 0).all() and (dx[0, 1, 0] == 0).all()
    bad = torch.zeros(1, 4, 2, dtype=torch.bool, device="cuda")
    bad[0, 2, 1] = True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all() and torch.isfinite(dx[~bad]).all()
    z = torch.zeros(1, 1, 1, 64, device="cuda")
    z[..., 63] = float("inf")  # component of no pair, beside one
    for layout, n in (("half", 24), ("pairs", 31), ("axis", 21)):
        t = simplicial_norm_rotate_fwd([z], eps=None, freqs=rotary_freqs(n), layout=layout, start=5)[0]
        assert torch.equal(t, z), layout


def test_determinant_logits_see_position_differences_alone():
    """q, k and k' rotated about an axis of each 3-component chunk: moving all positions
    by the same distance leaves the determinant attention as it is."""
    B, N, H, D = 1, 96, 2, 64
    xs = [_normal(B, N, H, D, seed=70 + i, dtype=F32) for i in range(3)]
    v, vp = (_normal(B, N, H, D, seed=80 + i, dtype=F32) for i in range(2))
    outs = []
    for start in (0, 4000):
        q, k, kp = norm_rotate(xs, eps=0.0, freqs=rotary_freqs(21), layout="axis", start=start)
        outs.append(simplicial_attn_det_fwd(q, k, kp, v, vp, 24, 8, 0.05)[0])
    plain = simplicial_attn_det_fwd(*norm_rotate(xs, eps=0.0), v, vp, 24, 8, 0.05)[0]
    torch.cuda.synchronize()
    # logits of 21 determinants of components up to ~4 (|det| ~ 20), each turn off by 8 U: off by 21 * 20 * 3 * 8 U * 0.05 < 1e-5
    assert (outs[0] - outs[1]).abs().max() < 1e-4
    assert (outs[0] - plain).abs().max() > 1e-2


def test_gradients_against_differences():
    """float32 directional differences of the whole map, q, k and the weights."""
    xs = [_normal(1, 6, 2, 32, seed=90 + i) for i in range(2)]
    ws = [1 + _normal(32, seed=95 + i, scale=0.2) for i in range(2)]
    dys = [_normal(1, 6, 2, 32, seed=97 + i) for i in range(2)]
    freqs = rotary_freqs(16)
    leaves = [t.clone().requires_grad_(True) for t in (*xs, *ws)]
    ys = norm_rotate(leaves[:2], leaves[2:], freqs=freqs, start=11)
    grads = torch.autograd.grad(ys, leaves, dys)
    step = 2.0 ** -8
    for i in range(4):
        d = _normal(*leaves[i].shape, seed=100 + i)
        ends = []
        for sign in (1, -1):
            t = [x.detach().clone() for x in leaves]
            t[i] += sign * step * d
            y = norm_rotate(t[:2], t[2:], freqs=freqs, start=11)
            ends.append(sum((a.double() * b.double()).sum() for a, b in zip(y, dys)))
        slope = (ends[0] - ends[1]) / (2 * step)
        want = (grads[i].double() * d.double()).sum()
        # third derivatives of the norm times step^2, and float32 sums over 2 step
        size = (grads[i].double() * d.double()).abs().sum()
        assert abs(slope - want) <= 1e-3 * size, i


def test_results_repeat_and_captured_graphs():
    B, N, D = 2, 700, 128
    xs = [_normal(B, N, h, D, seed=h, dtype=BF) for h in (8, 2)]
    dys = [_normal(B, N, h, D, seed=h + 9, dtype=BF) for h in (8, 2)]
    ws = [1 + _normal(D, seed=3 + i, dtype=BF, scale=0.1) for i in range(2)]
    pos = torch.arange(N, device="cuda")
    opts = dict(freqs=rotary_freqs(64), positions=pos)

    def both():
        return (*simplicial_norm_rotate_fwd(xs, ws, **opts), *(t for p in simplicial_norm_rotate_bwd(xs, dys, ws, **opts) for t in p))

    eager = both()
    again = both()
    assert all(torch.equal(a, b) for a, b in zip(eager, again))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for shift in (1, 2, 3):
        pos += shift
        eager = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), shift

"""Log probabilities of given tokens, entropy and top alternatives on the GPU against float64."""

import pytest
import torch

import layers_reference as ref
from paper_2507_02754_amd import (load_library, simplicial_logprobs_bwd, simplicial_logprobs_fwd, token_logprobs)

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NAMES = ("logprob", "entropy", "lse", "top_logprob", "top_index")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    load_library()


def _logits(R, V, dt, seed, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((R, V), generator=g) * scale).to(dt).cuda()


def _grads(R, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(R, generator=g).cuda() for _ in range(3)]


def _check(x, targets, top, label, grads=None):
    got = dict(zip(NAMES, simplicial_logprobs_fwd(x, targets, top)))
    if grads is not None:
        got["dx"] = simplicial_logprobs_bwd(x, targets, got["lse"], got["entropy"], *grads)
    torch.cuda.synchronize()
    want = ref.logprobs(x, targets, top, grads)
    for name, w in want.items():
        if name == "top_index":
            assert torch.equal(got[name], w), f"{label}: top_index"
        else:
            ref.close(got[name], *w, f"{label}: {name}")
    return got


SIZES = [(1, 1, 1), (1, 2, 2), (5, 3, 1), (2, 7, 7), (3, 63, 5), (4, 64, 32), (2, 129, 20), (510, 512, 0), (3, 1000, 8), (7, 4097, 5),
         (8, 50001, 8), (1, 50001, 32), (600, 2049, 3), (600, 8200, 4), (520, 33000, 2), (520, 70001, 1), (2, 140003, 32)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_float64(size, dt):
    """All numbers of slices, chunks a thread and threads; odd rows, whose starts
    are not 16-byte aligned; bf16 logits tie often."""
    R, V, top = size
    print(f"\n[logprobs] {size} {dt}", flush=True)
    x = _logits(R, V, dt, seed=V)
    targets = torch.randint(0, V, (R,), generator=torch.Generator().manual_seed(R)).cuda()
    if R > 2:
        targets[1] = -100  # left out
    _check(x, targets, top, str(size), _grads(R, V + 1))


@pytest.mark.parametrize("dt", [BF, F32])
def test_views_of_a_padded_vocabulary(dt):
    """Rows apart by more than the vocabulary: rows of dlogits and logits are aligned differently."""
    for V, pad in ((1001, 1024), (1003, 1005), (4000, 4001)):
        base = _logits(6, pad, dt, seed=V)
        base[:, V:] = float("nan")
        x = base[:, :V]
        _check(x, torch.arange(6).cuda(), 4, f"view {V} of {pad}", _grads(6, V))
        for start in (1, 5):
            part = base[:, start:V - 9]  # rows that begin anywhere
            _check(part, torch.arange(6).cuda(), 4, f"view {start} .. {V - 9} of {pad}", _grads(6, V))


@pytest.mark.parametrize("dt", [BF, F32])
def test_ties_and_orders(dt):
    """Rows of equal values, ascending, descending, few distinct values and signed zeros: the
    lowest token first, whatever the number of candidates."""
    V = 20011
    x = torch.zeros((6, V))
    x[1] = torch.arange(V) / 64.0
    x[2] = -torch.arange(V) / 64.0
    x[3] = torch.arange(V) % 3
    x[4, ::2] = -0.0
    x[5] = -3.0
    x[5, 17::1000] = 5.0
    _check(x.to(dt).cuda(), torch.tensor([0, V - 1, 5, 2, 1, 17]).cuda(), 32, "ties")
    many = torch.zeros((700, V))
    many[:, 1::7] = 1.0
    _check(many.to(dt).cuda(), torch.zeros(700, dtype=torch.int64).cuda(), 9, "ties of many rows")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [70, 5000, 50001])
def test_infinities_and_nan(V, dt):
    """Masked tokens (-inf, and the type's lowest value), a row of nothing else, rows with
    NaN or +inf, a target that is masked, left out or past the vocabulary."""
    x = _logits(9, V, dt, seed=3)
    x[0, 5:] = -float("inf")
    x[1] = -float("inf")
    x[2] = -float("inf")
    x[2, V - 1] = 2.5
    x[3, 1::2] = torch.finfo(dt).min
    x[4, V // 2] = float("nan")
    x[5, 3] = float("inf")
    x[6] = torch.finfo(dt).min
    x[7, 2] = 60.0
    targets = torch.tensor([20, 0, V - 1, 1, 0, 3, 2, V, -1]).cuda()
    got = dict(zip(NAMES, simplicial_logprobs_fwd(x, targets, 6)))
    want = ref.logprobs(x, targets, 6, _grads(9, 2))
    got["dx"] = simplicial_logprobs_bwd(x, targets, got["lse"], got["entropy"], *_grads(9, 2))
    torch.cuda.synchronize()
    whole = [0, 1, 2, 3, 6, 7, 8]
    for name, w in want.items():
        if name == "top_index":
            assert torch.equal(got[name][whole], w[whole])
        else:
            # a masked target's gradient passes through a log probability of -inf as any other
            ref.close(got[name][whole], w[0][whole], w[1][whole], name)
    for row in (4, 5):
        for name in NAMES[:4]:
            assert torch.isnan(got[name][row]).all(), (row, name)
        assert torch.isnan(got["dx"][row]).all()
        assert got["top_index"][row].unique().numel() == 6 and int(got["top_index"][row].max()) < V
    assert int(got["top_index"][4, 0]) == V // 2 and int(got["top_index"][5, 0]) == 3
    # a row without probability whose target is left out
    lp = simplicial_logprobs_fwd(x[1:2], torch.tensor([-1]).cuda())[0]
    assert lp.item() == 0.0


def test_autograd_of_each_output():
    x = _logits(12, 1001, F32, seed=1).view(3, 4, 1001).requires_grad_(True)
    targets = torch.randint(0, 1001, (3, 4), generator=torch.Generator().manual_seed(1)).cuda()
    g = _grads(12, 5)
    r = token_logprobs(x, targets, top=3)
    assert r.top_tokens.shape == (3, 4, 3) and r.entropy.shape == (3, 4)
    assert not r.top_logprobs.requires_grad
    for pick in ((0,), (1,), (2,), (0, 1, 2)):
        dx, = torch.autograd.grad([r[i] for i in pick], [x], [g[i].view(3, 4) for i in pick], retain_graph=True)
        names = {0: 0, 1: 1, 2: 2}
        grads = [g[names[i]] if i in pick else None for i in range(3)]
        want = ref.logprobs(x.detach().view(12, -1), targets.view(-1), grads=grads)["dx"]
        ref.close(dx.view(12, -1), *want, str(pick))
    assert token_logprobs(x[:, :, ::2], targets // 2).logprob.shape == (3, 4)


def test_gradient_against_differences():
    x = _logits(3, 40, F32, seed=9)
    targets = torch.tensor([3, -1, 39]).cuda()
    g = _grads(3, 4)
    leaf = x.clone().requires_grad_(True)
    dx, = torch.autograd.grad(list(token_logprobs(leaf, targets)[:3]), [leaf], g)
    d = _logits(3, 40, F32, seed=10, scale=1.0)
    step = 2.0 ** -7
    ends = [sum((a.double() * b.double()).sum() for a, b in zip(token_logprobs(x + s * step * d, targets)[:3], g)) for s in (1, -1)]
    slope, want = (ends[0] - ends[1]) / (2 * step), (dx.double() * d.double()).sum()
    assert abs(slope - want) <= 1e-3 * (dx.double() * d.double()).abs().sum()


def test_long_rows_pass_32_bits():
    """Rows whose offsets pass 2^31 elements: the last rows of a view with far apart rows."""
    V, stride, R = 300, 1 << 22, 1030  # 4.3e9 elements
    base = torch.empty(R * stride, dtype=BF, device="cuda")
    x = base.as_strided((R, V), (stride, 1))
    x.copy_(_logits(R, V, BF, seed=6))
    targets = (torch.arange(R) % V).cuda()
    _check(x, targets, 3, "far rows", _grads(R, 8))


def test_captured_graph_replays():
    x = _logits(8, 50001, BF, seed=2)
    targets = torch.arange(8).cuda()
    g = _grads(8, 1)

    def both():
        r = simplicial_logprobs_fwd(x, targets, 8)
        return (*r, simplicial_logprobs_bwd(x, targets, r[2], r[1], *g))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        x.copy_(_logits(8, 50001, BF, seed=20 + i))
        targets += 1
        eager = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), i

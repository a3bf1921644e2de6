"""A constant added to a row of logits changes no gradient: probabilities depend on
differences alone, whatever the size of lse."""

import pytest
import torch

import layers_reference as ref
from paper_2507_02754_amd import load_library, simplicial_logprobs_bwd, simplicial_logprobs_fwd, token_logprobs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    load_library()


def _grads(R, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(R, generator=g).cuda() for _ in range(3)]


# rows of one workgroup, of several (their results joined), and of a full chip
@pytest.mark.parametrize("size", [(4, 40), (3, 4097), (2, 50001), (600, 2049)], ids=str)
@pytest.mark.parametrize("dt, step, shift", [(F32, 2.0 ** -6, 1e4), (F32, 2.0 ** -6, -1e4), (F32, 2.0 ** -3, 1e6), (F32, 2.0 ** -3, -1e6),
                                             (F32, 8.0, 1e8), (F32, 2.0 ** -24, 0.0), (BF, 64.0, 10240.0), (BF, 8192.0, 2.0 ** 20)], ids=str)
def test_shifted_rows(size, dt, step, shift):
    """Logits on a grid of `step`, which the shifted ones keep (so that both are exact): the
    gradient within the bounds of the unshifted row's."""
    R, V = size
    g = torch.Generator().manual_seed(V)
    x = (torch.randn((R, V), generator=g) * 2 * max(1.0, step)).div(step).round().mul(step).cuda()
    moved = (x.double() + shift).to(dt)
    assert torch.equal(moved.double(), x.double() + shift)
    targets = torch.randint(0, V, (R,), generator=g).cuda()
    targets[0] = -1  # left out
    grads = _grads(R, V)
    want = ref.logprobs(x.to(dt) if dt == F32 else x, targets, grads=grads)["dx"]
    # What a bf16 gradient's own rounding adds; and the exponential is 0 where it is below the least normal
    # number: the gradient is p times a factor of no more than |d_lse| + |d_logprob| + |d_entropy| (|log p| +
    # entropy), so that p < 2^-126 as 0 takes up to 2^-126 of that factor.
    logp = torch.log_softmax(x.double(), 1)
    entropy = -(logp.exp() * logp).sum(1, keepdim=True)
    glp, gh, gl = (t.double().abs()[:, None] for t in grads)
    want = (want[0], want[1] + (ref.HALF[dt] - ref.U) * want[0].abs() + 2.0 ** -126 * (gl + glp + gh * (logp.abs() + entropy)))
    r = simplicial_logprobs_fwd(moved, targets, lse_lo=True)
    assert r[2].shape == (2, R)
    direct = simplicial_logprobs_bwd(moved, targets, r[2], r[1], *grads)
    leaf = moved.clone().requires_grad_(True)
    dx, = torch.autograd.grad(list(token_logprobs(leaf, targets)[:3]), [leaf], grads)
    assert torch.equal(dx, direct)
    ref.close(dx, *want, f"{size} {dt} + {shift}")
    # lse and what rounding took from it: twice the digits (the logarithm itself is float32's)
    lse = torch.logsumexp(moved.double(), 1)
    inner = torch.logsumexp(x.double(), 1)
    both = r[2].double().sum(0)
    assert torch.equal(r[2][0], simplicial_logprobs_fwd(moved, targets)[2])
    assert ((both - lse).abs() <= ref.logprobs(x, targets)["lse"][1] + 2 * ref.U * inner.abs()).all()


def test_lse_changed_in_place_is_noticed():
    x = torch.randn((3, 50), generator=torch.Generator().manual_seed(1)).cuda().requires_grad_(True)
    r = token_logprobs(x, torch.tensor([1, 2, 3]).cuda())
    with torch.no_grad():
        r.lse.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        r.logprob.sum().backward()

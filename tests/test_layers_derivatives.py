"""Derivatives that the layers' operators do not have are refused, not left out: with the
library replaced by constants (these run without a GPU)."""

import contextlib

import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2507_02754_amd import dot_attention, layers_autograd, layers_binding, norm_rotate, rotary_freqs, token_logprobs


@pytest.fixture
def stub(monkeypatch):
    """The binding without its checks and its library: zeros of the results' shapes."""
    class Rotate:
        def __init__(self, xs, *rest):
            self.xs = xs

        def forward(self):
            return [torch.zeros_like(x) for x in self.xs]

    class Dot:
        def __init__(self, q, *rest):
            self.q = q

        def forward(self, out_lo=None):
            return torch.zeros_like(self.q), torch.zeros(1)

    def logprobs(logits, targets, top=0, lse_lo=False):
        return [torch.zeros(len(targets)) for _ in range(5)]

    monkeypatch.setattr(layers_autograd, "_RotateCall", Rotate)
    monkeypatch.setattr(layers_autograd, "_DotCall", Dot)
    monkeypatch.setattr(layers_autograd, "simplicial_logprobs_fwd", logprobs)


X, W = torch.ones(1, 4, 2, 64), torch.ones(64)
TARGETS = torch.zeros(4, dtype=torch.int64)
CALLS = {
    "x": (X, lambda t: norm_rotate([X, t])),
    "weight": (W, lambda t: norm_rotate([X], weights=[t])),
    "q": (X, lambda t: dot_attention(t, X, X)),
    "k": (X, lambda t: dot_attention(X, t, X)),
    "v": (X, lambda t: dot_attention(X, X, t)),
    "slopes": (W[:2], lambda t: dot_attention(X, X, X, slopes=t)),
    "scale": (W[0], lambda t: dot_attention(X, X, X, scale=t)),
    "softcap": (W[0], lambda t: dot_attention(X, X, X, softcap=t)),
    "eps": (W[0], lambda t: norm_rotate([X], eps=t)),
    "freqs": (W[:32], lambda t: norm_rotate([X], freqs=t)),
    "an angle": (W[0], lambda t: norm_rotate([X], freqs=[t] * 32)),
    "logits": (torch.ones(4, 8), lambda t: token_logprobs(t, TARGETS)),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("mode", [contextlib.nullcontext, torch.no_grad], ids=["grad", "no_grad"])
def test_forward_mode_is_refused(stub, name, mode):
    x, call = CALLS[name]
    with mode(), forward_ad.dual_level():
        call(x)  # (no tangent: as ever)
        with pytest.raises(NotImplementedError, match="forward-mode"):
            call(forward_ad.make_dual(x, torch.ones_like(x)))


@pytest.mark.parametrize("name", ["slopes", "scale", "softcap", "eps", "freqs", "an angle"])
def test_options_are_not_trained(stub, name):
    """A tensor that asks for a gradient, where gradients are formed, whether or not of the
    other inputs."""
    x, call = CALLS[name]
    leaf = x.clone().requires_grad_(True)
    with pytest.raises(ValueError, match="no gradient"):
        call(leaf)
    with torch.no_grad():
        call(leaf)
    call(leaf.detach())


def test_angles_are_kept_as_numbers():
    """What is kept of a call's angles is found again, whatever they were given as."""
    want = rotary_freqs(32)
    x = torch.tensor(want, dtype=torch.float64)
    found = [layers_binding.rotary_angles(f) for f in (want, list(want), x, list(x), iter(want), x.numpy())]
    assert all(f is found[0] for f in found) and tuple(found[0][0]) == want and found[0][1] == 32
    assert layers_binding.rotary_angles(None)[1] == 0
    for i in range(100):
        layers_binding.rotary_angles([torch.tensor(float(i))])
    assert len(layers_binding._ANGLES) <= 64 and all(type(f) is float for kept in layers_binding._ANGLES for f in kept)


def test_weights_of_another_number(stub):
    """Refused alike whether or not a gradient is asked for; any iterable will do."""
    leaf = X.clone().requires_grad_(True)
    for x in (X, leaf):
        for weights in ([], [W, W], [None], (w for w in ())):
            with pytest.raises(ValueError, match="weight for every"):
                norm_rotate([x], weights=weights)
    norm_rotate([X, X], weights=(w for w in (W, W)))

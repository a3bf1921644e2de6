"""The operators of include/simplicial_layers.h as the layers call them, together."""

import copy

import pytest
import torch
import torch.nn.functional as F
import torch.utils.checkpoint

import layers_reference as ref
from paper_2507_02754_amd import (DotProductAttention, InterleavedStack, SimplicialAttention, dot_attention, load_library,
                                  norm_rotate, rotary_freqs, token_logprobs)

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    load_library()


def _seeded(module, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    with torch.no_grad():
        for p in module.parameters():
            if p.dim() == 2:
                p.copy_(torch.randn(p.shape, generator=g, device="cuda") * p.shape[1] ** -0.5)
            else:
                p.copy_(1 + 0.2 * torch.randn(p.shape, generator=g, device="cuda"))
    return module


def _turn64(x, freqs):
    positions = torch.arange(x.shape[1], device=x.device).expand(x.shape[:2])
    return ref.turn(x, positions, freqs, "half")


def _layer64(layer, x, documents, prefix):
    """The layer in float64 with plain torch operations."""
    m = copy.deepcopy(layer).double()
    b, n, _ = x.shape
    h, hk, d = m.n_heads, m.kv_heads, m.head_dim
    q, k, v = m.wqkv(x).view(b, n, h + 2 * hk, d).split([h, hk, hk], dim=2)
    if m.qk_norm:
        q, k = (t * (t.square().mean(-1, keepdim=True) + 1e-6) ** -0.5 * w for t, w in ((q, m.q_norm), (k, m.k_norm)))
    if m.freqs is not None:
        q, k = (_turn64(t, m.freqs) for t in (q, k))
    see, distance = ref.visible(b, n, n, True, m.window, documents, prefix, device=x.device)
    k, v = (t.repeat_interleave(h // hk, 2).transpose(1, 2) for t in (k, v))
    s = q.transpose(1, 2) @ k.transpose(2, 3) * d ** -0.5
    if m.softcap:
        s = m.softcap * torch.tanh(s / m.softcap)
    if m.alibi:
        s = s - (2.0 ** (-8.0 * torch.arange(1, h + 1, device=x.device) / h)).double()[:, None, None] * distance[:, None]
    s = s.masked_fill(~see[:, None], -torch.inf)
    o = torch.softmax(s, -1).nan_to_num(0.0) @ v
    return m.wo(o.transpose(1, 2).reshape(b, n, h * d)), m


OPTIONS = [
    dict(qk_norm=True, rope_base=10000.0, attn_dtype=F32),
    dict(kv_heads=2, rope_base=500.0, softcap=5.0, window=40, attn_dtype=F32),
    dict(kv_heads=1, qk_norm=True, alibi=True),
    dict(attn_dtype=BF),
]


@pytest.mark.parametrize("options", OPTIONS, ids=[str(i) for i in range(len(OPTIONS))])
@pytest.mark.parametrize("masks", ["none", "documents", "prefix"])
def test_layer_against_float64(options, masks):
    """Output, input gradient and weight gradients of the layer in float32 parameters."""
    torch.manual_seed(2)
    b, n, dm, h, d = 2, 90, 96, 4, 32
    layer = _seeded(DotProductAttention(dm, h, d, device="cuda", dtype=F32, **options), 4)
    x = torch.randn(b, n, dm, device="cuda", requires_grad=True)
    dy = torch.randn(b, n, dm, device="cuda")
    documents = prefix = None
    if masks == "documents":
        documents = (torch.arange(n, device="cuda") // 37).to(torch.int32).repeat(b, 1)
        documents[0, 80:] = -1
    if masks == "prefix":
        prefix = torch.tensor([10, 55], dtype=torch.int32, device="cuda")
    y = layer(x, documents, prefix)
    grads = torch.autograd.grad(y, [x, *layer.parameters()], dy)
    xr = x.detach().double().requires_grad_(True)
    yr, m = _layer64(layer, xr, documents, prefix)
    want = torch.autograd.grad(yr, [xr, *m.parameters()], dy.double())
    # 2-norms: the projections' float32 sums, and in bf16 q, k, v, P, dS and the attention's results
    # rounded (each 2^-8 relative at most, a handful of them in a chain; gradients of
    # dS = P (dP - Delta) relative to terms a few times their difference)
    tol = 1e-4 if layer.attn_dtype == F32 else 8 * 2.0 ** -8
    for name, a, r in zip(["y", "dx", *[n for n, _ in layer.named_parameters()]], [y, *grads], [yr, *want]):
        err = ((a.double() - r).norm() / r.norm()).item()
        assert err <= tol, (name, err)


def test_layer_without_options_is_as_before():
    torch.manual_seed(1)
    layer = DotProductAttention(64, 2, 32, device="cuda", dtype=F32)
    x = torch.randn(2, 33, 64, device="cuda")
    q, k, v = layer.wqkv(x).float().view(2, 33, 3, 2, 32).permute(2, 0, 3, 1, 4)
    o = F.scaled_dot_product_attention(q.contiguous(), k.contiguous(), v.contiguous(), is_causal=True)
    assert torch.equal(layer(x), layer.wo(o.transpose(1, 2).reshape(2, 33, -1)))
    with pytest.raises(ValueError, match="attn_dtype"):
        layer(x, prefix=torch.zeros(2, dtype=torch.int32, device="cuda"))


def test_simplicial_layer_with_normed_heads():
    """qk_norm is norm_rotate of q, k and k' before the attention; with rows of one size by
    construction it changes nothing but their size."""
    torch.manual_seed(0)
    layer = _seeded(SimplicialAttention(128, 2, 64, 32, 16, device="cuda", dtype=F32, qk_norm=True), 9)
    x = torch.randn(1, 70, 128, device="cuda")
    y = layer(x)
    plain = SimplicialAttention(128, 2, 64, 32, 16, device="cuda", dtype=F32)
    plain.load_state_dict({k: v for k, v in layer.state_dict().items() if not k.endswith("norm")})

    class Normed(torch.nn.Module):
        def __init__(self, lin, w):
            super().__init__()
            self.lin, self.w = lin, w

        def forward(self, x):
            t = self.lin(x).view(1, 70, 2, 64).to(BF).double()
            t = t * (t.square().mean(-1, keepdim=True) + 1e-6) ** -0.5 * self.w.double()
            return t.to(BF).view(1, 70, 128)

    for name in ("q", "k", "kp"):
        setattr(plain, "w" + name, Normed(getattr(plain, "w" + name), getattr(layer, name + "_norm")))
    # both round the normed rows to bf16; a few may fall to the other side
    assert (y - plain(x)).norm() / y.norm() < 1e-2
    y.sum().backward()
    assert all(torch.isfinite(p.grad).all() and p.grad.abs().max() > 0 for p in layer.parameters())


def _stack(dtype, seed=6):
    return _seeded(InterleavedStack(vocab=300, d_model=128, n_layers=4, n_heads=2, head_dim=64, w1=32, w2=16, device="cuda", dtype=dtype,
                                    qk_norm=True, dot_options=dict(qk_norm=True, rope_base=10000.0, softcap=30.0)), seed)


def test_stack_logprobs_are_its_loss():
    """The mean of -logprob is the cross entropy of the same logits, with the same gradients
    (both in float32 from the same logits), and the alternatives are the logits' largest."""
    model = _stack(F32)
    tokens = torch.randint(0, 300, (2, 65), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    r = model.logprobs(tokens, top=4)
    loss = model.loss(tokens)
    assert abs(-r.logprob.mean().item() - loss.item()) <= 1e-5 * loss.item()
    ga = torch.autograd.grad(-r.logprob.mean(), list(model.parameters()))
    gb = torch.autograd.grad(loss, list(model.parameters()))
    for (name, _), a, b in zip(model.named_parameters(), ga, gb):
        # the bf16 attention rounds gradients that differ in the last float32 digits
        assert (a - b).norm() <= 2e-2 * b.norm() + 1e-8, name
    with torch.no_grad():
        logits = model(tokens[:, :-1]).double()
    want = torch.log_softmax(logits, -1).sort(dim=-1, descending=True, stable=True)
    assert torch.equal(r.top_tokens, want.indices[..., :4])
    assert (r.top_logprobs - want.values[..., :4]).abs().max() < 1e-4
    assert (r.entropy.double() - torch.distributions.Categorical(logits=logits).entropy()).abs().max() < 1e-4


def test_training_steps_run():
    model = _stack(BF, seed=8)
    opt = torch.optim.AdamW(model.parameters(), lr=1e-3)
    tokens = torch.randint(0, 300, (2, 100), device="cuda")
    for _ in range(3):
        opt.zero_grad(set_to_none=True)
        r = model.logprobs(tokens)
        (-r.logprob.mean() - 0.01 * r.entropy.mean()).backward()
        for name, p in model.named_parameters():
            assert p.grad is not None and torch.isfinite(p.grad).all(), name
        opt.step()


def test_new_token_over_a_cache_is_the_whole_sequence():
    """Norm, rotation, attention and the next token's distribution, one token at a time
    over a cache, against the same over the whole sequence."""
    b, n, h, hk, d, vocab = 3, 40, 8, 2, 64, 501
    g = torch.Generator(device="cuda").manual_seed(3)

    def normal(*s):
        return torch.randn(s, generator=g, device="cuda").to(BF)

    qkv, head = normal(b, n, h + 2 * hk, d), normal(h * d, vocab) * (h * d) ** -0.5
    wq, wk = (1 + 0.1 * normal(d) for _ in range(2))
    freqs = rotary_freqs(d // 2)
    q, k, v = qkv.split([h, hk, hk], dim=2)
    qr, kr = norm_rotate([q, k], weights=[wq, wk], freqs=freqs)
    whole = dot_attention(qr, kr, v, softcap=20.0)
    k_cache = torch.full((b, 64, hk, d), float("nan"), dtype=BF, device="cuda")
    v_cache = k_cache.clone()
    first = torch.tensor([0, 5, 11], device="cuda")  # the sequences begin at different times
    rows = torch.arange(b, device="cuda")
    for t in range(n):
        at = first + t
        live = torch.full((b,), t, device="cuda")
        qt, kt = norm_rotate([q[:, t:t + 1], k[:, t:t + 1]], weights=[wq, wk], freqs=freqs, positions=live[:, None])
        k_cache[rows, live], v_cache[rows, live] = kt[:, 0], v[:, t]
        one = dot_attention(qt, k_cache, v_cache, softcap=20.0, k_lens=(live + 1).to(torch.int32))
        assert torch.equal(kt, kr[:, t:t + 1]) and torch.equal(qt, qr[:, t:t + 1])
        # the split of the key axis is another: P of both forms rounded to bf16 at another maximum
        assert (one.double() - whole[:, t:t + 1].double()).abs().max() <= 3 * 2.0 ** -8 * v[:, :t + 1].abs().max()
        r = token_logprobs((one.reshape(b, -1) @ head), at % vocab, top=5)
        assert torch.isfinite(r.logprob).all() and (r.top_logprobs[:, 0] >= r.logprob).all()


def _one_step(qkv, head, ws, targets, ids, freqs):
    b, n = qkv.shape[:2]
    q, k, v = qkv.split([4, 2, 2], dim=2)
    q, k = norm_rotate([q, k], weights=ws, freqs=freqs, positions=torch.arange(n, device="cuda"))
    o = dot_attention(q, k, v, documents=ids, softcap=10.0)
    r = token_logprobs(o.view(b * n, -1) @ head.t(), targets.view(-1))
    return torch.autograd.grad([r.logprob, r.entropy], [qkv, head, *ws], [torch.ones_like(r.logprob), 0.1 * torch.ones_like(r.entropy)])


def _step_inputs(seed=3, n=75):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(2, n, 8, 64, generator=g, device="cuda").to(BF).requires_grad_(True)
    head = (torch.randn(200, 256, generator=g, device="cuda") / 16).to(BF).requires_grad_(True)
    ws = [torch.ones(64, device="cuda", requires_grad=True) for _ in range(2)]
    targets = torch.randint(0, 200, (2, n), device="cuda", generator=g)
    ids = (torch.arange(n, device="cuda") // 30).to(torch.int32).expand(2, n).contiguous()
    return qkv, head, ws, targets, ids, rotary_freqs(32)


def test_saved_tensors_elsewhere():
    """Hooks that keep the saved tensors on the host (and bring them back to other places,
    with other strides): the same gradients."""
    inputs = _step_inputs()
    want = _one_step(*inputs)
    with torch.autograd.graph.save_on_cpu():
        got = _one_step(*inputs)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_backward_twice_and_checkpointed():
    """The same gradients from a second backward of a kept graph, and from a forward run
    again in the backward."""
    qkv, head, ws, targets, ids, freqs = _step_inputs()

    def loss(qkv, head, *ws):
        q, k, v = qkv.split([4, 2, 2], dim=2)
        q, k = norm_rotate([q, k], weights=list(ws), freqs=freqs)
        o = dot_attention(q, k, v, documents=ids, window=40)
        return token_logprobs(o.view(-1, head.shape[1]) @ head.t(), targets.view(-1)).logprob.sum()

    leaves = [qkv, head, *ws]
    whole = loss(*leaves)
    first = torch.autograd.grad(whole, leaves, retain_graph=True)
    second = torch.autograd.grad(whole, leaves)
    again = torch.autograd.grad(torch.utils.checkpoint.checkpoint(loss, *leaves, use_reentrant=False), leaves)
    for a, b, c in zip(first, second, again):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_changes_in_place_are_noticed():
    qkv, _, ws, _, ids, freqs = _step_inputs()
    q, k, v = (t.contiguous() for t in qkv.split([4, 2, 2], dim=2))
    o = dot_attention(q, k, v, documents=ids)
    ids += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()


def test_the_same_tensor_twice():
    """One tensor as queries and keys with one weight, one as keys and values: gradients are
    the sums of those of copies."""
    qkv, _, ws, _, ids, freqs = _step_inputs()
    x, w = qkv.detach()[:, :, :4].contiguous(), ws[0].detach() + 0.5
    dout = torch.randn(x.shape, device="cuda").to(BF)
    xs, wt = [x.clone().requires_grad_(True) for _ in range(3)], [w.clone().requires_grad_(True) for _ in range(2)]
    q, k = norm_rotate(xs[:2], weights=wt, freqs=freqs)
    apart = torch.autograd.grad(dot_attention(q, k, xs[2], documents=ids), xs + wt, dout)
    one, weight = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
    q, k = norm_rotate([one, one], weights=[weight, weight], freqs=freqs)
    dx, dw = torch.autograd.grad(dot_attention(q, k, one, documents=ids), [one, weight], dout)
    total = sum(g.double() for g in apart[:3])
    # (two roundings of partial sums to bf16)
    assert ((dx.double() - total).abs() <= 2 * ref.HALF[BF] * sum(g.double().abs() for g in apart[:3])).all()
    assert torch.equal(dw, apart[3] + apart[4])


def test_another_stream():
    """Calls on a stream of their own, the inputs made on it."""
    want = _one_step(*_step_inputs())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _one_step(*_step_inputs())
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_two_graphs_replayed_in_turn():
    """Two captured steps of other sizes, whose workspaces are their own."""
    cases = [_step_inputs(5, 75), _step_inputs(6, 300)]
    graphs, held = [], []
    for c in cases:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            _one_step(*c)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append(_one_step(*c))
        graphs.append(g)
    want = [_one_step(*c) for c in cases]
    for i in (0, 1, 1, 0, 1):
        for t in held[i]:
            t.zero_()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[i], held[i])), i


def test_captured_training_step():
    """Norm and rotation, attention, a head and the log probabilities with all gradients in
    one graph, replayed on new inputs with eager work between."""
    b, n, h, hk, d, vocab = 2, 130, 4, 2, 64, 1000
    g = torch.Generator(device="cuda").manual_seed(7)

    def normal(*s):
        return torch.randn(s, generator=g, device="cuda")

    qkv = normal(b, n, h + 2 * hk, d).to(BF).requires_grad_(True)
    head = (normal(vocab, h * d) * (h * d) ** -0.5).to(BF).requires_grad_(True)
    ws = [(1 + 0.1 * normal(d)).requires_grad_(True) for _ in range(2)]
    targets = torch.randint(0, vocab, (b, n), device="cuda", generator=g)
    ids = (torch.arange(n, device="cuda") // 50).to(torch.int32).expand(b, n).contiguous()
    weight = torch.full((b, n), 1.0 / (b * n), device="cuda")
    freqs = rotary_freqs(d // 2)

    def step():
        q, k, v = qkv.split([h, hk, hk], dim=2)
        q, k = norm_rotate([q, k], weights=ws, freqs=freqs)
        o = dot_attention(q, k, v, documents=ids, softcap=10.0)
        r = token_logprobs(o.view(b * n, h * d) @ head.t(), targets.view(-1))
        out = [r.logprob, r.entropy]
        return [*(t.detach() for t in out), *torch.autograd.grad(out, [qkv, head, *ws], [weight.view(-1), 0.1 * weight.view(-1)])]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        with torch.no_grad():
            qkv.copy_(normal(*qkv.shape))
            targets.copy_(torch.randint(0, vocab, (b, n), device="cuda", generator=g))
        eager = step()
        graph.replay()
        torch.cuda.synchronize()
        for j, (x, y) in enumerate(zip(eager, held)):
            assert torch.equal(x, y), (i, j)

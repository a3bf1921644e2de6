"""Which arithmetic the layers of a stack are given (these run without a GPU)."""

import pytest
import torch

from paper_2507_02754_amd import DotProductAttention, InterleavedStack

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("stack, options, want", [
    (F32, dict(qk_norm=True), F32), (F32, dict(window=8, attn_dtype=None), F32), (BF, dict(qk_norm=True), BF),
    (F32, dict(rope_base=10000.0, attn_dtype=BF), BF), (BF, dict(attn_dtype=F32), F32),
    (F32, None, None), (F32, {}, None), (BF, dict(qk_norm=False), None), (F32, dict(kv_heads=2), None)], ids=str)
def test_a_stack_hands_its_type_to_its_dot_layers(stack, options, want):
    """Where options select the kernels and name no type of their own; without any the layers
    stay torch's float32 attention."""
    model = InterleavedStack(vocab=10, d_model=32, n_layers=4, n_heads=2, head_dim=16, w1=8, w2=4, attn_dtype=stack, dot_options=options)
    assert model.simplicial_layers() == [3] and model.layers[3].attn.attn_dtype == stack
    for block in model.layers[:3]:
        assert isinstance(block.attn, DotProductAttention) and block.attn.attn_dtype == want

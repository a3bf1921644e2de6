"""How the work of a dot-product attention is split, seen by the workspace it asks for (these
run without a GPU)."""

import os

import pytest
import torch

from paper_2507_02754_amd import binding, simplicial_dot_attn_bwd_workspace_size

BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2507_02754_amd import build
        build.build()


def _parts(B, N, H, Hkv, D, window=0, documents=False, causal=True):
    """Workgroups that share a block of keys: the backward's float32 partial sums, over those of one."""
    size = simplicial_dot_attn_bwd_workspace_size(B, N, N, H, Hkv, D, causal, window, documents, BF)
    rows = 512 * B * Hkv * ((H // Hkv * N + 31) // 32) + (8 * B * ((N + 31) // 32) if documents else 0)
    return round((size - rows) / (8 * B * N * Hkv * D))


def test_documents_share_key_blocks_among_more_only_where_rows_are_many():
    for B, N, H, Hkv in ((1, 4096, 8, 8), (4, 2048, 16, 4), (2, 4096, 16, 4)):
        assert _parts(B, N, H, Hkv, 128) == _parts(B, N, H, Hkv, 128, documents=True) == 4
    assert _parts(1, 16384, 8, 2, 128) == 4 and _parts(1, 16384, 8, 2, 128, documents=True) == 8


def test_a_window_leaves_a_block_of_keys_few_rows():
    """None to share among workgroups, whatever the length of the sequence."""
    assert _parts(1, 4096, 8, 8, 128) == 4 and _parts(1, 4096, 8, 8, 128, window=512) == 0
    assert _parts(1, 16384, 8, 2, 128, window=300) == 0 and _parts(1, 16384, 8, 2, 128, window=2000) == 4
    assert _parts(1, 16384, 8, 2, 128, window=300, causal=False) == 4
    assert _parts(1, 12000, 8, 2, 64) > 0 == _parts(1, 12000, 8, 2, 64, window=900)
    # a window that hides nothing is none
    for N in (4096, 16384):
        assert _parts(1, N, 8, 2, 128, window=N) == _parts(1, N, 8, 2, 128)

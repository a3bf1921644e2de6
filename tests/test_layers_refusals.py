"""Calls of the layers' operators that are refused, and arguments that are read, before any
HIP call (these run without a GPU)."""

import os

import pytest
import torch

from paper_2507_02754_amd import binding, layers_binding

A = 0x10000  # never read: every library call below is refused

only_without_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake pointers: only where no GPU is visible")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2507_02754_amd import build
        build.build()
    return layers_binding._library()


@only_without_gpu
def test_logprobs_dtype_with_low_parts(lib):
    """The flag changes neither the workspace nor what is refused."""
    lo = layers_binding.LOGPROBS_LSE_LO
    size = lib.simplicial_logprobs_fwd_workspace_size
    for R, V in ((1, 100), (2, 100001), (1 << 26, 100)):
        for dtype in (0, 1):
            assert size(R, V, 1, dtype) == size(R, V, 1, dtype | lo)
    for dtype in (3 | lo, 2 * lo, -1, lo - (1 << 31)):
        assert size(2, 100001, 1, dtype) == 0
        assert lib.simplicial_logprobs_fwd(A, A, A, A, A, 0, 0, A, 1 << 40, 2, 100001, 100001, 0, dtype, None) == 2
        assert lib.simplicial_logprobs_bwd(A, A, A, A, A, 0, 0, A, 4, 100, 100, dtype, None) == 2
    for lse in (0, A + 2):
        assert lib.simplicial_logprobs_fwd(A, A, A, A, lse, 0, 0, A, 1 << 40, 4, 100, 100, 0, 1 | lo, None) == 1
        assert lib.simplicial_logprobs_bwd(A, A, lse, A, A, 0, 0, A, 4, 100, 100, 1 | lo, None) == 1

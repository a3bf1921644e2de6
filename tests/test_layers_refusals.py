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


@only_without_gpu
@pytest.mark.parametrize("backward", [False, True])
def test_scales_and_caps_past_float32(lib, backward):
    """Quotients and products that overflow or lose digits are refused (an infinity times a
    score of 0 would be NaN); the workspace is asked for where they do not."""
    def rc(scale, cap):
        B, Nq, Nk, H, Hkv, D = 1, 1, 4096, 8, 2, 128
        f = lib.simplicial_dot_attn_bwd if backward else lib.simplicial_dot_attn_fwd
        return f(*[A] * (10 if backward else 6), A, 0, B, Nq, Nk, H, Hkv, D, *(1024, 1024, 128), *(1 << 20, 256, 128) * 2, scale, cap,
                 1, 0, 0, 0, 0, 0, 1, None)
    for scale, cap in ((0.1, 0.0), (0.0, 1.0), (-3.0, 50.0), (0.1, 1e-30), (0.1, 1e30), (2.0, 2.0 ** 125), (1e38, 0.0), (0.0, 1e30)):
        assert rc(scale, cap) == 3, (scale, cap)
    for scale, cap in ((0.1, 3e38), (0.1, 1e-39), (0.0, 1e-39), (1e-3, 2.0 ** 120), (1e30, 1e-20), (3e38, 0.0), (-3e38, 0.0), (1e20, 1e-25)):
        assert rc(scale, cap) == 1, (scale, cap)


class FakeTensor:
    """What the checks before the library look at."""
    shape, dtype, device, is_cuda = torch.Size((1, 4, 2, 64)), torch.bfloat16, torch.device("cuda", 0), True

    def dim(self):
        return 4

    def numel(self):
        return 512

    def stride(self, *i):
        return (512, 128, 64, 1)[i[0]] if i else (512, 128, 64, 1)

    def data_ptr(self):
        return A


def test_a_cap_that_float32_rounds_to_none():
    x = FakeTensor()
    for cap in (1e-46, 1e-39):
        with pytest.raises(ValueError, match="softcap"):
            layers_binding._DotCall(x, x, x, None, True, 0, cap, None, None, None, None)
    layers_binding._DotCall(x, x, x, None, True, 0, 1e-30, None, None, None, None)


def test_workspace_sizes_of_windows_past_32_bits(lib):
    """As of a window that hides nothing; negative ones as an invalid call's."""
    for size in (layers_binding.simplicial_dot_attn_fwd_workspace_size, layers_binding.simplicial_dot_attn_bwd_workspace_size):
        def of(window):
            return size(2, 1, 5000, 8, 2, 128, True, window, True, torch.bfloat16)
        assert of(5000) == of(1 << 31) == of((1 << 32) + 5) == of(1 << 70) == of(0) > 0
        assert of(-1) == of(-(1 << 32)) == of(5 - (1 << 32)) == 0


def test_positions_past_64_bits():
    x = FakeTensor()
    for start in (1 << 63, (1 << 63) - 3, (1 << 64) + 5, -(1 << 63) - 1):
        with pytest.raises(ValueError, match="start"):
            layers_binding._RotateCall([x], None, 1e-6, layers_binding.rotary_angles(None), "half", None, start)
    for start in (0, (1 << 63) - 4, -(1 << 63)):
        layers_binding._RotateCall([x], None, 1e-6, layers_binding.rotary_angles(None), "half", None, start)

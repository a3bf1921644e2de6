"""The entry points of include/simplicial_layers.h: exported, and invalid arguments are
refused on the host before any HIP call (these run without a GPU)."""

import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2507_02754_amd import binding, dot_attention, layers_binding, norm_rotate, rotary_freqs, token_logprobs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "simplicial_layers.h")
A = 0x10000       # never read: every call below is refused
ODD = 0x10008

only_without_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake pointers: only where no GPU is visible")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2507_02754_amd import build
        build.build()
    return layers_binding._library()


def test_library_exports_every_declared_symbol(lib):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(simplicial_\w+)\s*\(", src)))
    assert len(declared) == 10
    out = subprocess.run(["nm", "-D", "--defined-only", binding.LIB_PATH], capture_output=True, text=True, check=True).stdout
    exported = set(re.findall(r"\bT (simplicial_\w+)", out))
    for name in declared:
        assert name in exported and hasattr(lib, name), name


def _rotate(lib, backward=False, count=2, x=None, strides=None, weight=None, heads=(4, 2), pos=0, pos_stride=0, B=2, N=8,
            D=64, norm=1, eps=1e-6, layout=0, freqs=rotary_freqs(32), nfreq=None, dtype=1, wdtype=0, y=None, dw=None, ws=A,
            ws_bytes=1 << 30):
    n = max(len(heads), 1)
    pointers = lambda v: (ctypes.c_void_p * n)(*v)  # noqa: E731
    x, y = x or [A] * n, y or [A] * n
    strides = strides or [N * 64 * 9, 64 * 9, 64] * n
    head = (count, pointers(x), (ctypes.c_int64 * (3 * n))(*strides), None if weight is None else pointers(weight))
    f = (ctypes.c_double * max(len(freqs), 1))(*freqs)
    tail = (B, N, D, norm, eps, layout, f, len(freqs) if nfreq is None else nfreq, dtype, wdtype, None)
    h = (ctypes.c_int32 * n)(*heads)
    if not backward:
        return lib.simplicial_norm_rotate_fwd(*head, pointers(y), h, pos, pos_stride, 0, *tail)
    return lib.simplicial_norm_rotate_bwd(*head, pointers(y), pointers(y), None if dw is None else pointers(dw), h, pos,
                                          pos_stride, 0, ws, ws_bytes, *tail)


@only_without_gpu
@pytest.mark.parametrize("backward", [False, True])
def test_norm_rotate_refusals(lib, backward):
    def rc(**kw):
        return _rotate(lib, backward, **kw)
    for bad in (dict(count=0), dict(count=4), dict(x=[A, 0]), dict(x=[ODD, A]), dict(y=[A, 0]), dict(heads=(4, 0)),
                dict(B=0), dict(N=-1), dict(D=0), dict(B=1 << 20, N=1 << 20), dict(strides=[4608, 576, 64, 4608, 576, 12]),
                dict(strides=[4608, -576, 64] * 2), dict(weight=[A, A + 2]), dict(weight=[A, A], norm=0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(layout=3), dict(layout=-1), dict(nfreq=33), dict(nfreq=-1), dict(layout=2, nfreq=22),
                dict(freqs=[float("inf")] * 8), dict(pos=A + 4), dict(pos=A, pos_stride=3), dict(pos_stride=-1)):
        assert rc(**bad) == 1, bad
    for bad in (dict(D=48), dict(D=256), dict(dtype=2), dict(wdtype=5), dict(nfreq=12)):
        assert rc(**bad) == 2, bad
    if backward:
        assert rc(weight=[A, A], dw=[A, A], ws_bytes=16) == 3
        assert rc(weight=[A, A], dw=[A, A], ws=0) == 1
        assert rc(dw=[A, 0], norm=0) == 1
    assert lib.simplicial_norm_rotate_bwd_workspace_size(4, 1, 1, 64) == 0
    assert lib.simplicial_norm_rotate_bwd_workspace_size(1, 1, 1, 63) == 0


def _dot(lib, backward=False, ptrs=None, ws=A, ws_bytes=1 << 40, B=2, Nq=8, Nk=16, H=4, Hkv=2, D=64, q=None, k=None, scale=0.1,
         cap=0.0, causal=1, window=0, opts=(0, 0, 0, 0), dtype=1):
    n = 10 if backward else 6
    q, k = q or (Nq * H * D, H * D, D), k or (Nk * Hkv * D, Hkv * D, D)
    tail = (B, Nq, Nk, H, Hkv, D, *q, *k, *k, scale, cap, causal, window, *opts, dtype, None)
    f = lib.simplicial_dot_attn_bwd if backward else lib.simplicial_dot_attn_fwd
    return f(*(ptrs or [A] * n), ws, ws_bytes, *tail)


@only_without_gpu
@pytest.mark.parametrize("backward", [False, True])
def test_dot_attention_refusals(lib, backward):
    def rc(**kw):
        return _dot(lib, backward, **kw)
    n = 10 if backward else 6
    for i in range(n):
        for bad in (0, ODD):
            if i != 4 or bad:  # (out_lo may be null)
                assert rc(ptrs=[A] * i + [bad] + [A] * (n - i - 1)) == 1, i
    assert rc(dtype=0) == 1  # out_lo is of bf16 results
    for bad in (dict(B=0), dict(Nq=0), dict(Nk=0), dict(H=0), dict(Hkv=0), dict(D=-64), dict(Nq=17), dict(H=4, Hkv=3),
                dict(H=2, Hkv=4), dict(window=-1), dict(scale=float("nan")), dict(cap=-1.0), dict(cap=float("inf")),
                dict(q=(2048, 256, 12)), dict(k=(-8, 128, 64)), dict(opts=(A + 2, 0, 0, 0)), dict(opts=(0, A + 1, 0, 0)),
                dict(Nk=(1 << 30) + 1), dict(B=1 << 22, Nk=1 << 10), dict(opts=(0, A, 0, 0), ws=0)):
        assert rc(**bad) == 1, bad
    for bad in (dict(D=48), dict(D=256), dict(dtype=2), dict(q=(1 << 40, 1 << 30, 64)), dict(k=(1 << 40, 1 << 26, 64))):
        assert rc(**bad) == 2, bad
    assert rc(opts=(0, A, 0, 0), ws_bytes=8) == 3
    for size in (lib.simplicial_dot_attn_fwd_workspace_size, lib.simplicial_dot_attn_bwd_workspace_size):
        assert size(2, 17, 16, 4, 2, 64, 1, 0, 1, 1) == 0 and size(2, 8, 16, 4, 2, 48, 1, 0, 1, 1) == 0
        assert size(2, 8, 16, 4, 2, 64, 1, 0, 1, 1) > 0
    # few queries over a long cache: parts of the key axis, no less with more keys
    assert 0 < lib.simplicial_dot_attn_fwd_workspace_size(1, 1, 4096, 8, 2, 128, 1, 0, 0, 1)


@only_without_gpu
def test_logprobs_refusals(lib):
    def fwd(x=A, t=A, lp=A, h=A, lse=A, tl=A, ti=A, ws=A, ws_bytes=1 << 40, R=4, V=100, stride=100, top=2, dtype=1):
        return lib.simplicial_logprobs_fwd(x, t, lp, h, lse, tl, ti, ws, ws_bytes, R, V, stride, top, dtype, None)

    def bwd(x=A, t=A, lse=A, h=A, g=A, dx=A, R=4, V=100, stride=100, dtype=1):
        return lib.simplicial_logprobs_bwd(x, t, lse, h, g, 0, 0, dx, R, V, stride, dtype, None)
    for f in (fwd, bwd):
        for bad in (dict(x=0), dict(x=A + 1), dict(t=0), dict(t=A + 4), dict(lse=0), dict(h=A + 2), dict(R=0), dict(V=0),
                    dict(stride=99), dict(R=1 << 26), dict(R=1 << 20, V=1 << 20, stride=1 << 20)):
            assert f(**bad) == 1, (f.__name__, bad)
        assert f(dtype=3) == 2 and f(V=4000001, stride=4000001) == 2
    for bad in (dict(top=-1), dict(top=33), dict(V=3, top=4), dict(tl=0), dict(ti=0), dict(ti=A + 4), dict(lp=0)):
        assert fwd(**bad) == 1, bad
    assert fwd(V=100001, stride=100001, ws=0) == 1 and fwd(V=100001, stride=100001, ws_bytes=0) == 3
    assert bwd(dx=0) == 1 and bwd(dx=ODD) == 1 and bwd(g=A + 2) == 1


@only_without_gpu
def test_sizes_past_a_launch(lib):
    """Calls whose launches would hold 2^32 threads or more, or whose offsets pass their type, just
    past the largest that do not."""
    large = 64 * 9
    for kw in (dict(heads=(1, 1), D=128, B=1, N=1 << 28, strides=[0, large, 64] * 2),
               dict(heads=(1 << 24, 2), D=128, B=1, N=1, strides=[0, large, 64] * 2)):
        assert _rotate(lib, freqs=(), **kw) == 1, kw
    assert _dot(lib, B=1, Nq=1, Nk=1 << 28, H=1, Hkv=1, D=16, k=(0, 16, 16)) == 1
    fits = lambda R, V, dtype: lib.simplicial_logprobs_fwd(A, A, A, A, A, A, A, 0, 0, R, V, V, 1, dtype, None) != 1  # noqa: E731
    size = lib.simplicial_logprobs_fwd_workspace_size
    for R, V, dtype in ((1 << 24, 1024, 0), (1 << 25, 1024, 1), ((1 << 26) - 1, 2000, 1)):
        assert not fits(R, V, dtype) and size(R, V, 1, dtype) == 0
    # 16 slices and more of a row: the workspace is asked for
    assert size(1 << 18, 1 << 17, 1, 1) > 0 and size(1 << 16, 1 << 17, 1, 0) > 0


def test_python_refusals():
    """What the binding refuses before the library is called (CPU tensors)."""
    x = torch.zeros(1, 4, 2, 64)
    with pytest.raises(ValueError, match="GPU"):
        norm_rotate([x])
    with pytest.raises(ValueError, match="1 to 3"):
        norm_rotate([])
    with pytest.raises(ValueError, match="weight for every"):
        norm_rotate([x, x], weights=[torch.ones(64), None])
    with pytest.raises(ValueError, match="GPU"):
        dot_attention(x, x, x)
    with pytest.raises(ValueError, match=r"\[B, N, heads, D\]"):
        dot_attention(x[0], x, x)
    with pytest.raises(ValueError, match="slopes"):
        dot_attention(x, x, x, slopes=torch.ones(2, requires_grad=True))
    with pytest.raises(ValueError, match="targets"):
        token_logprobs(torch.zeros(3, 5), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="GPU"):
        token_logprobs(torch.zeros(3, 5), torch.zeros(3, dtype=torch.int64))
    assert rotary_freqs(4, 10000.0) == pytest.approx((1.0, 0.1, 0.01, 0.001))

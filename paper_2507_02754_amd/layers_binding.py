"""ctypes binding of the entry points of include/simplicial_layers.h (argument
marshalling only), in the manner of `binding`: tensors are checked for device,
dtype, layout and shape, outputs and workspaces are allocated with torch, and the
raw pointers plus torch's current HIP stream on the tensors' device go to the
library. There is no fallback implementation.
"""

import ctypes

import torch

from .binding import _DTYPES, SimplicialAttnError, _stream, load_library

__all__ = [
    "rotary_freqs",
    "simplicial_norm_rotate_fwd",
    "simplicial_norm_rotate_bwd",
    "simplicial_dot_attn_fwd",
    "simplicial_dot_attn_fwd_workspace_size",
    "simplicial_dot_attn_bwd",
    "simplicial_dot_attn_bwd_workspace_size",
    "simplicial_logprobs_fwd",
    "simplicial_logprobs_bwd",
]

ROTATE_LAYOUTS = {"half": 0, "pairs": 1, "axis": 2}
ROTATE_MAX = 3
LOGPROBS_MAX_TOP = 32
LOGPROBS_LSE_LO = 0x100  # added to the dtype: lse is [2, R]

_lib = None


def _library():
    """The library with this module's entry points declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = load_library()
    vp, i64, i32, f32, size = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    lib.simplicial_norm_rotate_fwd.argtypes = [i32] + [vp] * 5 + [vp, i64, i64, i64, i64, i64, i32, f32, i32, vp, i32,
                                                                  i32, i32, vp]
    lib.simplicial_norm_rotate_bwd.argtypes = [i32] + [vp] * 7 + [vp, i64, i64, vp, size, i64, i64, i64, i32, f32, i32,
                                                                  vp, i32, i32, i32, vp]
    lib.simplicial_norm_rotate_bwd_workspace_size.argtypes = [i32, i64, i64, i64]
    dot = [i64] * 15 + [f32, f32, i32, i32] + [vp] * 4 + [i32, vp]
    lib.simplicial_dot_attn_fwd.argtypes = [vp] * 7 + [size] + dot
    lib.simplicial_dot_attn_bwd.argtypes = [vp] * 11 + [size] + dot
    lib.simplicial_logprobs_fwd.argtypes = [vp] * 8 + [size, i64, i64, i64, i32, i32, vp]
    lib.simplicial_logprobs_bwd.argtypes = [vp] * 8 + [i64, i64, i64, i32, vp]
    for name in ("norm_rotate_fwd", "norm_rotate_bwd", "dot_attn_fwd", "dot_attn_bwd", "logprobs_fwd", "logprobs_bwd"):
        getattr(lib, "simplicial_" + name).restype = ctypes.c_int
    for name in ("dot_attn_fwd", "dot_attn_bwd"):
        f = getattr(lib, f"simplicial_{name}_workspace_size")
        f.argtypes = [i64] * 6 + [i32] * 4
        f.restype = size
    lib.simplicial_logprobs_fwd_workspace_size.argtypes = [i64, i64, i32, i32]
    lib.simplicial_logprobs_fwd_workspace_size.restype = size
    lib.simplicial_norm_rotate_bwd_workspace_size.restype = size
    _lib = lib
    return lib


def _call(entry, device, *args):
    """The entry point on the device's current stream, with that device current."""
    f = getattr(_lib or _library(), entry)
    if device.index == torch.cuda.current_device():
        rc = f(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            rc = f(*args, _stream(device))
    if rc != 0:
        raise SimplicialAttnError(rc, entry)


def _workspace(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check_view(t, name, like=None):
    """A [B, N, heads, D] GPU tensor of a supported dtype with unit innermost stride."""
    if t.dim() != 4:
        raise ValueError(f"{name} must be [B, N, heads, D], got shape {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name}: unsupported dtype {t.dtype}; expected float32 or bfloat16")
    if t.numel() == 0:
        raise ValueError(f"{name} is empty: shape {tuple(t.shape)}")
    if t.stride(3) != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name} has {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")


def _strides(t):
    """Batch, position and head strides; 0 along a dimension of one element, whose stride says nothing."""
    s, n = t.stride(), t.shape
    return (s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0, s[2] if n[2] > 1 else 0)


def _check_like(t, shape, dtype, device, name):
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")


# ---- norm and rotation ----


def rotary_freqs(count, base=10000.0):
    """`count` angles per position, base^(-i / count): the geometric series of a
    rotation with `count` pairs."""
    return tuple(float(base) ** (-i / count) for i in range(count))


_ANGLES = {}  # the last ones by value: (array, their number)


def rotary_angles(freqs, check=None):
    """(ctypes array, its length) of angles given as numbers, a tensor of them, or None. What is
    kept are Python numbers (a tensor's elements would never be found again). check(*t) is called
    with the tensors among them."""
    if freqs is None:
        freqs = ()
    elif isinstance(freqs, torch.Tensor):
        if check is not None:
            check(freqs)
        freqs = freqs.tolist()
    freqs = tuple(freqs)
    found = _ANGLES.get(freqs)
    if found is None:
        if check is not None:
            check(*[f for f in freqs if isinstance(f, torch.Tensor)])
        numbers = tuple(map(float, freqs))
        found = _ANGLES.get(numbers)
    if found is None:
        if len(_ANGLES) >= 64:
            _ANGLES.pop(next(iter(_ANGLES)), None)
        found = _ANGLES[numbers] = ((ctypes.c_double * max(len(numbers), 1))(*numbers), len(numbers))
    return found


class _RotateCall:
    """Checked arguments of a norm and rotation, in the form the library takes: the same
    for the forward and its backward."""

    __slots__ = ("n", "shapes", "dtype", "device", "strides", "xs", "weights", "heads", "pos", "tail", "kept")

    def __init__(self, xs, weights, eps, angles, layout, positions, start):  # angles: of rotary_angles
        n = len(xs)
        if not 1 <= n <= ROTATE_MAX:
            raise ValueError(f"1 to {ROTATE_MAX} tensors, got {n}")
        x0 = xs[0]
        for t, x in enumerate(xs):
            _check_view(x, "x", x0)
        B, N, _, D = x0.shape
        shapes = [x.shape for x in xs]
        for t, s in enumerate(shapes):
            if s[0] != B or s[1] != N or s[3] != D:
                raise ValueError(f"x[{t}] has shape {tuple(s)}, expected [B, N, heads, D] of {tuple(x0.shape)}")
        code = ROTATE_LAYOUTS.get(layout)
        if code is None:
            raise ValueError(f"layout {layout!r}; expected one of {', '.join(ROTATE_LAYOUTS)}")
        device = x0.device
        wdtype = torch.float32
        if weights is not None:
            if len(weights) != n:
                raise ValueError(f"{len(weights)} weights for {n} tensors")
            given = [w for w in weights if w is not None]
            if given:
                wdtype = given[0].dtype
                if eps is None:
                    raise ValueError("weights need a norm (eps is None)")
                if wdtype not in _DTYPES:
                    raise ValueError(f"unsupported weight dtype {wdtype}; expected float32 or bfloat16")
            for w in given:
                _check_like(w, (D,), wdtype, device, "a weight")
        pos, pos_stride = None, 0
        if positions is not None:
            if positions.dtype != torch.int64 or positions.device != device or positions.shape not in ((N,), (B, N)):
                raise ValueError(f"positions must be int64 of shape [{N}] or [{B}, {N}] on {device}, got "
                                 f"{positions.dtype} {tuple(positions.shape)} on {positions.device}")
            if N > 1 and positions.stride(-1) != 1:
                raise ValueError("positions must be contiguous in their last dimension")
            if positions.dim() == 2 and B > 1:
                pos_stride = positions.stride(0)
            pos = positions.data_ptr()
        self.n, self.shapes, self.dtype, self.device = n, shapes, x0.dtype, device
        self.heads = (ctypes.c_int32 * n)(*[s[2] for s in shapes])
        self.strides = (ctypes.c_int64 * (3 * n))(*[s for x in xs for s in _strides(x)])
        self.xs = _pointers(xs)
        self.weights = None if weights is None else _pointers(weights)
        if not -(1 << 63) <= int(start) <= (1 << 63) - N:
            raise ValueError(f"start {start}: positions are 64-bit numbers")
        self.pos = (pos, pos_stride, int(start))
        self.tail = (B, N, D, eps is not None, float(eps or 0.0), code, *angles, _DTYPES[x0.dtype],
                     _DTYPES[wdtype])
        self.kept = (xs, weights, positions)  # what the pointers point to

    def places(self):
        """Where the tensors lie: the arguments hold for other tensors with the same ones."""
        xs, weights, positions = self.kept
        return ([(x.data_ptr(), x.stride()) for x in xs], weights and [_ptr(w) for w in weights], _ptr(positions))

    def forward(self, out=None):
        if out is None:
            out = [torch.empty(s, dtype=self.dtype, device=self.device) for s in self.shapes]
        else:
            for s, y in zip(self.shapes, out, strict=True):
                _check_like(y, s, self.dtype, self.device, "an output")
        _call("simplicial_norm_rotate_fwd", self.device, self.n, self.xs, self.strides, self.weights, _pointers(out),
              self.heads, *self.pos, *self.tail)
        return list(out)

    def backward(self, dys, weight_grads=True, grads=None):
        n, device = self.n, self.device
        if len(dys) != n:
            raise ValueError(f"{len(dys)} gradients for {n} tensors")
        for s, dy in zip(self.shapes, dys):
            _check_like(dy, s, self.dtype, device, "an output's gradient")
        if grads is None:
            grads = [torch.empty(s, dtype=self.dtype, device=device) for s in self.shapes]
        else:
            for s, dx in zip(self.shapes, grads, strict=True):
                _check_like(dx, s, self.dtype, device, "an input's gradient")
        dws, dw, workspace, nbytes = [None] * n, None, None, 0
        if weight_grads and self.weights is not None:
            dws = [None if t is None else torch.empty_like(t) for t in self.kept[1]]
            dw = _pointers(dws)
            B, N, D = self.tail[:3]
            nbytes = (_lib or _library()).simplicial_norm_rotate_bwd_workspace_size(n, B, N, D)
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        _call("simplicial_norm_rotate_bwd", device, n, self.xs, self.strides, self.weights, _pointers(dys), _pointers(grads),
              dw, self.heads, *self.pos, _ptr(workspace), nbytes, *self.tail)
        return list(grads), dws


def _pointers(tensors):
    return _POINTERS[len(tensors)](*[None if t is None else t.data_ptr() for t in tensors])


_POINTERS = {n: ctypes.c_void_p * n for n in range(1, ROTATE_MAX + 1)}


def simplicial_norm_rotate_fwd(xs, weights=None, eps=1e-6, freqs=None, layout="half", positions=None, start=0, out=None):
    """RMS norm of each head and position rotation of one to three tensors (q, k,
    k') in one launch; returns their results as a list of contiguous tensors.

    xs[t] is [B, N, heads_t, D] (a view with 16-byte aligned rows will do), weights[t]
    [D] or None; eps None: no norm. `freqs` (numbers, see `rotary_freqs`) are the angles per
    position of the pairs that `layout` names: "half" (i, n + i), "pairs" (2 i, 2 i + 1)
    or "axis" (3 i, 3 i + 1: the first two of each 3-component chunk of the determinant
    logits); None: no rotation. Positions: int64 [N] or [B, N], or start, start + 1, ..."""
    return _RotateCall(xs, weights, eps, rotary_angles(freqs), layout, positions, start).forward(out)


def simplicial_norm_rotate_bwd(xs, dys, weights=None, eps=1e-6, freqs=None, layout="half", positions=None, start=0,
                               weight_grads=True, grads=None):
    """(dxs, dweights) of simplicial_norm_rotate_fwd: lists, the latter with None where
    there is no weight, or all None with weight_grads False."""
    return _RotateCall(xs, weights, eps, rotary_angles(freqs), layout, positions, start).backward(dys, weight_grads, grads)


# ---- dot-product attention ----


def _window(window, Nk):
    """As a 32-bit number: no distance reaches Nk."""
    return max(min(int(window), Nk), -1)


def simplicial_dot_attn_fwd_workspace_size(B, Nq, Nk, H, Hkv, D, causal, window, has_documents, dtype):
    dt = _DTYPES.get(dtype, dtype)
    return int(_library().simplicial_dot_attn_fwd_workspace_size(B, Nq, Nk, H, Hkv, D, bool(causal), _window(window, Nk),
                                                                 bool(has_documents), int(dt)))


def simplicial_dot_attn_bwd_workspace_size(B, Nq, Nk, H, Hkv, D, causal, window, has_documents, dtype):
    dt = _DTYPES.get(dtype, dtype)
    return int(_library().simplicial_dot_attn_bwd_workspace_size(B, Nq, Nk, H, Hkv, D, bool(causal), _window(window, Nk),
                                                                 bool(has_documents), int(dt)))


class _DotCall:
    """Checked arguments of a dot-product attention, in the form the library takes: the same
    for the forward and its backward."""

    __slots__ = ("q", "k", "v", "plan", "args", "kept")

    def __init__(self, q, k, v, scale, causal, window, softcap, slopes, documents, prefix, k_lens):
        _check_view(q, "q", q)
        _check_view(k, "k", q)
        _check_view(v, "v", q)
        B, Nq, H, D = q.shape
        kshape = k.shape
        Nk, Hkv = kshape[1], kshape[2]
        if kshape != v.shape or kshape[0] != B or kshape[3] != D:
            raise ValueError(f"k and v must be [{B}, Nk, Hkv, {D}], got {tuple(kshape)} and {tuple(v.shape)}")
        if H % Hkv:
            raise ValueError(f"{H} query heads are no multiple of {Hkv} heads of k and v")
        if Nq > Nk:
            raise ValueError(f"{Nq} queries of {Nk} keys: the queries are the last of the keys' positions")
        device = q.device
        if slopes is not None:
            _check_like(slopes, (H,), torch.float32, device, "slopes")
        if documents is not None:
            _check_like(documents, (B, Nk), torch.int32, device, "documents")
        if prefix is not None:
            _check_like(prefix, (B,), torch.int32, device, "prefix")
        if k_lens is not None:
            _check_like(k_lens, (B,), torch.int32, device, "k_lens")
        softcap = float(softcap)
        if 0 < softcap < 2.0 ** -126:  # (0, no cap, to float32)
            raise ValueError(f"softcap {softcap} is below what float32 holds")
        if int(window) < 0:
            raise ValueError(f"window {window} is negative")
        causal, window, dt = bool(causal), _window(window, Nk), _DTYPES[q.dtype]
        self.q, self.k, self.v = q, k, v
        self.plan = (B, Nq, Nk, H, Hkv, D, causal, window, documents is not None, dt)
        self.args = (B, Nq, Nk, H, Hkv, D, *_strides(q), *_strides(k), *_strides(v), D ** -0.5 if scale is None else float(scale),
                     softcap, causal, window, _ptr(slopes), _ptr(documents), _ptr(prefix), _ptr(k_lens), dt)
        self.kept = (slopes, documents, prefix, k_lens)  # what the pointers point to

    def places(self):
        """As _RotateCall's."""
        return ([t.stride() for t in (self.q, self.k, self.v)], [_ptr(t) for t in self.kept])

    def forward(self, out=None, lse=None, out_lo=None):
        q = self.q
        device, (B, Nq, _, H) = q.device, self.plan[:4]
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=device)
        else:
            _check_like(out, q.shape, q.dtype, device, "out")
        if lse is None:
            lse = torch.empty((B, H, Nq), dtype=torch.float32, device=device)
        else:
            _check_like(lse, (B, H, Nq), torch.float32, device, "lse")
        if out_lo is not None:
            _check_like(out_lo, q.shape, torch.bfloat16, device, "out_lo")
        nbytes = (_lib or _library()).simplicial_dot_attn_fwd_workspace_size(*self.plan)
        workspace = _workspace(nbytes, device)
        _call("simplicial_dot_attn_fwd", device, q.data_ptr(), self.k.data_ptr(), self.v.data_ptr(), out.data_ptr(),
              _ptr(out_lo), lse.data_ptr(), _ptr(workspace), nbytes, *self.args)
        return out, lse

    def backward(self, out, dout, lse, out_lo=None, grads=None):
        q = self.q
        device, (B, Nq, _, H) = q.device, self.plan[:4]
        _check_like(out, q.shape, q.dtype, device, "out")
        _check_like(dout, q.shape, q.dtype, device, "dout")
        _check_like(lse, (B, H, Nq), torch.float32, device, "lse")
        if out_lo is not None:
            _check_like(out_lo, q.shape, torch.bfloat16, device, "out_lo")
        if grads is None:
            grads = tuple([torch.empty(t.shape, dtype=t.dtype, device=device) for t in (q, self.k, self.v)])
        else:
            for t, g, name in zip((q, self.k, self.v), grads, ("dq", "dk", "dv"), strict=True):
                _check_like(g, t.shape, t.dtype, device, name)
        nbytes = (_lib or _library()).simplicial_dot_attn_bwd_workspace_size(*self.plan)
        workspace = _workspace(nbytes, device)
        _call("simplicial_dot_attn_bwd", device, q.data_ptr(), self.k.data_ptr(), self.v.data_ptr(), out.data_ptr(),
              _ptr(out_lo), dout.data_ptr(), lse.data_ptr(), *[g.data_ptr() for g in grads], _ptr(workspace), nbytes, *self.args)
        return grads


def simplicial_dot_attn_fwd(q, k, v, scale=None, causal=True, window=0, softcap=0.0, slopes=None, documents=None, prefix=None,
                            k_lens=None, out=None, lse=None, out_lo=None):
    """(O, LSE) of dot-product attention: q [B, Nq, H, D], k and v [B, Nk, Hkv, D] (H a
    multiple of Hkv), the queries the last Nq of the sequence's positions; LSE is
    [B, H, Nq] float32. Views with 16-byte aligned rows will do.

    `scale` defaults to 1/sqrt(D); `softcap` > 0 caps scores by softcap * tanh(s / softcap);
    slopes [H] float32 subtract slope * distance. A query at position p sees keys j <= p
    (causal) with |p - j| < window (window > 0), and those before prefix[b] ([B] int32); with
    `documents` ([B, Nk] int32, negative: padding) of its own document alone. k_lens [B]
    int32: filled lengths of a cache, its last Nq positions the queries. A query that sees
    no key gives O = 0 and LSE = -inf. `out_lo` (bfloat16 as O): takes what rounding O to
    bfloat16 took from it, for the backward."""
    call = _DotCall(q, k, v, scale, causal, window, softcap, slopes, documents, prefix, k_lens)
    return call.forward(out, lse, out_lo)


def simplicial_dot_attn_bwd(q, k, v, out, dout, lse, scale=None, causal=True, window=0, softcap=0.0, slopes=None,
                            documents=None, prefix=None, k_lens=None, grads=None, out_lo=None):
    """(dQ, dK, dV) of simplicial_dot_attn_fwd with the same options; `out`, `lse` and
    (where it was asked for: without it the gradients have the rounding of O in them)
    `out_lo` are its results. The slopes get no gradient."""
    call = _DotCall(q, k, v, scale, causal, window, softcap, slopes, documents, prefix, k_lens)
    return call.backward(out, dout, lse, out_lo, grads)


# ---- log probabilities ----


def _check_logits(logits, targets):
    if logits.dim() != 2 or logits.numel() == 0:
        raise ValueError(f"logits must be [R, V], got shape {tuple(logits.shape)}")
    if not logits.is_cuda:
        raise ValueError("logits must be a GPU tensor")
    if logits.dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {logits.dtype}; expected float32 or bfloat16")
    R, V = logits.shape
    if (V > 1 and logits.stride(1) != 1) or (R > 1 and logits.stride(0) < V):
        raise ValueError("logits must be contiguous in their last dimension, rows apart")
    _check_like(targets, (R,), torch.int64, logits.device, "targets")
    return R, V, logits.stride(0) if R > 1 else V


def simplicial_logprobs_fwd(logits, targets, top=0, lse_lo=False):
    """(logprob, entropy, lse, top_logprob, top_index) of the rows of logits [R, V]:
    the log probability of targets [R] (int64; negative: left out, 0), the entropy of
    the distribution, the log of the sum of exponentials ([R] float32 each), and the `top` (at most
    32) most probable tokens with their log probabilities ([R, top], equal logits by
    ascending token). With `lse_lo` lse is [2, R], for the backward: lse and what its rounding
    to float32 took from it."""
    R, V, stride = _check_logits(logits, targets)
    top = int(top)
    if not 0 <= top <= min(V, LOGPROBS_MAX_TOP):
        raise ValueError(f"top {top} is not within 0 .. {min(V, LOGPROBS_MAX_TOP)}")
    device, dt = logits.device, _DTYPES[logits.dtype]
    logprob, entropy = (torch.empty(R, dtype=torch.float32, device=device) for _ in range(2))
    lse = torch.empty((2, R) if lse_lo else (R,), dtype=torch.float32, device=device)
    top_logprob = torch.empty((R, top), dtype=torch.float32, device=device)
    top_index = torch.empty((R, top), dtype=torch.int64, device=device)
    nbytes = (_lib or _library()).simplicial_logprobs_fwd_workspace_size(R, V, top, dt)
    workspace = _workspace(nbytes, device)
    _call("simplicial_logprobs_fwd", device, logits.data_ptr(), targets.data_ptr(), logprob.data_ptr(), entropy.data_ptr(),
          lse.data_ptr(), _ptr(top_logprob) if top else None, _ptr(top_index) if top else None, _ptr(workspace), nbytes, R, V,
          stride, top, dt | LOGPROBS_LSE_LO if lse_lo else dt)
    return logprob, entropy, lse, top_logprob, top_index


def simplicial_logprobs_bwd(logits, targets, lse, entropy, d_logprob=None, d_entropy=None, d_lse=None, out=None):
    """Gradient of the logits from those of logprob, entropy and lse ([R] float32; None: zeros).
    lse [2, R], from a forward with lse_lo: without it the probabilities carry the rounding of
    lse to float32."""
    R, V, stride = _check_logits(logits, targets)
    device = logits.device
    lo = lse.dim() == 2
    _check_like(lse, (2, R) if lo else (R,), torch.float32, device, "lse")
    _check_like(entropy, (R,), torch.float32, device, "entropy")
    for t, name in ((d_logprob, "d_logprob"), (d_entropy, "d_entropy"), (d_lse, "d_lse")):
        if t is not None:
            _check_like(t, (R,), torch.float32, device, name)
    if out is None:
        out = torch.empty((R, V), dtype=logits.dtype, device=device)
    else:
        _check_like(out, (R, V), logits.dtype, device, "out")
    _call("simplicial_logprobs_bwd", device, logits.data_ptr(), targets.data_ptr(), lse.data_ptr(), entropy.data_ptr(),
          _ptr(d_logprob), _ptr(d_entropy), _ptr(d_lse), out.data_ptr(), R, V, stride,
          _DTYPES[logits.dtype] | (LOGPROBS_LSE_LO if lo else 0))
    return out

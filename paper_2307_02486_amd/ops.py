"""Python entry points of the dilated-attention forward and backward passes.

`plan`/`dilated_attn`, `plan_bwd`/`dilated_attn_bwd` and `xpos` mirror the
C ABI (dilated_attn_plan / dilated_attn_fwd, dilated_attn_bwd_plan /
dilated_attn_bwd, dilated_attn_xpos), and so do `qk_norm_xpos` and its
gradients, `cache_append` and `paged_attn` (both also on a cache in 8 bits),
`page_weights` and `evict_pages`: torch supplies device memory and the stream,
every step of the computation runs in the HIP kernels of libdilated_attn.so.
"""
from __future__ import annotations

import ctypes
import functools
from typing import Sequence, Tuple

import torch

from . import _lib

_DTYPES = {torch.float32: _lib.DA_F32, torch.bfloat16: _lib.DA_BF16}


def _dtype_code(dtype) -> int:
    if dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    return _DTYPES[dtype]


def _pattern_key(patterns) -> tuple:
    return tuple((int(w), int(r)) for (w, r) in patterns)


@functools.lru_cache(maxsize=256)
def _plan_cached(entry: str, B: int, N: int, H: int, D: int, pats: tuple, causal: int, dtype_code: int,
                 scale: float):
    """One dilated_attn_plan (or _bwd_plan) call per distinct problem: the
    returned dict is shared, callers must not modify it."""
    lib = _lib.load()
    arr, n = _lib.pattern_array(pats)
    info = _lib.PlanInfo()
    rc = getattr(lib, entry)(B, N, H, D, arr, n, causal, dtype_code, scale, ctypes.byref(info))
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    return {k: getattr(info, k) for k, _ in _lib.PlanInfo._fields_}


@functools.lru_cache(maxsize=256)
def _pattern_array_cached(pats: tuple):
    return _lib.pattern_array(pats)


_PREPARED: dict = {}  # calls by their integers, at most 256


def _prepared(entry: str, shape, patterns, causal: int, dtype_code: int, scale: float):
    """(workspace bytes, ctypes pattern array, pattern count) of a call.  Entries
    are kept under the patterns' integers only and found by the patterns as
    given, that is if these equal the integers at this call: whatever converts
    to an integer is converted at each call, and nothing given is kept."""
    patterns = tuple(patterns)
    try:
        hit = _PREPARED.get((entry, *shape, patterns, causal, dtype_code, scale))
        if hit is not None:
            return hit
    except TypeError:  # patterns given as lists
        pass
    pats = _pattern_key(patterns)
    info = _plan_cached(entry, *shape, pats, causal, dtype_code, scale)
    hit = (max(256, int(info["workspace_bytes"])), *_pattern_array_cached(pats))
    if len(_PREPARED) >= 256:
        _PREPARED.clear()
    _PREPARED[(entry, *shape, pats, causal, dtype_code, scale)] = hit
    return hit


@functools.lru_cache(maxsize=256)
def _workspace_bytes(entry: str, *dims: int) -> int:
    """The workspace size a dilated_attn_*_workspace entry point reports."""
    lib = _lib.load()
    need = ctypes.c_uint64(0)
    rc = getattr(lib, entry)(*dims, ctypes.byref(need))
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    return need.value


def _raw_stream(device: torch.device) -> int:
    """The HIP stream of torch's current stream on a device (the stream object
    that torch.cuda.current_stream builds costs 2 us a call)."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _call_on(dev: int, function, *args) -> int:
    """function(*args) with `dev` as the current device, whose null stream is meant
    where the stream is 0."""
    if torch._C._cuda_getDevice() == dev:
        return function(*args)
    with torch.cuda.device(dev):
        return function(*args)


def plan(B: int, N: int, H: int, D: int, patterns: Sequence[Tuple[int, int]], causal: bool = True,
         dtype=torch.bfloat16, scale: float | None = None) -> dict:
    """Validate a problem and return its workspace size and work counts (host only)."""
    return dict(_plan_cached("dilated_attn_plan", int(B), int(N), int(H), int(D), _pattern_key(patterns),
                             int(bool(causal)), _dtype_code(dtype), float(scale or 0.0)))


def plan_raw(B, N, H, D, patterns, causal, dtype_code, scale):
    """Call dilated_attn_plan with raw integer arguments; return (rc, info dict)."""
    lib = _lib.load()
    arr, n = _lib.pattern_array(patterns)
    info = _lib.PlanInfo()
    rc = lib.dilated_attn_plan(B, N, H, D, arr, n, causal, dtype_code, scale, ctypes.byref(info))
    return rc, {k: getattr(info, k) for k, _ in _lib.PlanInfo._fields_}


def workspace_for(q: torch.Tensor, patterns, causal=True, scale=None) -> torch.Tensor:
    """Allocate (with torch) the device workspace a call on q's shape needs."""
    B, N, H, D = q.shape
    info = _plan_cached("dilated_attn_plan", B, N, H, D, _pattern_key(patterns), int(bool(causal)),
                        _dtype_code(q.dtype), float(scale or 0.0))
    return torch.empty(max(256, int(info["workspace_bytes"])), dtype=torch.uint8, device=q.device)


def _check_like(name: str, t: torch.Tensor, shape, dtype, device):
    if t.shape != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")


def _stream_use(stream, owned):
    """Tensors this binding allocated on torch's current stream but handed to
    another stream's kernels: tell the allocator, so that their memory is not
    reused before that stream's work is done.  stream None: the current one."""
    if stream is not None and stream != torch.cuda.current_stream(stream.device):
        for t in owned:
            t.record_stream(stream)


def dilated_attn(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                 patterns: Sequence[Tuple[int, int]], causal: bool = True,
                 scale: float | None = None, out: torch.Tensor | None = None,
                 lse: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                 stream: torch.cuda.Stream | None = None):
    """Dilated-attention forward.  q, k, v: [B, N, H, D] contiguous on the GPU.

    Returns (out [B,N,H,D] in q's dtype, lse [B,H,N] float32).  Work is
    enqueued on `stream` (default: torch's current stream) and not waited for.
    A given out, lse or workspace must be a contiguous tensor of the right
    shape, dtype and device (workspace: uint8, at least the planned size).
    """
    lib = _lib.load()
    if q.device.type != "cuda":
        raise RuntimeError("dilated_attn runs on the GPU only; q must be a device tensor")
    if q.dim() != 4:
        raise ValueError("q, k, v must be [B, N, H, D]")
    for t in (q, k, v):
        if not t.is_contiguous() or t.shape != q.shape or t.dtype != q.dtype or t.device != q.device:
            raise ValueError("q, k, v must be contiguous tensors of the same shape, dtype and device")
    B, N, H, D = q.shape
    dcode = _dtype_code(q.dtype)
    sc = float(scale or 0.0)
    ws_bytes, arr, n = _prepared("dilated_attn_plan", q.shape, patterns, int(bool(causal)), dcode, sc)
    owned = []
    if out is None:
        out = torch.empty_like(q)
        owned.append(out)
    else:
        _check_like("out", out, q.shape, q.dtype, q.device)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
        owned.append(lse)
    else:
        _check_like("lse", lse, (B, H, N), torch.float32, q.device)
    if workspace is None:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device)
        owned.append(workspace)
    elif workspace.dtype != torch.uint8 or workspace.device != q.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
    raw = _raw_stream(q.device) if stream is None else stream.cuda_stream
    rc = lib.dilated_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                              B, N, H, D, arr, n, int(bool(causal)), dcode, sc,
                              workspace.data_ptr(), workspace.numel(), raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, owned)
    return out, lse


class StageTimer:
    """Context manager around dilated_attn_profile_begin/end: HIP event timing
    of the two launches of each call made inside it (on the call's own
    stream).  ms_attention and ms_combine sum the attention and the combine
    stage."""

    def __init__(self, capacity: int = 4096):
        self.capacity = capacity
        self.ms_attention = self.ms_combine = 0.0
        self.calls = 0

    def __enter__(self):
        lib = _lib.load()
        rc = lib.dilated_attn_profile_begin(self.capacity)
        if rc != 0:
            raise _lib.DilatedAttnError(rc, lib)
        return self

    def __exit__(self, *exc):
        lib = _lib.load()
        a, c, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_int64()
        rc = lib.dilated_attn_profile_end(ctypes.byref(a), ctypes.byref(c), ctypes.byref(n))
        if rc != 0 and exc[0] is None:
            raise _lib.DilatedAttnError(rc, lib)
        self.ms_attention, self.ms_combine, self.calls = a.value, c.value, n.value
        return False


def plan_bwd(B: int, N: int, H: int, D: int, patterns: Sequence[Tuple[int, int]], causal: bool = True,
             dtype=torch.bfloat16, scale: float | None = None) -> dict:
    """Validate a backward problem and return its workspace size and work (host only)."""
    return dict(_plan_cached("dilated_attn_bwd_plan", int(B), int(N), int(H), int(D), _pattern_key(patterns),
                             int(bool(causal)), _dtype_code(dtype), float(scale or 0.0)))


def bwd_workspace_for(q: torch.Tensor, patterns, causal=True, scale=None) -> torch.Tensor:
    """Allocate (with torch) the device workspace a backward call on q's shape needs."""
    B, N, H, D = q.shape
    info = plan_bwd(B, N, H, D, patterns, causal, q.dtype, scale)
    return torch.empty(max(256, int(info["workspace_bytes"])), dtype=torch.uint8, device=q.device)


def dilated_attn_bwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                     lse: torch.Tensor, dout: torch.Tensor, patterns: Sequence[Tuple[int, int]],
                     causal: bool = True, scale: float | None = None, dq: torch.Tensor | None = None,
                     dk: torch.Tensor | None = None, dv: torch.Tensor | None = None,
                     workspace: torch.Tensor | None = None, stream: torch.cuda.Stream | None = None):
    """Dilated-attention backward: (dq, dk, dv) given the forward's inputs and
    outputs (out, lse) and dout, all on the GPU, [B, N, H, D] contiguous
    (lse [B, H, N] float32).  Enqueued on `stream` and not waited for.  A
    given dq, dk, dv or workspace must be a contiguous tensor of the right
    shape, dtype and device."""
    lib = _lib.load()
    if q.device.type != "cuda":
        raise RuntimeError("dilated_attn_bwd runs on the GPU only; q must be a device tensor")
    if q.dim() != 4:
        raise ValueError("tensors must be [B, N, H, D]")
    for t in (q, k, v, out, dout):
        if not t.is_contiguous() or t.shape != q.shape or t.dtype != q.dtype or t.device != q.device:
            raise ValueError("q, k, v, out, dout must be contiguous tensors of the same shape, dtype, device")
    B, N, H, D = q.shape
    _check_like("lse", lse, (B, H, N), torch.float32, q.device)
    dcode = _dtype_code(q.dtype)
    sc = float(scale or 0.0)
    ws_bytes, arr, n = _prepared("dilated_attn_bwd_plan", q.shape, patterns, int(bool(causal)), dcode, sc)
    owned = []
    grads = []
    for name, g in (("dq", dq), ("dk", dk), ("dv", dv)):
        if g is None:
            g = torch.empty_like(q)
            owned.append(g)
        else:
            _check_like(name, g, q.shape, q.dtype, q.device)
        grads.append(g)
    dq, dk, dv = grads
    if workspace is None:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device)
        owned.append(workspace)
    elif workspace.dtype != torch.uint8 or workspace.device != q.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
    raw = _raw_stream(q.device) if stream is None else stream.cuda_stream
    rc = lib.dilated_attn_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                              dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, N, H, D,
                              arr, n, int(bool(causal)), dcode, sc,
                              workspace.data_ptr(), workspace.numel(), raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, owned)
    return dq, dk, dv


def xpos(x: torch.Tensor, sign: int, transpose: bool = False, center: int | None = None,
         base: float = 10000.0, gamma: float = 0.4, scale_base: float = 512.0,
         out: torch.Tensor | None = None, stream: torch.cuda.Stream | None = None) -> torch.Tensor:
    """xPos of a [B, N, H, D] query (sign=+1) or key (sign=-1) tensor on the
    GPU, or its transpose (transpose=True, the backward's map); center
    defaults to N // 2.  `out` may be x itself.  Enqueued on `stream`."""
    lib = _lib.load()
    if x.device.type != "cuda":
        raise RuntimeError("xpos runs on the GPU only; x must be a device tensor")
    if x.dim() != 4 or not x.is_contiguous():
        raise ValueError("x must be a contiguous [B, N, H, D] tensor")
    B, N, H, D = x.shape
    owned = []
    if out is None:
        out = torch.empty_like(x)
        owned.append(out)
    if out.shape != x.shape or out.dtype != x.dtype or out.device != x.device or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor like x")
    raw = _raw_stream(x.device) if stream is None else stream.cuda_stream
    rc = lib.dilated_attn_xpos(x.data_ptr(), out.data_ptr(), B, N, H, D, int(sign), int(bool(transpose)),
                               N // 2 if center is None else int(center), float(base), float(gamma),
                               float(scale_base), _dtype_code(x.dtype), raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, owned)
    return out


def wgrad(dy: torch.Tensor, x: torch.Tensor, out: torch.Tensor | None = None, bias_grad: bool = False,
          stream: torch.cuda.Stream | None = None):
    """dw = dy^T x for bf16 dy [K, M] and x [K, N] on the GPU (M, N multiples
    of 128): the weight gradient of a projection y = x w^T + b.  With
    bias_grad=True returns (dw, db), db = the column sums of dy.  Enqueued on
    `stream`; the float32 workspace comes from torch's caching allocator."""
    lib = _lib.load()
    if dy.device.type != "cuda" or x.device != dy.device:
        raise RuntimeError("wgrad runs on the GPU only; dy and x must be tensors of one device")
    if dy.dim() != 2 or x.dim() != 2 or dy.shape[0] != x.shape[0] or not dy.is_contiguous() \
            or not x.is_contiguous() or x.dtype != dy.dtype:
        raise ValueError("dy [K, M] and x [K, N] must be contiguous 2-D tensors of one dtype")
    K, M = dy.shape
    N = x.shape[1]
    need = _workspace_bytes("dilated_attn_wgrad_workspace", K, M, N)
    owned = []
    if out is None:
        out = torch.empty((M, N), dtype=dy.dtype, device=dy.device)
        owned.append(out)
    if out.shape != (M, N) or out.dtype != dy.dtype or out.device != dy.device or not out.is_contiguous():
        raise ValueError("out must be a contiguous [M, N] tensor of dy's dtype")
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=dy.device)
    raw = _raw_stream(dy.device) if stream is None else stream.cuda_stream
    db = torch.empty((M,), dtype=dy.dtype, device=dy.device) if bias_grad else None
    owned += [ws, db] if bias_grad else [ws]
    rc = lib.dilated_attn_wgrad(dy.data_ptr(), x.data_ptr(), out.data_ptr(), db.data_ptr() if bias_grad else None,
                                K, M, N, _dtype_code(dy.dtype), ws.data_ptr(), need, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, owned)
    return (out, db) if bias_grad else out


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor, eps: float = 1e-5,
               stream: torch.cuda.Stream | None = None):
    """LayerNorm over the last dimension of a contiguous bf16 tensor on the
    GPU (E a multiple of 8, at most 2048).  Returns (y, mean, rstd), the
    statistics float32 per row for layer_norm_bwd."""
    lib = _lib.load()
    if x.device.type != "cuda":
        raise RuntimeError("layer_norm runs on the GPU only; x must be a device tensor")
    if not x.is_contiguous() or not weight.is_contiguous() or not bias.is_contiguous():
        raise ValueError("x, weight and bias must be contiguous")
    if x.dim() == 0 or x.shape[-1] == 0:
        raise ValueError("x must have a non-empty last dimension")
    E = x.shape[-1]
    if weight.shape != (E,) or bias.shape != (E,) or weight.dtype != x.dtype or bias.dtype != x.dtype \
            or weight.device != x.device or bias.device != x.device:
        raise ValueError("weight and bias must be [E] tensors of x's dtype and device")
    rows = x.numel() // E
    y = torch.empty_like(x)
    mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    rstd = torch.empty_like(mean)
    raw = _raw_stream(x.device) if stream is None else stream.cuda_stream
    rc = lib.dilated_attn_layernorm_fwd(x.data_ptr(), weight.data_ptr(), bias.data_ptr(), y.data_ptr(),
                                        mean.data_ptr(), rstd.data_ptr(), rows, E, float(eps),
                                        _dtype_code(x.dtype), raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, [y, mean, rstd])
    return y, mean, rstd


def layer_norm_bwd(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, mean: torch.Tensor,
                   rstd: torch.Tensor, stream: torch.cuda.Stream | None = None):
    """Gradients (dx, dweight, dbias) of layer_norm given its saved mean and
    rstd; the float32 workspace comes from torch's caching allocator."""
    lib = _lib.load()
    if dy.device.type != "cuda" or x.device != dy.device:
        raise RuntimeError("layer_norm_bwd runs on the GPU only")
    if dy.shape != x.shape or dy.dtype != x.dtype or not dy.is_contiguous() or not x.is_contiguous():
        raise ValueError("dy and x must be contiguous tensors of one shape and dtype")
    if x.dim() == 0 or x.shape[-1] == 0:
        raise ValueError("x must have a non-empty last dimension")
    E = x.shape[-1]
    rows = x.numel() // E
    if weight.shape != (E,) or weight.dtype != x.dtype or weight.device != x.device:
        raise ValueError("weight must be an [E] tensor of x's dtype and device")
    if mean.numel() != rows or rstd.numel() != rows or mean.dtype != torch.float32 or rstd.dtype != torch.float32 \
            or not mean.is_contiguous() or not rstd.is_contiguous() or not weight.is_contiguous():
        raise ValueError("mean and rstd must be contiguous float32 tensors of one value per row")
    need = _workspace_bytes("dilated_attn_layernorm_bwd_workspace", rows, E)
    dx = torch.empty_like(x)
    dw = torch.empty((E,), dtype=x.dtype, device=x.device)
    db = torch.empty_like(dw)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    raw = _raw_stream(x.device) if stream is None else stream.cuda_stream
    rc = lib.dilated_attn_layernorm_bwd(dy.data_ptr(), x.data_ptr(), weight.data_ptr(), mean.data_ptr(),
                                        rstd.data_ptr(), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), rows, E,
                                        _dtype_code(x.dtype), ws.data_ptr(), need, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, [ws, dx, dw, db])
    return dx, dw, db


def _token_stride(name: str, t: torch.Tensor, lead: int, dtype, device) -> int:
    """Elements between the tokens of a [..., heads, D] tensor with `lead`
    leading dimensions whose heads are contiguous and whose tokens are evenly
    spaced (a contiguous tensor, or a slice of a joint projection's output)."""
    if t.dim() != lead + 2 or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a {lead + 2}-dimensional {dtype} tensor on {device}")
    H, D = t.shape[-2:]
    if (D > 1 and t.stride(-1) != 1) or (H > 1 and t.stride(-2) != D):
        raise ValueError(f"{name} must have the heads of a token contiguous")
    sizes, strides = t.shape[:lead], t.stride()[:lead]
    step, span = None, 1
    for n, s in zip(reversed(sizes), reversed(strides)):
        if n > 1:
            if step is None:
                step = s
                if span != 1:
                    raise ValueError(f"{name} must have its tokens evenly spaced")
            elif s != step * span:
                raise ValueError(f"{name} must have its tokens evenly spaced")
        span *= n
    return H * D if step is None else step


def _contiguous_like(t: torch.Tensor) -> torch.Tensor:
    """An empty contiguous tensor of t's shape (half the host time of torch.empty with a shape and a device)."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


# The sizes and strides of a call, validated and with what follows from them,
# by the shapes (at most 256 of each operator; nothing of a tensor is kept).
_HEADS: dict = {}
_APPENDS: dict = {}
_PAGED: dict = {}
_WEIGHTS: dict = {}


def _keep(known: dict, key, value):
    if len(known) >= 256:
        known.clear()
    known[key] = value
    return value


def _qk_call(q: torch.Tensor, k: torch.Tensor, q_weight: torch.Tensor, k_weight: torch.Tensor):
    """(B, N, H, Hkv, D, q's and k's token strides, dtype code) of a head norm's inputs."""
    key = (q.shape, k.shape, q.stride(), k.stride(), q.dtype)
    call = _HEADS.get(key)
    if call is None:
        if q.device.type != "cuda":
            raise RuntimeError("the head norms run on the GPU only; q must be a device tensor")
        if q.dim() != 4 or k.dim() != 4 or k.shape[:2] != q.shape[:2] or k.shape[3] != q.shape[3]:
            raise ValueError("q and k must be [B, N, H, D] and [B, N, Hkv, D]")
        B, N, H, D = q.shape
        call = _keep(_HEADS, key, (B, N, H, k.shape[2], D, _token_stride("q", q, 2, q.dtype, q.device),
                                   _token_stride("k", k, 2, q.dtype, k.device), _dtype_code(q.dtype), (D,)))
    dev, dt = q.get_device(), q.dtype
    if dev < 0:
        raise RuntimeError("the head norms run on the GPU only; q must be a device tensor")
    if k.dtype != dt or k.get_device() != dev:
        raise ValueError(f"k must be a {dt} tensor on {q.device}")
    if q_weight.shape != call[8] or k_weight.shape != call[8] or q_weight.dtype != dt or k_weight.dtype != dt \
            or q_weight.get_device() != dev or k_weight.get_device() != dev \
            or not q_weight.is_contiguous() or not k_weight.is_contiguous():
        raise ValueError(f"q_weight and k_weight must be contiguous {dt} tensors of shape {call[8]} on {q.device}")
    return call


def qk_norm_xpos(q: torch.Tensor, k: torch.Tensor, q_weight: torch.Tensor, k_weight: torch.Tensor,
                 eps: float = 1e-6, center: int | None = None, base: float = 10000.0, gamma: float = 0.4,
                 scale_base: float = 512.0, stream: torch.cuda.Stream | None = None):
    """RMS norm of every head of q [B, N, H, D] and k [B, N, Hkv, D] with the
    weights [D], then xPos (sign +1 for q, -1 for k; center defaults to
    N // 2), in one pass.  The heads of a token are contiguous and the tokens
    evenly spaced.  Returns new contiguous (q_out, k_out).  Enqueued on `stream`."""
    lib = _lib.load()
    B, N, H, Hkv, D, qs, ks, dcode, _ = _qk_call(q, k, q_weight, k_weight)
    qo, ko = _contiguous_like(q), _contiguous_like(k)
    raw = _raw_stream(q.device) if stream is None else stream.cuda_stream
    rc = lib.dilated_attn_qk_norm_xpos(q.data_ptr(), k.data_ptr(), q_weight.data_ptr(), k_weight.data_ptr(),
                                       qo.data_ptr(), ko.data_ptr(), B, N, H, Hkv, D, qs, ks, float(eps),
                                       N // 2 if center is None else int(center), float(base), float(gamma),
                                       float(scale_base), dcode, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, [qo, ko])
    return qo, ko


def qk_norm_xpos_bwd(dq_out: torch.Tensor, dk_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                     q_weight: torch.Tensor, k_weight: torch.Tensor, eps: float = 1e-6, center: int | None = None,
                     base: float = 10000.0, gamma: float = 0.4, scale_base: float = 512.0,
                     stream: torch.cuda.Stream | None = None):
    """Gradients (dq, dk, dq_weight, dk_weight) of qk_norm_xpos given its inputs
    and the contiguous gradients of its outputs; the float32 workspace comes
    from torch's caching allocator."""
    lib = _lib.load()
    B, N, H, Hkv, D, qs, ks, dcode, _ = _qk_call(q, k, q_weight, k_weight)
    _check_like("dq_out", dq_out, q.shape, q.dtype, q.device)
    _check_like("dk_out", dk_out, k.shape, q.dtype, q.device)
    need = _workspace_bytes("dilated_attn_qk_norm_xpos_bwd_workspace", B, N, D)
    dq, dk = torch.empty_like(dq_out), torch.empty_like(dk_out)
    dqw, dkw = torch.empty_like(q_weight), torch.empty_like(k_weight)
    ws = q.new_empty(need, dtype=torch.uint8)
    raw = _raw_stream(q.device) if stream is None else stream.cuda_stream
    rc = lib.dilated_attn_qk_norm_xpos_bwd(
        dq_out.data_ptr(), dk_out.data_ptr(), q.data_ptr(), k.data_ptr(), q_weight.data_ptr(), k_weight.data_ptr(),
        dq.data_ptr(), dk.data_ptr(), dqw.data_ptr(), dkw.data_ptr(), B, N, H, Hkv, D, qs, ks, float(eps),
        N // 2 if center is None else int(center), float(base), float(gamma), float(scale_base), dcode,
        ws.data_ptr(), need, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, [dq, dk, dqw, dkw, ws])
    return dq, dk, dqw, dkw


def _cache_shape(k_cache: torch.Tensor, block_table: torch.Tensor, D: int):
    """(B, Hkv, num_pages, page_size, max_pages) of a cache and its table."""
    if k_cache.dim() != 4:
        raise ValueError("k_cache and v_cache must be [num_pages, Hkv, page_size, D]")
    pages, Hkv, page, Dc = k_cache.shape
    if Dc != D:
        raise ValueError(f"k_cache holds heads of {Dc}, the call has heads of {D}")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B, max_pages]")
    B, max_pages = block_table.shape
    return B, Hkv, pages, page, max_pages


CACHE_F8 = torch.float8_e4m3fn  # values of a cache in 8 bits
CACHE_SCALE = torch.float8_e8m0fnu  # powers of two, one for each block of tokens and key head
CACHE_BLOCK = 16  # tokens of a block (a page of fewer is one block)


def cache_scale_shape(k_cache) -> tuple:
    """[num_pages, Hkv, blocks of a page]: the shape of the scales of a cache in 8 bits (a tensor or its shape)."""
    pages, Hkv, page, _ = getattr(k_cache, "shape", k_cache)
    return pages, Hkv, page // min(page, CACHE_BLOCK)


def _check_scale(name: str, scale, cache: torch.Tensor):
    """Refuse a cache in 8 bits without its scales, or with others than its own."""
    if scale is None:
        raise ValueError(f"a cache in 8 bits needs {name}")
    if scale.dtype != CACHE_SCALE or scale.get_device() != cache.get_device() or not scale.is_contiguous() \
            or scale.shape != cache_scale_shape(cache):
        raise ValueError(f"{name} must be a contiguous {CACHE_SCALE} tensor of shape {list(cache_scale_shape(cache))} "
                         f"on the cache's device")


def _cache_args(k_cache, v_cache, block_table, seq_lens, q_start, pages, page, max_pages):
    return _lib.PagedCacheArgs(k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                               q_start.data_ptr(), pages, page, max_pages)


def _check_cache(dev: int, dtype, B: int, k_cache, v_cache, block_table, seq_lens, q_start):
    """Refuse cache tensors of another type, device, shape or layout than the call's."""
    i32 = torch.int32
    if dev < 0 or k_cache.get_device() != dev or v_cache.get_device() != dev or block_table.get_device() != dev \
            or seq_lens.get_device() != dev or q_start.get_device() != dev:
        raise ValueError("the cache, block_table, seq_lens and q_start must be on the tokens' device")
    if k_cache.dtype != dtype or v_cache.dtype != dtype or v_cache.shape != k_cache.shape \
            or not k_cache.is_contiguous() or not v_cache.is_contiguous():
        raise ValueError(f"k_cache and v_cache must be contiguous {dtype} tensors of one shape")
    if block_table.dtype != i32 or seq_lens.dtype != i32 or q_start.dtype != i32 \
            or seq_lens.shape != (B,) or q_start.shape != (B + 1,) or not block_table.is_contiguous() \
            or not seq_lens.is_contiguous() or not q_start.is_contiguous():
        raise ValueError(f"block_table, seq_lens and q_start must be contiguous int32 tensors of shapes "
                         f"[{B}, max_pages], [{B}] and [{B + 1}]")


def cache_append(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor,
                 v_cache: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor, q_start: torch.Tensor,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-6,
                 rotate: bool = True, center: int = 0, base: float = 10000.0, gamma: float = 0.4,
                 scale_base: float = 512.0, stream: torch.cuda.Stream | None = None,
                 k_scale: torch.Tensor | None = None, v_scale: torch.Tensor | None = None):
    """New keys and values into a paged cache, the keys normed (with k_weight)
    and rotated by xPos on the way; returns the queries normed (with q_weight)
    and rotated, [T, H, D], or None without q.

    q [T, H, D], k and v [T, Hkv, D]: the new tokens of all sequences side by
    side, those of sequence b in rows q_start[b]:q_start[b + 1] (int32 [B + 1]).
    They are the last of its seq_lens[b] tokens (int32 [B]).  Token p lies in
    page block_table[b, p // page_size] (int32 [B, max_pages]) of k_cache and
    v_cache [num_pages, Hkv, page_size, D], page_size a power of two.  `center`
    is the xPos centre, the same for the life of a cache.  Enqueued on `stream`.

    A cache in 8 bits: k_cache and v_cache are float8_e4m3fn, k_scale and v_scale
    float8_e8m0fnu [num_pages, Hkv, page_size / 16] (cache_scale_shape), a power of
    two for each block of 16 tokens and key head.  An element is its e4m3 value
    times its block's scale, the least that cuts no value off; a block keeps its
    scale or takes a larger one as tokens come, its older values then rescaled."""
    lib = _lib.load()
    key = (None if q is None else (q.shape, q.stride()), k.shape, k.stride(), v.shape, v.stride(), k.dtype,
           k_cache.shape, block_table.shape)
    call = _APPENDS.get(key)
    if call is None:
        if k.device.type != "cuda":
            raise RuntimeError("cache_append runs on the GPU only; k must be a device tensor")
        if k.dim() != 3 or v.shape != k.shape:
            raise ValueError("k and v must be [T, Hkv, D]")
        T, Hkv, D = k.shape
        ks, vs = _token_stride("k", k, 1, k.dtype, k.device), _token_stride("v", v, 1, v.dtype, v.device)
        B, cached, pages, page, max_pages = _cache_shape(k_cache, block_table, D)
        if cached != Hkv:
            raise ValueError(f"the cache has {cached} key heads, k has {Hkv}")
        H, qs = Hkv, Hkv * D
        if q is not None:
            if q.dim() != 3 or q.shape[0] != T or q.shape[2] != D:
                raise ValueError("q must be [T, H, D] for the tokens of k")
            H, qs = q.shape[1], _token_stride("q", q, 1, q.dtype, q.device)
        call = _keep(_APPENDS, key, (T, B, H, Hkv, D, qs, ks, vs, _dtype_code(k.dtype), pages, page, max_pages))
    T, B, H, Hkv, D, qs, ks, vs, dcode, pages, page, max_pages = call
    dev, dt = k.get_device(), k.dtype
    if dev < 0:
        raise RuntimeError("cache_append runs on the GPU only; k must be a device tensor")
    f8 = k_cache.dtype == CACHE_F8
    _check_cache(dev, CACHE_F8 if f8 else dt, B, k_cache, v_cache, block_table, seq_lens, q_start)
    if f8:
        _check_scale("k_scale", k_scale, k_cache)
        _check_scale("v_scale", v_scale, v_cache)
    elif k_scale is not None or v_scale is not None:
        raise ValueError(f"k_scale and v_scale go with a cache of {CACHE_F8}")
    if v.dtype != dt or v.get_device() != dev:
        raise ValueError(f"v must be a {dt} tensor on {k.device}")
    qo = None
    if q is not None:
        if q.dtype != dt or q.get_device() != dev:
            raise ValueError(f"q must be a {dt} tensor on {k.device}")
        qo = _contiguous_like(q)
    elif q_weight is not None:
        raise ValueError("q_weight without q")
    if q_weight is not None:
        _check_like("q_weight", q_weight, (D,), dt, k.device)
    if k_weight is not None:
        _check_like("k_weight", k_weight, (D,), dt, k.device)
    cache, append = _cache_args(k_cache, v_cache, block_table, seq_lens, q_start, pages, page, max_pages), \
        lib.dilated_attn_cache_append
    if f8:
        cache, append = _lib.PagedCacheF8Args(cache, k_scale.data_ptr(), v_scale.data_ptr()), \
            lib.dilated_attn_cache_append_f8
    raw = _raw_stream(k.device) if stream is None else stream.cuda_stream
    rc = _call_on(
        dev, append, None if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(),
        None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
        None if qo is None else qo.data_ptr(), cache, T, B, H, Hkv, D, qs, ks, vs, float(eps),
        1 if rotate else 0, int(center), float(base), float(gamma), float(scale_base), dcode, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    if qo is not None:
        _stream_use(stream, [qo])
    return qo


@functools.lru_cache(maxsize=256)
def _paged_workspace(shape: tuple, pats: tuple, dtype_code: int) -> int:
    lib = _lib.load()
    arr, n = _pattern_array_cached(pats)
    need = ctypes.c_uint64(0)
    rc = lib.dilated_attn_paged_workspace(*shape, arr, n, dtype_code, ctypes.byref(need))
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    return need.value


def paged_attn(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
               seq_lens: torch.Tensor, q_start: torch.Tensor, patterns: Sequence[Tuple[int, int]],
               max_new: int | None = None, scale: float | None = None, out: torch.Tensor | None = None,
               lse: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
               stream: torch.cuda.Stream | None = None, k_scale: torch.Tensor | None = None,
               v_scale: torch.Tensor | None = None):
    """Causal dilated attention of new tokens q [T, H, D] over a paged cache that
    holds their keys and values already (see cache_append for the cache and
    the sequences' arrays): a token at position p gets what row p of
    dilated_attn gives on its sequence.  H is a multiple of the cache's heads.

    max_new, the most new tokens of any sequence if the caller knows it,
    spares what only longer ones need where it is at most 4.  Returns (out
    [T, H, D], lse [H, T] float32); a token of no sequence has zeros and -inf.
    Enqueued on `stream`.  A given workspace is a contiguous uint8 tensor of
    at least paged_workspace_bytes.

    A cache in 8 bits comes with k_scale and v_scale, as for cache_append.  Its
    table may name pages outside the pool (-1, say): they hold no keys, and a row
    all of whose keys are gone has zeros and -inf."""
    lib = _lib.load()
    patterns = tuple(patterns)
    shapes = (q.shape, q.stride(), q.dtype, k_cache.shape, block_table.shape, max_new)
    try:
        call = _PAGED.get((shapes, patterns))
    except TypeError:  # patterns given as lists
        call = None
    if call is None:
        if q.device.type != "cuda":
            raise RuntimeError("paged_attn runs on the GPU only; q must be a device tensor")
        if q.dim() != 3:
            raise ValueError("q must be [T, H, D]")
        T, H, D = q.shape
        B, Hkv, pages, page, max_pages = _cache_shape(k_cache, block_table, D)
        dcode, pats = _dtype_code(q.dtype), _pattern_key(patterns)
        new = T if max_new is None else int(max_new)
        need = _paged_workspace((T, B, H, Hkv, D, pages, page, max_pages, new), pats, dcode)
        call = _keep(_PAGED, (shapes, pats), (T, B, H, Hkv, D, _token_stride("q", q, 1, q.dtype, q.device), dcode, pages,
                                              page, max_pages, new, max(need, 16), *_pattern_array_cached(pats)))
    T, B, H, Hkv, D, qs, dcode, pages, page, max_pages, new, need, arr, n = call
    dev = q.get_device()
    if dev < 0:
        raise RuntimeError("paged_attn runs on the GPU only; q must be a device tensor")
    f8 = k_cache.dtype == CACHE_F8
    _check_cache(dev, CACHE_F8 if f8 else q.dtype, B, k_cache, v_cache, block_table, seq_lens, q_start)
    if f8:
        _check_scale("k_scale", k_scale, k_cache)
        _check_scale("v_scale", v_scale, v_cache)
    elif k_scale is not None or v_scale is not None:
        raise ValueError(f"k_scale and v_scale go with a cache of {CACHE_F8}")
    owned = []
    if out is None:
        out = _contiguous_like(q)
        owned.append(out)
    else:
        _check_like("out", out, (T, H, D), q.dtype, q.device)
    if lse is None:
        lse = q.new_empty((H, T), dtype=torch.float32)
        owned.append(lse)
    else:
        _check_like("lse", lse, (H, T), torch.float32, q.device)
    if workspace is None:
        workspace, nbytes = q.new_empty(need, dtype=torch.uint8), need
        owned.append(workspace)
    else:
        if workspace.dtype != torch.uint8 or workspace.device != q.device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
        nbytes = workspace.numel()
    cache, attend = _cache_args(k_cache, v_cache, block_table, seq_lens, q_start, pages, page, max_pages), \
        lib.dilated_attn_paged_fwd
    if f8:
        cache, attend = _lib.PagedCacheF8Args(cache, k_scale.data_ptr(), v_scale.data_ptr()), \
            lib.dilated_attn_paged_fwd_f8
    raw = _raw_stream(q.device) if stream is None else stream.cuda_stream
    rc = _call_on(dev, attend, q.data_ptr(), cache, out.data_ptr(), lse.data_ptr(), T, B, H, Hkv, D, qs, new, arr, n,
                  dcode, float(scale or 0.0), workspace.data_ptr(), nbytes, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, owned)
    return out, lse


def paged_workspace_bytes(T: int, B: int, H: int, Hkv: int, D: int, num_pages: int, page_size: int, max_pages: int,
                          patterns: Sequence[Tuple[int, int]], max_new: int | None = None,
                          dtype=torch.bfloat16) -> int:
    """Validate a paged_attn problem and return the workspace it needs (host only)."""
    shape = (int(T), int(B), int(H), int(Hkv), int(D), int(num_pages), int(page_size), int(max_pages),
             int(T if max_new is None else max_new))
    return _paged_workspace(shape, _pattern_key(patterns), _dtype_code(dtype))


@functools.lru_cache(maxsize=256)
def _weight_workspace(shape: tuple, pats: tuple, dtype_code: int) -> int:
    lib = _lib.load()
    arr, n = _pattern_array_cached(pats)
    need = ctypes.c_uint64(0)
    rc = lib.dilated_attn_page_weights_workspace(*shape, arr, n, dtype_code, ctypes.byref(need))
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    return need.value


def page_weights(q: torch.Tensor, lse: torch.Tensor, k_cache: torch.Tensor, k_scale: torch.Tensor,
                 block_table: torch.Tensor, seq_lens: torch.Tensor, q_start: torch.Tensor,
                 patterns: Sequence[Tuple[int, int]], weights: torch.Tensor, scale: float | None = None,
                 workspace: torch.Tensor | None = None, stream: torch.cuda.Stream | None = None,
                 max_new: int | None = None) -> torch.Tensor:
    """The attention that each page of a cache in 8 bits gets from the new tokens,
    added to weights (float32 [num_pages], which is returned): over the page's
    keys, the tokens q [T, H, D] of its sequence that see them, their heads and
    the patterns that hold the pair, the sum of exp(scale q.k - lse).

    q, the cache and the sequences' arrays are those of paged_attn, lse [H, T]
    what it returned; a row without a finite lse adds nothing.  Each head of a
    token that sees a key adds one in all.  The tables name a page once.
    max_new, the most new tokens of any sequence if the caller knows it, chooses how
    the work is cut.  Enqueued on `stream`.  A given workspace is a contiguous uint8
    tensor of at least page_weights_workspace_bytes, one call's at a time."""
    lib = _lib.load()
    patterns = tuple(patterns)
    shapes = (q.shape, q.stride(), q.dtype, k_cache.shape, block_table.shape, max_new)
    try:
        call = _WEIGHTS.get((shapes, patterns))
    except TypeError:  # patterns given as lists
        call = None
    if call is None:
        if q.device.type != "cuda":
            raise RuntimeError("page_weights runs on the GPU only; q must be a device tensor")
        if q.dim() != 3:
            raise ValueError("q must be [T, H, D]")
        T, H, D = q.shape
        B, Hkv, pages, page, max_pages = _cache_shape(k_cache, block_table, D)
        dcode, pats = _dtype_code(q.dtype), _pattern_key(patterns)
        new = int(max_new or 0)
        need = _weight_workspace((T, B, H, Hkv, D, pages, page, max_pages, new), pats, dcode)
        call = _keep(_WEIGHTS, (shapes, pats), (T, B, H, Hkv, D, _token_stride("q", q, 1, q.dtype, q.device), dcode, pages,
                                                page, max_pages, new, max(need, 16), *_pattern_array_cached(pats)))
    T, B, H, Hkv, D, qs, dcode, pages, page, max_pages, new, need, arr, n = call
    dev = q.get_device()
    if dev < 0:
        raise RuntimeError("page_weights runs on the GPU only; q must be a device tensor")
    if k_cache.dtype != CACHE_F8:
        raise ValueError(f"k_cache must be a {CACHE_F8} tensor, a cache in 8 bits")
    _check_cache(dev, CACHE_F8, B, k_cache, k_cache, block_table, seq_lens, q_start)
    _check_scale("k_scale", k_scale, k_cache)
    _check_like("lse", lse, (H, T), torch.float32, q.device)
    _check_like("weights", weights, (pages,), torch.float32, q.device)
    owned = []
    if workspace is None:
        workspace, nbytes = q.new_empty(need, dtype=torch.uint8), need
        owned.append(workspace)
    else:
        if workspace.dtype != torch.uint8 or workspace.device != q.device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
        nbytes = workspace.numel()
    cache = _lib.PagedCacheF8Args(_cache_args(k_cache, k_cache, block_table, seq_lens, q_start, pages, page, max_pages),
                                  k_scale.data_ptr(), None)
    raw = _raw_stream(q.device) if stream is None else stream.cuda_stream
    rc = _call_on(dev, lib.dilated_attn_page_weights, q.data_ptr(), lse.data_ptr(), cache, weights.data_ptr(), T, B, H,
                  Hkv, D, qs, new, arr, n, dcode, float(scale or 0.0), workspace.data_ptr(), nbytes, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, owned)
    return weights


def page_weights_workspace_bytes(T: int, B: int, H: int, Hkv: int, D: int, num_pages: int, page_size: int,
                                 max_pages: int, patterns: Sequence[Tuple[int, int]], dtype=torch.bfloat16,
                                 max_new: int | None = None) -> int:
    """Validate a page_weights problem and return the workspace it needs (host only)."""
    shape = (int(T), int(B), int(H), int(Hkv), int(D), int(num_pages), int(page_size), int(max_pages),
             int(max_new or 0))
    return _weight_workspace(shape, _pattern_key(patterns), _dtype_code(dtype))


def evict_pages(weights: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor, page_size: int, keep: int,
                first: int = 1, last: int = 1, stream: torch.cuda.Stream | None = None):
    """The pages of least weight out of each sequence's table, until it has `keep`.

    weights float32 [num_pages], block_table int32 [B, max_pages], seq_lens int32
    [B]; entries of a row outside [0, num_pages) are pages that are not there.  Of
    equal weights the page that comes first goes.  The row's first `first` entries
    and the last `last` of those that its length reaches into never go.  Returns
    (table, freed, count): the table with -1 for what goes, the pages that go in
    the row's order and -1 after them [B, max_pages], and how many they are [B].
    Enqueued on `stream`."""
    lib = _lib.load()
    dev = weights.get_device()
    if dev < 0:
        raise RuntimeError("evict_pages runs on the GPU only; weights must be a device tensor")
    if block_table.dim() != 2 or weights.dim() != 1:
        raise ValueError("weights must be [num_pages] and block_table [B, max_pages]")
    B, max_pages = block_table.shape
    _check_like("weights", weights, weights.shape, torch.float32, weights.device)
    _check_like("block_table", block_table, (B, max_pages), torch.int32, weights.device)
    _check_like("seq_lens", seq_lens, (B,), torch.int32, weights.device)
    table, freed = torch.empty_like(block_table), torch.empty_like(block_table)
    count = torch.empty_like(seq_lens)
    raw = _raw_stream(weights.device) if stream is None else stream.cuda_stream
    keep, first, last = (min(int(n), 2 ** 31 - 1) for n in (keep, first, last))  # more than a table has
    rc = _call_on(dev, lib.dilated_attn_evict_pages, weights.data_ptr(), block_table.data_ptr(), seq_lens.data_ptr(),
                  table.data_ptr(), freed.data_ptr(), count.data_ptr(), B, weights.numel(), int(page_size), max_pages,
                  keep, first, last, raw)
    if rc != 0:
        raise _lib.DilatedAttnError(rc, lib)
    _stream_use(stream, [table, freed, count])
    return table, freed, count

"""ctypes binding of the C ABI in include/tas_step.h: the attention part of one
serving iteration (append to the paged KV cache, attention over it).

Every operator runs in the HIP kernels of ``libtas_step.so``; this module checks
tensors and converts arguments. It raises if the library is missing: there is no
fallback. The functions keep the C names; ``Step`` bundles them for one batch,
allocating the workspace and outputs as PyTorch tensors.

    step = Step(n_new, kv_len, blocks, heads=32, kv_heads=8, head_dim=128,
                block_tokens=16, n_blocks=8192)
    for layer in layers:
        q = step.append(layer.qkv(x), k_cache, v_cache, cos, sin)
        o = step.attention(q, k_cache, v_cache)
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct

import numpy as np
import torch
from torch.autograd import forward_ad

from .tas import TAS_OK, TasError, _stream

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libtas_step.so")
TAS_F16, TAS_BF16 = 0, 1
DTYPES = {torch.float16: TAS_F16, torch.bfloat16: TAS_BF16}

_P, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class tas_batch(ctypes.Structure):
    _fields_ = [("heads", _i32), ("kv_heads", _i32), ("head_dim", _i32), ("block_tokens", _i32),
                ("n_req", _i32), ("n_blocks", _i32), ("causal", _i32), ("n_prefix", _i32),
                ("n_new", _P), ("kv_len", _P), ("blocks", _P), ("blocks_stride", _i64),
                ("prefix_first", _P), ("prefix_len", _P), ("prefix_blocks", _P),
                ("prefix_stride", _i64)]


class tas_cache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_block", _i64), ("k_head", _i64), ("k_token", _i64),
                ("v_block", _i64), ("v_head", _i64), ("v_token", _i64)]


class tas_append(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("rot_dim", _i32), ("interleaved", _i32),
                ("eps", ctypes.c_float), ("qkv", _P), ("qkv_stride", _i64), ("q_out", _P),
                ("q_out_stride", _i64), ("q_weight", _P), ("k_weight", _P), ("cos", _P),
                ("sin", _P), ("positions", _i64), ("cache", tas_cache)]


class tas_attention(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("scale", ctypes.c_float), ("q", _P), ("q_stride", _i64),
                ("out", _P), ("out_stride", _i64), ("lse", _P), ("cache", tas_cache)]


# The same two structs for Step's calls, which are made for every layer: packing takes
# a third of the time of a ctypes constructor.
_CACHE = "PPqqqqqq"
_APPEND = struct.Struct("iiifPqPqPPPPq" + _CACHE)
_ATTENTION = struct.Struct("ifPqPqP" + _CACHE)
_CACHE_FP4 = 4 * "Pqqq"
_APPEND_FP4 = struct.Struct("iiifPqPqPPPPq" + _CACHE_FP4)  # those of include/tas_fp4.h
_ATTENTION_FP4 = struct.Struct("ifPqPqP" + _CACHE_FP4)
assert _APPEND.size == ctypes.sizeof(tas_append)
assert _ATTENTION.size == ctypes.sizeof(tas_attention)

EXPORTS = ["tas_step_create", "tas_step_bytes", "tas_step_bind", "tas_step_attach",
           "tas_step_destroy", "tas_step_tokens", "tas_step_append", "tas_step_attention",
           "tas_step_plan"]

_lib = None


def lib():
    """Load libtas_step.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run __graft_entry__.build() "
                              "or python -m paper_2606_18431_amd.build")
        L = ctypes.CDLL(LIB_PATH)
        L.tas_step_bytes.argtypes = [_P]
        L.tas_step_bytes.restype = ctypes.c_size_t
        L.tas_step_create.argtypes = [_P, ctypes.POINTER(_P)]
        L.tas_step_bind.argtypes = [_P, _P, ctypes.c_size_t, _P]
        L.tas_step_attach.argtypes = [_P, _P, ctypes.c_size_t]
        L.tas_step_destroy.argtypes = [_P]
        L.tas_step_destroy.restype = None
        L.tas_step_tokens.argtypes = [_P]
        L.tas_step_tokens.restype = _i64
        L.tas_step_append.argtypes = [_P, _P, _P]
        L.tas_step_attention.argtypes = [_P, _P, _P]
        L.tas_step_plan.argtypes = [_P, _P, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)]
        L.tas_fp4_append.argtypes = [_P, _P, _P]
        L.tas_fp4_attention.argtypes = [_P, _P, _P]
        L.tas_fp4_pack.argtypes = [_P, _P]
        L.tas_fp4_values.argtypes = [_P, _P]
        L.tas_fp4_cache_values.argtypes = [_P, _P]
        L.tas_fp4_weights_bytes.argtypes = [_i64, _i64]
        L.tas_fp4_weights_bytes.restype = ctypes.c_size_t
        L.tas_fp4_weights.argtypes = [_i64, _i64, _P, _i64, _P, _i64, _P, _P]
        L.tas_fp4_linear.argtypes = [_P, _P]
        L.tas_fp4_linear_kernel.argtypes = [_i64, _i64, _i64]
        _lib = L
    return _lib


def _check(rc: int, what: str):
    if rc != TAS_OK:
        raise TasError(rc, what)


def _int32(x, what):
    """A contiguous int32 array of whole numbers (no value changes on the way)."""
    a = np.asarray(x)
    if a.size and a.dtype.kind not in "iu":
        raise ValueError(f"{what} holds {a.dtype}, expected whole numbers")
    if a.size and (a.min() < -2 ** 31 or a.max() >= 2 ** 31):
        raise ValueError(f"{what} holds values beyond 32 bits")
    return np.ascontiguousarray(a, np.int32)


def _size(x, what):
    """A whole number of 32 bits (ctypes would cut a longer one)."""
    x = operator.index(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{what} is {x}, beyond 32 bits")
    return x


def make_batch(n_new, kv_len, blocks, *, heads, kv_heads, head_dim, block_tokens, n_blocks,
               prefix_first=None, prefix_len=None, prefix_blocks=None, causal=True):
    """tas_batch over host arrays; returns (struct, keepalive). ``blocks`` is
    [n_req, pages] and ``prefix_blocks`` [groups, pages], rows as long as the
    longest context needs. The three prefix arguments: all or none."""
    given = [x is not None for x in (prefix_first, prefix_len, prefix_blocks)]
    if any(given) != all(given):
        raise ValueError("prefix_first, prefix_len and prefix_blocks: all or none")
    n, kv, bl = _int32(n_new, "n_new"), _int32(kv_len, "kv_len"), _int32(blocks, "blocks")
    if n.ndim != 1 or kv.shape != n.shape:
        raise ValueError(f"n_new has shape {n.shape}, kv_len {kv.shape}")
    if bl.ndim != 2 or bl.shape[0] != len(n):
        raise ValueError(f"blocks has shape {bl.shape} for {len(n)} requests")
    keep = [n, kv, bl]
    b = tas_batch(_size(heads, "heads"), _size(kv_heads, "kv_heads"), _size(head_dim, "head_dim"),
                  _size(block_tokens, "block_tokens"), len(n), _size(n_blocks, "n_blocks"),
                  int(bool(causal)), 0, n.ctypes.data, kv.ctypes.data, bl.ctypes.data, bl.shape[1])
    if prefix_first is not None:
        pf = _int32(prefix_first, "prefix_first")
        pl = _int32(prefix_len, "prefix_len")
        pb = _int32(prefix_blocks, "prefix_blocks")
        if pf.ndim != 1 or len(pf) < 2 or pl.shape != (len(pf) - 1,):
            raise ValueError(f"prefix_first has shape {pf.shape}, prefix_len {pl.shape}")
        if pb.ndim != 2 or pb.shape[0] != len(pl):
            raise ValueError(f"prefix_blocks has shape {pb.shape} for {len(pl)} groups")
        keep += [pf, pl, pb]
        b.n_prefix, b.prefix_stride = len(pl), pb.shape[1]
        b.prefix_first, b.prefix_len = pf.ctypes.data, pl.ctypes.data
        b.prefix_blocks = pb.ctypes.data
    return b, keep


def tas_step_create(batch: tas_batch) -> int:
    """Returns a step handle (int)."""
    ctx = _P()
    _check(lib().tas_step_create(ctypes.byref(batch), ctypes.byref(ctx)), "tas_step_create")
    return ctx.value


def tas_step_bytes(ctx) -> int:
    return int(lib().tas_step_bytes(ctx))


def tas_step_bind(ctx, ws: int, ws_bytes: int, stream=None):
    """``ws``: a device address."""
    _check(lib().tas_step_bind(ctx, ws, ws_bytes, _stream(stream)), "tas_step_bind")


def tas_step_attach(ctx, ws: int, ws_bytes: int):
    """``ws``: a device address, where the caller puts the plan."""
    _check(lib().tas_step_attach(ctx, ws, ws_bytes), "tas_step_attach")


def tas_step_tokens(ctx) -> int:
    return int(lib().tas_step_tokens(ctx))


def tas_step_plan(ctx) -> bytes:
    """The plan that tas_step_bind copies to the device."""
    n = ctypes.c_size_t()
    _check(lib().tas_step_plan(ctx, None, 0, ctypes.byref(n)), "tas_step_plan")
    buf = ctypes.create_string_buffer(n.value)
    _check(lib().tas_step_plan(ctx, buf, n.value, ctypes.byref(n)), "tas_step_plan")
    return buf.raw


def tas_step_append(ctx, args: tas_append, stream=None):
    _check(lib().tas_step_append(ctx, ctypes.byref(args), _stream(stream)), "tas_step_append")


def tas_step_attention(ctx, args: tas_attention, stream=None):
    _check(lib().tas_step_attention(ctx, ctypes.byref(args), _stream(stream)),
           "tas_step_attention")


def tas_step_destroy(ctx):
    if ctx:
        lib().tas_step_destroy(ctx)


def _no_tangent(*tensors):
    """Refuses dual tensors of forward-mode differentiation: a result without a tangent
    would say that its derivative is zero."""
    if forward_ad._current_level >= 0:
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise NotImplementedError("the serving step has no forward-mode derivative")


class _NoBackward(torch.autograd.Function):
    """Outputs of inputs that require a gradient say so, and refuse to compute it."""

    @staticmethod
    def forward(ctx, out, *inputs):
        return out.detach()

    @staticmethod
    def backward(ctx, *grads):
        raise NotImplementedError("the serving step has no backward pass")


class Step:
    """The plan of one batch on one GPU: made once when the scheduler has
    formed the batch, used for every layer.

    Caches are tensors [n_blocks, kv_heads, block_tokens, head_dim], any strides
    (a permuted view serves other orders) whose last is 1. Calls are enqueued on
    ``stream`` (a torch stream; default: the current one); outputs are allocated
    on that stream unless given, and the tensors of a call may be dropped while it
    is under way there (what it reads has to be written before: order the streams).
    Attention calls of one step share its workspace: keep them on one stream, or
    order them. A step is used by one host thread at a time. A graph that captured
    its calls reads its workspace: keep the step as long as the graph.

    There is no backward pass: where an input requires a gradient (and grad mode is on),
    the output does too, and a backward pass through it raises NotImplementedError. So does
    a call with a dual tensor of forward-mode differentiation."""

    def __init__(self, n_new, kv_len, blocks, *, heads, kv_heads, head_dim, block_tokens,
                 n_blocks, prefix_first=None, prefix_len=None, prefix_blocks=None, causal=True,
                 device="cuda"):
        self.ctx = None
        self._lib = lib()
        self._args = ctypes.create_string_buffer(_APPEND_FP4.size)  # the longest
        self._args_p = ctypes.addressof(self._args)
        b, keep = make_batch(n_new, kv_len, blocks, heads=heads, kv_heads=kv_heads,
                             head_dim=head_dim, block_tokens=block_tokens, n_blocks=n_blocks,
                             prefix_first=prefix_first, prefix_len=prefix_len,
                             prefix_blocks=prefix_blocks, causal=causal)
        self.ctx = tas_step_create(b)
        self.tokens = tas_step_tokens(self.ctx)
        self.ws_bytes = tas_step_bytes(self.ctx)
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.index = self.device.index
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.q_shape = (self.tokens, heads, head_dim)
        self.qkv_shape = (self.tokens, heads + 2 * kv_heads, head_dim)
        self.cache_shape = (n_blocks, kv_heads, block_tokens, head_dim)
        self.codes_shape = (n_blocks, kv_heads, block_tokens, head_dim // 2)
        self.scales_shape = (n_blocks, kv_heads, block_tokens, head_dim // 32)
        with torch.cuda.device(self.device):
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("a step is made outside of a graph's capture")
            # The plan goes through pinned memory (which torch keeps until it is copied)
            # without waiting: planning the next batch does not wait for the layers of this.
            n = ctypes.c_size_t()
            _check(self._lib.tas_step_plan(self.ctx, None, 0, ctypes.byref(n)), "tas_step_plan")
            plan = torch.empty(n.value, dtype=torch.uint8, pin_memory=True)
            _check(self._lib.tas_step_plan(self.ctx, plan.data_ptr(), n.value, ctypes.byref(n)),
                   "tas_step_plan")
            self._home = torch._C._cuda_getCurrentRawStream(self.index)
            self.ws = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=self.device)
            at = -self.ws.data_ptr() % 256
            self.ws[at:at + n.value].copy_(plan, non_blocking=True)
            self._copied = torch.cuda.Event()
            self._copied.record()
        tas_step_attach(self.ctx, self.ws.data_ptr() + at, self.ws_bytes)
        self._there = False  # the plan, as far as the host knows
        self._streams = {self._home}  # that the workspace is recorded on

    # ------------------------------------------------------------ argument checks

    def _rows(self, t, shape, dtype, what):
        """Address and token stride of a [tokens, heads, head_dim] tensor."""
        if t.dtype != dtype or t.get_device() != self.index or t.shape != shape:
            raise ValueError(f"{what} is {t.dtype} {tuple(t.shape)} on {t.device}, expected "
                             f"{dtype} {shape} on {self.device}")
        s0, s1, s2 = t.stride()
        if s2 != 1 or (s1 != self.head_dim and shape[1] > 1):
            raise ValueError(f"{what}: the heads of a token have to be adjacent, strides "
                             f"{t.stride()}")
        # one token: its stride says nothing
        return t.data_ptr(), s0 if self.tokens > 1 else shape[1] * self.head_dim

    def _cache(self, k, v, dtype):
        if k.dtype != dtype or v.dtype != dtype or k.get_device() != self.index \
                or v.get_device() != self.index or k.shape != self.cache_shape \
                or v.shape != self.cache_shape:
            raise ValueError(
                f"caches are {k.dtype} {tuple(k.shape)} on {k.device} and {v.dtype} "
                f"{tuple(v.shape)} on {v.device}, expected {dtype} {self.cache_shape} on "
                f"{self.device}")
        k0, k1, k2, k3 = k.stride()
        v0, v1, v2, v3 = v.stride()
        if k3 != 1 or v3 != 1:
            raise ValueError(f"caches: head_dim is not the fastest, strides {k.stride()} and "
                             f"{v.stride()}")
        return k.data_ptr(), v.data_ptr(), k0, k1, k2, v0, v1, v2

    def _cache_fp4(self, cache):
        codes, scales, index, byte = self.codes_shape, self.scales_shape, self.index, torch.uint8
        got = []
        for t, shape in ((cache.k, codes), (cache.v, codes), (cache.k_scale, scales),
                         (cache.v_scale, scales)):
            stride = t.stride()
            if t.shape != shape or stride[3] != 1 or t.dtype != byte or t.get_device() != index:
                raise ValueError(f"the cache holds {t.dtype} {tuple(t.shape)}, strides "
                                 f"{stride}, on {t.device}, expected adjacent uint8 {shape} "
                                 f"on {self.device}")
            got += t.data_ptr(), *stride[:3]
        return got

    def _dtype(self, t, what):
        code = DTYPES.get(t.dtype)
        if code is None:
            raise ValueError(f"{what} is {t.dtype}: float16 or bfloat16")
        return code

    def _turn(self, dtype, cos, sin, q_weight, k_weight):
        """rot_dim, the addresses of the weights and angles, and their positions."""
        rot = positions = cos_p = sin_p = qw_p = kw_p = 0
        if (cos is None) != (sin is None):
            raise ValueError("cos and sin: both or neither")
        if cos is not None:
            shape = cos.shape
            if len(shape) != 2 or sin.shape != shape or cos.dtype != torch.float32 \
                    or sin.dtype != torch.float32 or cos.get_device() != self.index \
                    or sin.get_device() != self.index or not cos.is_contiguous() \
                    or not sin.is_contiguous():
                raise ValueError("cos and sin: contiguous float32 [positions, rot_dim / 2] "
                                 f"on {self.device}")
            positions, rot = shape[0], 2 * shape[1]
            cos_p, sin_p = cos.data_ptr(), sin.data_ptr()
        if (q_weight is None) != (k_weight is None):
            raise ValueError("q_weight and k_weight: both or neither")
        if q_weight is not None:
            for t in (q_weight, k_weight):
                if t.dtype != dtype or t.get_device() != self.index \
                        or t.shape != self.q_shape[2:] or not t.is_contiguous():
                    raise ValueError(f"weights: contiguous {dtype} [{self.head_dim}] on "
                                     f"{self.device}")
            qw_p, kw_p = q_weight.data_ptr(), k_weight.data_ptr()
        return rot, qw_p, kw_p, cos_p, sin_p, positions

    def _lse(self, lse):
        if lse.dtype != torch.float32 or lse.get_device() != self.index \
                or lse.shape != self.q_shape[:2] or not lse.is_contiguous():
            raise ValueError(f"lse: contiguous float32 {(self.tokens, self.heads)} on "
                             f"{self.device}")
        return lse.data_ptr()

    def _out(self, out, like, stream):
        """The output, its address and its token stride."""
        if out is not None:
            return (out, *self._rows(out, self.q_shape, like.dtype, "out"))
        if stream is None:
            out = like.new_empty(self.q_shape)
        else:
            with torch.cuda.stream(stream):
                out = like.new_empty(self.q_shape)
        return out, out.data_ptr(), self.heads * self.head_dim

    def _keep(self, stream, *tensors):
        """The memory of tensors used on another stream than the current one is not given
        away before the work there is done."""
        if stream.cuda_stream != torch._C._cuda_getCurrentRawStream(self.index):
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)

    def _no_backward(self, out, *inputs):
        for t in inputs:
            if t is not None and t.requires_grad and torch.is_grad_enabled():
                return _NoBackward.apply(out, *inputs)
        return out

    def _enqueue(self, call, stream):
        if self.ctx is None:
            raise ValueError("the step is closed")
        if stream is None:
            raw = torch._C._cuda_getCurrentRawStream(self.index)
        else:
            raw = stream.cuda_stream
        if not self._there or raw not in self._streams:
            self._admit(raw, stream)
        if torch._C._cuda_getDevice() == self.index:
            rc = call(self.ctx, self._args_p, raw)
        else:
            with torch.cuda.device(self.device):
                rc = call(self.ctx, self._args_p, raw)
        if rc != TAS_OK:
            raise TasError(rc, call.__name__)

    def _admit(self, raw, stream):
        """Orders a call's stream behind the plan's copy, and the end of the workspace behind
        the stream."""
        on = torch.cuda.current_stream(self.device) if stream is None else stream
        self._there = self._there or self._copied.query()
        if not self._there:
            with torch.cuda.stream(on):
                capturing = torch.cuda.is_current_stream_capturing()
            if capturing:  # its replays would not wait for the copy
                raise ValueError("the step's plan is still under way to the device: synchronize "
                                 "before the capture")
            if raw != self._home:
                on.wait_event(self._copied)
        if raw not in self._streams:
            self.ws.record_stream(on)
            self._streams.add(raw)

    # ------------------------------------------------------------ the operators

    def append(self, qkv, k_cache, v_cache, cos=None, sin=None, *, q_weight=None, k_weight=None,
               eps=1e-6, interleaved=False, out=None, stream=None):
        """Norm (with weights), rotate (with angles) and append the new tokens.

        ``qkv``: [tokens, heads + 2 kv_heads, head_dim], queries, keys, values.
        ``cos``, ``sin``: float32 [positions, rot_dim / 2], rot_dim a multiple of
        16; None: no rotation. ``q_weight``, ``k_weight``: [head_dim], or both
        None. Keys and values go to the caches; returns the queries."""
        _no_tangent(qkv, k_cache, v_cache, cos, sin, q_weight, k_weight, out)
        dtype = self._dtype(qkv, "qkv")
        qkv_p, qkv_s = self._rows(qkv, self.qkv_shape, qkv.dtype, "qkv")
        cache = self._cache(k_cache, v_cache, qkv.dtype)
        turn = self._turn(qkv.dtype, cos, sin, q_weight, k_weight)
        out, out_p, out_s = self._out(out, qkv, stream)
        _APPEND.pack_into(self._args, 0, dtype, turn[0], 1 if interleaved else 0, eps, qkv_p,
                          qkv_s, out_p, out_s, *turn[1:], *cache)
        self._enqueue(self._lib.tas_step_append, stream)
        if stream is not None:
            self._keep(stream, qkv, k_cache, v_cache, cos, sin, q_weight, k_weight, out)
        return self._no_backward(out, qkv, q_weight, k_weight, cos, sin)

    def attention(self, q, k_cache, v_cache, *, scale=None, out=None, lse=None, stream=None):
        """softmax(scale q K^T) V of every new token and head over its request's
        prefix and context. ``scale``: default 1 / sqrt(head_dim). ``lse``: a
        float32 [tokens, heads] to receive the log of the sum of the exponentials.
        ``out`` may be ``q``. Returns [tokens, heads, head_dim]."""
        _no_tangent(q, k_cache, v_cache, out, lse)
        dtype = self._dtype(q, "q")
        q_p, q_s = self._rows(q, self.q_shape, q.dtype, "q")
        cache = self._cache(k_cache, v_cache, q.dtype)
        out, out_p, out_s = self._out(out, q, stream)
        lse_p = 0 if lse is None else self._lse(lse)
        if scale is None:
            scale = self.head_dim ** -0.5
        _ATTENTION.pack_into(self._args, 0, dtype, scale, q_p, q_s, out_p, out_s, lse_p, *cache)
        self._enqueue(self._lib.tas_step_attention, stream)
        if stream is not None:
            self._keep(stream, q, k_cache, v_cache, lse, out)
        return self._no_backward(out, q, k_cache, v_cache)

    def append_fp4(self, qkv, cache, cos=None, sin=None, *, q_weight=None, k_weight=None,
                   eps=1e-6, interleaved=False, out=None, stream=None):
        """``append`` to a cache in four bits (``fp4.Cache``): keys and values are
        rounded to it. Returns the queries."""
        _no_tangent(qkv, cos, sin, q_weight, k_weight, out)
        dtype = self._dtype(qkv, "qkv")
        qkv_p, qkv_s = self._rows(qkv, self.qkv_shape, qkv.dtype, "qkv")
        tensors = self._cache_fp4(cache)
        turn = self._turn(qkv.dtype, cos, sin, q_weight, k_weight)
        out, out_p, out_s = self._out(out, qkv, stream)
        _APPEND_FP4.pack_into(self._args, 0, dtype, turn[0], 1 if interleaved else 0, eps, qkv_p,
                              qkv_s, out_p, out_s, *turn[1:], *tensors)
        self._enqueue(self._lib.tas_fp4_append, stream)
        if stream is not None:
            self._keep(stream, qkv, *cache, cos, sin, q_weight, k_weight, out)
        return self._no_backward(out, qkv, q_weight, k_weight, cos, sin)

    def attention_fp4(self, q, cache, *, scale=None, out=None, lse=None, stream=None):
        """``attention`` over a cache in four bits (``fp4.Cache``)."""
        _no_tangent(q, out, lse)
        dtype = self._dtype(q, "q")
        q_p, q_s = self._rows(q, self.q_shape, q.dtype, "q")
        tensors = self._cache_fp4(cache)
        out, out_p, out_s = self._out(out, q, stream)
        lse_p = 0 if lse is None else self._lse(lse)
        if scale is None:
            scale = self.head_dim ** -0.5
        _ATTENTION_FP4.pack_into(self._args, 0, dtype, scale, q_p, q_s, out_p, out_s, lse_p,
                                 *tensors)
        self._enqueue(self._lib.tas_fp4_attention, stream)
        if stream is not None:
            self._keep(stream, q, *cache, lse, out)
        return self._no_backward(out, q)

    def close(self):
        if getattr(self, "ctx", None):
            tas_step_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

"""ctypes binding of the C ABI in include/tas_fp4.h: a serving iteration in four bits.

Elements are a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, times the power of two that 32
adjacent ones share. ``pack`` rounds a tensor to that form (codes of two elements a byte,
a byte of scale for 32), ``values`` gives back what it stands for. ``Cache`` is a layer's
paged KV cache in it, for ``step.Step.append_fp4`` and ``attention_fp4``; ``Weights`` a
matrix, for ``linear``:

    step = Step(n_new, kv_len, blocks, heads=32, kv_heads=8, head_dim=128,
                block_tokens=16, n_blocks=8192)
    for layer in layers:
        qkv = fp4.linear(x, layer.qkv).view(-1, 48, 128)
        q = step.append_fp4(qkv, layer.cache, cos, sin)
        o = step.attention_fp4(q, layer.cache)
        x = fp4.linear(o.flatten(1), layer.out)

Every operator runs in the HIP kernels of ``libtas_step.so``: no fallback. Calls are
enqueued on ``stream`` (a torch stream; default: the current one of the tensors' device),
outputs are allocated there, and the tensors of a call may be dropped while it is under way.
There is no backward pass: one through an output of inputs that require a gradient raises
NotImplementedError, and so does a call with a dual tensor of forward-mode differentiation.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple

import torch

from .step import DTYPES, _NoBackward, _no_tangent, lib
from .tas import TAS_OK, TasError

_P, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
BLOCK = 32  # elements with one scale


class tas_rows(ctypes.Structure):
    _fields_ = [("p", _P), ("stride", _i64 * 3)]


class tas_cache_fp4(ctypes.Structure):
    _fields_ = [("k", tas_rows), ("v", tas_rows), ("k_scale", tas_rows), ("v_scale", tas_rows)]


class tas_append_fp4(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("rot_dim", _i32), ("interleaved", _i32),
                ("eps", ctypes.c_float), ("qkv", _P), ("qkv_stride", _i64), ("q_out", _P),
                ("q_out_stride", _i64), ("q_weight", _P), ("k_weight", _P), ("cos", _P),
                ("sin", _P), ("positions", _i64), ("cache", tas_cache_fp4)]


class tas_attention_fp4(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("scale", ctypes.c_float), ("q", _P), ("q_stride", _i64),
                ("out", _P), ("out_stride", _i64), ("lse", _P), ("cache", tas_cache_fp4)]


class tas_tensor_fp4(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("reserved", _i32), ("n", _i64 * 3), ("cols", _i64),
                ("x", tas_rows), ("codes", tas_rows), ("scales", tas_rows)]


class tas_cache_values_fp4(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("head_dim", _i32), ("n_blocks", _i64), ("kv_heads", _i64),
                ("block_tokens", _i64), ("cache", tas_cache_fp4), ("k", _P), ("v", _P)]


class tas_linear_fp4(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("reserved", _i32), ("tokens", _i64), ("rows", _i64),
                ("cols", _i64), ("x", _P), ("x_stride", _i64), ("weights", _P), ("y", _P),
                ("y_stride", _i64)]


# Those of the calls below, packed (a third of the time of a ctypes constructor).
_TENSOR = struct.Struct("iiqqqq" + 3 * "Pqqq")
_CACHE_VALUES = struct.Struct("iiqqq" + 4 * "Pqqq" + "PP")
_LINEAR = struct.Struct("iiqqqPqPPq")
assert _TENSOR.size == ctypes.sizeof(tas_tensor_fp4)
assert _CACHE_VALUES.size == ctypes.sizeof(tas_cache_values_fp4)
assert _LINEAR.size == ctypes.sizeof(tas_linear_fp4)

EXPORTS = ["tas_fp4_append", "tas_fp4_attention", "tas_fp4_pack", "tas_fp4_values",
           "tas_fp4_cache_values", "tas_fp4_weights_bytes", "tas_fp4_weights", "tas_fp4_linear",
           "tas_fp4_linear_kernel"]
LINEAR_KERNELS = 14


def _call(index, stream, call, *args):
    """Enqueues on a device's stream."""
    raw = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == index:
        rc = call(*args, raw)
    else:
        with torch.cuda.device(index):
            rc = call(*args, raw)
    if rc != TAS_OK:
        raise TasError(rc, call.__name__)


def _keep(index, stream, *tensors):
    """The memory of tensors used on another stream than the current one is not given away
    before the work there is done."""
    if stream.cuda_stream != torch._C._cuda_getCurrentRawStream(index):
        for t in tensors:
            t.record_stream(stream)


def _empty(like, shape, dtype, stream):
    """A new tensor on the device of another, for the stream's use."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _no_backward(out, x):
    if x.requires_grad and torch.is_grad_enabled():
        return _NoBackward.apply(out, x)
    return out


def _gpu(t, what):
    if t.device.type != "cuda":
        raise ValueError(f"{what} is on {t.device}: a GPU's memory")
    return t.get_device()


def _rows(t, size, what):
    """(sizes of three leading dimensions, row's length, address and strides in bytes) of a
    tensor of elements of ``size`` bytes."""
    shape, stride = t.shape, t.stride()
    d = len(shape)
    if not 1 <= d <= 4:
        raise ValueError(f"{what} has {d} dimensions: one to four")
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{what}: the elements of a row have to be adjacent, strides {stride}")
    if d < 4:
        shape, stride = (1,) * (4 - d) + tuple(shape), (0,) * (4 - d) + stride
    a, b, c, cols = shape
    return (a, b, c), cols, (t.data_ptr(), size * stride[0], size * stride[1], size * stride[2])


def _adjacent(t, n, row):
    """Address and strides of a new tensor of n rows of so many bytes."""
    return t.data_ptr(), row * n[1] * n[2], row * n[2], row


def pack(x, *, stream=None):
    """(codes [..., n / 2], scales [..., n / 32]), uint8, of a float16 or bfloat16 tensor
    [..., n] of one to four dimensions, elements of a row adjacent, rows 16-byte aligned."""
    _no_tangent(x)
    dtype = DTYPES.get(x.dtype)
    if dtype is None:
        raise ValueError(f"x is {x.dtype}: float16 or bfloat16")
    if x.requires_grad and torch.is_grad_enabled():
        raise NotImplementedError("rounding to four bits has no gradient: detach x")
    index = _gpu(x, "x")
    n, cols, at = _rows(x, 2, "x")
    if cols % BLOCK or not cols:
        raise ValueError(f"rows of {cols} elements: a multiple of {BLOCK}")
    lead = x.shape[:-1]
    codes = _empty(x, (*lead, cols // 2), torch.uint8, stream)
    scales = _empty(x, (*lead, cols // BLOCK), torch.uint8, stream)
    args = _TENSOR.pack(dtype, 0, *n, cols, *at, *_adjacent(codes, n, cols // 2),
                        *_adjacent(scales, n, cols // BLOCK))
    _call(index, stream, lib().tas_fp4_pack, args)
    if stream is not None:
        _keep(index, stream, x, codes, scales)
    return codes, scales


def values(codes, scales, dtype, *, stream=None):
    """What codes [..., n / 2] and scales [..., n / 32] (uint8, bytes of a row adjacent, rows
    of codes 4-byte aligned) stand for, [..., n] in float16 or bfloat16."""
    code = DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"{dtype}: float16 or bfloat16")
    index = _gpu(codes, "codes")
    n, half, at = _rows(codes, 1, "codes")
    scales_n, blocks, scales_at = _rows(scales, 1, "scales")
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or not half \
            or half != 16 * blocks or scales_n != n or codes.dim() != scales.dim() \
            or scales.get_device() != index:
        raise ValueError(f"codes are {codes.dtype} {tuple(codes.shape)} on {codes.device}, scales "
                         f"{scales.dtype} {tuple(scales.shape)} on {scales.device}: uint8, 16 "
                         "bytes of codes to one of scales")
    x = _empty(codes, (*codes.shape[:-1], 2 * half), dtype, stream)
    args = _TENSOR.pack(code, 0, *n, 2 * half, *_adjacent(x, n, 4 * half), *at, *scales_at)
    _call(index, stream, lib().tas_fp4_values, args)
    if stream is not None:
        _keep(index, stream, codes, scales, x)
    return x


class Cache(NamedTuple):
    """One layer's paged cache in four bits: ``k`` and ``v`` are the codes, uint8
    [n_blocks, kv_heads, block_tokens, head_dim / 2], ``k_scale`` and ``v_scale`` uint8
    [n_blocks, kv_heads, block_tokens, head_dim / 32]; any strides whose last is 1, rows of
    codes 16-byte aligned, of scales to their length."""

    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor

    @classmethod
    def zeros(cls, n_blocks, kv_heads, block_tokens, head_dim, device="cuda"):
        """A cache of zeros."""
        def z(row):
            return torch.zeros((n_blocks, kv_heads, block_tokens, row), dtype=torch.uint8,
                               device=device)
        return cls(z(head_dim // 2), z(head_dim // 2), z(head_dim // BLOCK), z(head_dim // BLOCK))

    def values(self, dtype, *, stream=None):
        """The keys and values that the pool stands for, [n_blocks, kv_heads,
        block_tokens, head_dim] in float16 or bfloat16."""
        code = DTYPES.get(dtype)
        if code is None:
            raise ValueError(f"{dtype}: float16 or bfloat16")
        index = _gpu(self.k, "k")
        codes = self.k.shape
        if len(codes) != 4 or codes[3] not in (32, 64):
            raise ValueError(f"k is {tuple(codes)}: four dimensions, rows of 32 or 64")
        *n, half = codes
        scales, at = (*n, half // 16), []
        for t, shape, name in ((self.k, codes, "k"), (self.v, codes, "v"),
                               (self.k_scale, scales, "k_scale"),
                               (self.v_scale, scales, "v_scale")):
            stride = t.stride()
            if t.shape != shape or stride[3] != 1 or t.dtype != torch.uint8 \
                    or t.get_device() != index:
                raise ValueError(f"{name} is {t.dtype} {tuple(t.shape)}, strides {stride}, on "
                                 f"{t.device}, expected adjacent uint8 {tuple(shape)} on "
                                 f"{self.k.device}")
            at += t.data_ptr(), *stride[:3]
        both = _empty(self.k, (2, *n, 2 * half), dtype, stream)
        k, v = both.unbind()
        _call(index, stream, lib().tas_fp4_cache_values,
              _CACHE_VALUES.pack(code, 2 * half, *n, *at, k.data_ptr(), v.data_ptr()))
        if stream is not None:
            _keep(index, stream, *self, both)
        return k, v


class Weights:
    """A matrix [rows, cols] in four bits, laid out for the products: made once from its
    codes [rows, cols / 2] and scales [rows, cols / 32] (as ``pack`` gives them; bytes of a
    row adjacent, rows of codes 16-byte aligned), on the current stream or ``stream``. Other streams' products wait for that. A graph that
    captured its products reads it: keep it as long as the graph."""

    def __init__(self, codes, scales, *, stream=None):
        index = _gpu(codes, "codes")
        if codes.dim() != 2 or codes.dtype != torch.uint8 or scales.dtype != torch.uint8 \
                or scales.get_device() != index \
                or scales.shape != (codes.shape[0], codes.shape[1] // 16) \
                or codes.shape[1] % 16 or codes.stride(1) != 1 \
                or (scales.stride(1) != 1 and scales.shape[1] > 1):
            raise ValueError(f"codes are {codes.dtype} {tuple(codes.shape)} on {codes.device}, "
                             f"scales {scales.dtype} {tuple(scales.shape)} on {scales.device}: "
                             "uint8 [rows, cols / 2] and [rows, cols / 32], rows adjacent")
        self.rows, self.cols = codes.shape[0], 2 * codes.shape[1]
        self.device, self.index = codes.device, index
        n_bytes = lib().tas_fp4_weights_bytes(self.rows, self.cols)
        if not n_bytes:
            raise ValueError(f"a matrix of {self.rows} x {self.cols}: sizes out of range")
        on = torch.cuda.current_stream(self.device) if stream is None else stream
        with torch.cuda.stream(on):
            if torch.cuda.is_current_stream_capturing():
                raise ValueError("weights are laid out outside of a graph's capture")
            self._data = torch.empty(n_bytes + 256, dtype=torch.uint8, device=self.device)
            self._at = self._data.data_ptr() + -self._data.data_ptr() % 256
            many = self.rows > 1
            _call(index, on, lib().tas_fp4_weights, self.rows, self.cols, codes.data_ptr(),
                  codes.stride(0) if many else 0, scales.data_ptr(),
                  scales.stride(0) if many else 0, self._at)
            self._laid = torch.cuda.Event()
            self._laid.record()
        if stream is not None:
            _keep(index, stream, codes, scales)
        self._home = on.cuda_stream
        self._there = False  # laid out, as far as the host knows
        self._streams = {self._home}  # that the memory is recorded on

    def _admit(self, raw, stream):
        """Orders a call's stream behind the layout, and the end of the memory behind the
        stream."""
        on = torch.cuda.current_stream(self.device) if stream is None else stream
        self._there = self._there or self._laid.query()
        if not self._there:
            with torch.cuda.stream(on):
                capturing = torch.cuda.is_current_stream_capturing()
            if capturing:  # its replays would not wait for the layout
                raise ValueError("the weights are still being laid out: synchronize before the "
                                 "capture")
            if raw != self._home:
                on.wait_event(self._laid)
        if raw not in self._streams:
            self._data.record_stream(on)
            self._streams.add(raw)


def linear(x, weights, *, out=None, stream=None):
    """x W^T of float16 or bfloat16 tokens [tokens, cols] (16-byte aligned, any stride that is
    a multiple of 8 up to 2^24) and ``Weights`` of [rows, cols]: [tokens, rows] of x's type. The
    products are summed in 32 bits, in an order that depends on the sizes alone."""
    _no_tangent(x, out)
    dtype, index, rows, cols = DTYPES.get(x.dtype), weights.index, weights.rows, weights.cols
    shape, stride = x.shape, x.stride()
    if dtype is None or len(shape) != 2 or x.get_device() != index or shape[1] != cols \
            or stride[1] != 1:
        raise ValueError(f"x is {x.dtype} {tuple(shape)}, strides {stride}, on {x.device}, "
                         f"expected float16 or bfloat16 [tokens, {cols}], rows adjacent, on "
                         f"{weights.device}")
    tokens = shape[0]
    if out is None:
        out = _empty(x, (tokens, rows), x.dtype, stream)
        out_stride = rows
    elif out.dtype != x.dtype or out.get_device() != index or out.shape != (tokens, rows) \
            or (out.stride(1) != 1 and rows > 1):
        raise ValueError(f"out is {out.dtype} {tuple(out.shape)}, strides {out.stride()}, on "
                         f"{out.device}, expected {x.dtype} {(tokens, rows)}, rows adjacent, on "
                         f"{weights.device}")
    else:  # one token: its stride says nothing
        out_stride = out.stride(0) if tokens > 1 else rows
    raw = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if not weights._there or raw not in weights._streams:
        weights._admit(raw, stream)
    args = _LINEAR.pack(dtype, 0, tokens, rows, cols, x.data_ptr(),
                        stride[0] if tokens > 1 else cols, weights._at, out.data_ptr(),
                        out_stride)
    _call(index, stream, lib().tas_fp4_linear, args)
    if stream is not None:
        _keep(index, stream, x, out)
    return _no_backward(out, x)

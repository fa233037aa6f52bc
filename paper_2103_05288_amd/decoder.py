"""Handles of the operators around a decoder's attention: rotary positions, a cache of keys and values in
pages, attention over it (the functions of the same names in include/disc.h, which says what they compute).

The handles check the tensors they are given (type, shape, strides, device) and marshal them; a call that
does not fit raises DiscError before anything runs.  Launches go to torch's current stream of the context's
device unless `stream` (a hipStream_t as a number) says otherwise.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Sequence

from . import binding
from .binding import DiscError

STORAGE_IDS = {"i8": 1, "e4m3": 2}
LAYOUT_IDS = {"half": 0, "interleaved": 1}

_torch = None
_TYPES = {}


def _types():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
        _TYPES.update({"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn})
    return _TYPES


def _refuse(message: str):
    raise DiscError(-1, message)


def _stream_of(device: int):
    """A function of the device that gives the hipStream_t of torch's current stream there (a context's device need not be
    torch's current one)."""
    if device < 0:
        return lambda d: 0
    # (not part of torch's public interface: a torch without it takes the public way)
    return getattr(_torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: _torch.cuda.current_stream(d).cuda_stream)


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                       original_length: int = 0, fast: float = 32.0, slow: float = 1.0):
    """Radians a position for the rotary_dim / 2 pairs, and the magnitude that goes with them: the arguments of
    Context.register_rotary.

    The pair j turns by base^(-2j / rotary_dim) a position.  `scaling`, for contexts `factor` times as long as the
    `original_length` a model was trained on:
      "linear"    positions are divided by the factor
      "base"      the base grows by factor^(R / (R - 2)), so that the slowest pair turns `factor` times slower and the
                  fastest as before
      "by_parts"  a pair that makes at least `fast` turns within the original length keeps its frequency, one that makes
                  at most `slow` is divided by the factor, in between is interpolated; magnitude 0.1 ln(factor) + 1
    """
    R = int(rotary_dim)
    if R < 2 or R % 2:
        _refuse(f"rotary_dim is even and at least 2 (got {rotary_dim})")
    if not (base > 0.0 and math.isfinite(base)):
        _refuse(f"base is positive (got {base})")
    if scaling is not None and not (factor >= 1.0 and math.isfinite(factor)):
        _refuse(f"factor is at least 1 (got {factor})")
    if scaling == "base":
        if R < 4:
            _refuse("scaling the base takes a rotary_dim of at least 4")
        base = base * factor ** (R / (R - 2.0))
    f = [base ** (-2.0 * j / R) for j in range(R // 2)]
    if scaling is None or scaling == "base":
        return f, 1.0
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "by_parts":
        if original_length < 1 or not fast > slow:
            _refuse("scaling by parts takes the original length, and fast > slow")
        out = []
        for x in f:
            turns = original_length * x / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - slow) / (fast - slow)))
            out.append(x * (keep + (1.0 - keep) / factor))
        return out, 0.1 * math.log(factor) + 1.0
    _refuse(f"scaling is None, 'linear', 'base' or 'by_parts' (got {scaling!r})")


class _Handle:
    def __init__(self, ctx, oid: int, dtype: str, head_dim: int):
        self.ctx, self.id, self.head_dim = ctx, oid, head_dim
        self._dtype = _types()[dtype]
        self._device = ctx.device
        self._stream = _stream_of(ctx.device)

    def _rows(self, t, what: str):
        """A tensor [rows, heads, head_dim] whose last axis is dense -> (rows, heads, row stride, head stride)."""
        if t.dtype is not self._dtype:
            _refuse(f"{what} is {t.dtype}, the operator was registered for {self._dtype}")
        if t.get_device() != self._device:
            _refuse(f"{what} is on {t.device}, the context on device {self._device}")
        if t.dim() != 3:
            _refuse(f"{what} has {t.dim()} axes, [rows, heads, head_dim] is wanted")
        rows, heads, d = t.shape
        if d != self.head_dim:
            _refuse(f"{what} has heads of {d} elements, the operator was registered for {self.head_dim}")
        a, b, c = t.stride()
        if c != 1:
            _refuse(f"{what}: the elements of a head are not next to each other")
        return rows, heads, a, b

    def _plain(self, t, what: str, dtypes, shape):
        """A dense tensor of one of the types and the shape."""
        if t.dtype not in dtypes:
            _refuse(f"{what} is {t.dtype}, {' or '.join(str(d) for d in dtypes)} is wanted")
        if t.get_device() != self._device:
            _refuse(f"{what} is on {t.device}, the context on device {self._device}")
        if tuple(t.shape) != shape or not t.is_contiguous():
            _refuse(f"{what} is {tuple(t.shape)} with strides {t.stride()}, dense {shape} is wanted")

    def _call(self, fn, dims, inputs, outputs, workspace, stream):
        rc = binding._pylaunch.launch(fn, self.ctx.h.value or 0, self.id, dims, inputs, outputs, workspace, 0, stream)
        if rc != 0:
            self.ctx._check(rc)


class RotaryHandle(_Handle):
    """Rotary positions (disc_rotary)."""

    def __init__(self, ctx, oid, dtype, head_dim):
        super().__init__(ctx, oid, dtype, head_dim)
        self._fn = C.cast(ctx.lib.disc_rotary, C.c_void_p).value
        self._i32, self._i64 = _torch.int32, _torch.int64

    def launch(self, positions, inputs: Sequence, outputs: Sequence, backward: bool = False, stream: Optional[int] = None):
        """Turns up to four tensors [tokens, heads, head_dim] (queries, keys) by the positions [tokens] of their tokens.
        An output may be its input (in place).  backward=True: the inputs are gradients of the results, the outputs
        those of the inputs."""
        stream = self._stream(self._device) if stream is None else stream
        quick = getattr(binding._pylaunch, "rotary", None)      # all of a call that fits, in C
        if quick is not None:
            rc = quick(self._fn, self.ctx.h.value or 0, self.id, self._dtype, self._device, self.head_dim, self._i32, self._i64, positions, inputs,
                       outputs, backward, stream)
            if rc is not None:
                return self.ctx._check(rc)
        if positions.dtype not in (self._i32, self._i64) or positions.dim() != 1 or not positions.is_contiguous():
            _refuse("positions is a dense int32 or int64 tensor [tokens]")
        if positions.get_device() != self._device:
            _refuse(f"positions is on {positions.device}, the context on device {self._device}")
        if len(inputs) != len(outputs):
            _refuse(f"{len(inputs)} inputs and {len(outputs)} outputs")
        tokens = positions.shape[0]
        dims = [tokens, positions.element_size(), 1 if backward else 0]
        for x, y in zip(inputs, outputs):
            n, heads, a, b = self._rows(x, "an input")
            m, also, c, d = self._rows(y, "an output")
            if n != tokens or m != tokens or heads != also:
                _refuse(f"an input of {n} x {heads} and an output of {m} x {also} rows at {tokens} positions")
            dims += (heads, a, b, c, d)
        self._call(self._fn, dims, [positions, *inputs], outputs, None, stream)


class CacheHandle(_Handle):
    """A cache of keys and values in pages (disc_cache_store, disc_cache_load, disc_cache_attend).

    `pages` of the calls: (k_pages, v_pages), dense [pages, kv_heads, page_size, head_dim] of the storage's type, and
    with 8-bit storage (k_pages, v_pages, k_scales, v_scales), the scales fp32 [pages, kv_heads, page_size]."""

    def __init__(self, ctx, oid, dtype, head_dim, storage):
        super().__init__(ctx, oid, dtype, head_dim)
        self.storage = storage
        self._scaled = storage in STORAGE_IDS
        self._stored = (_types()[storage] if self._scaled else self._dtype,)
        self._store = C.cast(ctx.lib.disc_cache_store, C.c_void_p).value
        self._load = C.cast(ctx.lib.disc_cache_load, C.c_void_p).value
        self._attend = C.cast(ctx.lib.disc_cache_attend, C.c_void_p).value
        self._i64, self._i32, self._f32 = (_torch.int64,), (_torch.int32,), (_torch.float32,)

    def _pages(self, pages):
        if len(pages) != (4 if self._scaled else 2):
            _refuse("pages is (k_pages, v_pages, k_scales, v_scales)" if self._scaled else "pages is (k_pages, v_pages)")
        shape = tuple(pages[0].shape)
        if len(shape) != 4 or shape[3] != self.head_dim:
            _refuse(f"k_pages is {shape}, [pages, kv_heads, page_size, {self.head_dim}] is wanted")
        self._plain(pages[0], "k_pages", self._stored, shape)
        self._plain(pages[1], "v_pages", self._stored, shape)
        if self._scaled:
            self._plain(pages[2], "k_scales", self._f32, shape[:3])
            self._plain(pages[3], "v_scales", self._f32, shape[:3])
        return shape

    def _rows_quickly(self, fn, store, slots, rows, pages, stream):
        quick = getattr(binding._pylaunch, "cache_rows", None)
        return None if quick is None else quick(fn, self.ctx.h.value or 0, self.id, self._dtype, self._device, self.head_dim, self._scaled,
                                                self._stored[0], self._i64[0], self._f32[0], store, slots, rows, pages, stream)

    def _slots(self, slots, rows, pages):
        count, kv_heads, page_size, _ = self._pages(pages)
        if len(rows) != 2:
            _refuse("rows are [keys, values]")
        n, heads, a, b = self._rows(rows[0], "keys")
        m, also, c, d = self._rows(rows[1], "values")
        if n != m or heads != also or heads != kv_heads:
            _refuse(f"keys of {n} x {heads} and values of {m} x {also} rows for pages of {kv_heads} heads")
        self._plain(slots, "slots", self._i64, (n,))
        return [n, heads, count, page_size, a, b, c, d]

    def store(self, rows: Sequence, slots, pages: Sequence, stream: Optional[int] = None):
        """Keys and values [tokens, kv_heads, head_dim] into the slots (int64, page * page_size + place; outside the pages,
        as -1: left out)."""
        stream = self._stream(self._device) if stream is None else stream
        rc = self._rows_quickly(self._store, True, slots, rows, pages, stream)
        if rc is not None:
            return self.ctx._check(rc)
        dims = self._slots(slots, rows, pages)
        self._call(self._store, dims, [slots, *rows], pages, None, stream)

    def load(self, slots, pages: Sequence, rows: Sequence, stream: Optional[int] = None):
        """The rows of the slots back into keys and values [tokens, kv_heads, head_dim] (outside the pages: zeros)."""
        stream = self._stream(self._device) if stream is None else stream
        rc = self._rows_quickly(self._load, False, slots, rows, pages, stream)
        if rc is not None:
            return self.ctx._check(rc)
        dims = self._slots(slots, rows, pages)
        self._call(self._load, dims, [slots, *pages], rows, None, stream)

    def workspace_bytes(self, batch: int, q_heads: int, kv_heads: int, longest: int, prefix_length: int = 0, page_size: int = 8) -> int:
        """Bytes of workspace that attend takes for up to `batch` sequences, a page table that holds up to `longest` tokens a
        sequence (table_width * page_size, whatever the lengths are) and a prefix of up to prefix_length.  What was asked for at
        the smallest page size (the default) serves every page size of tables that hold no more."""
        width = -(-int(longest) // page_size)
        dims = [batch, q_heads, kv_heads, 1, page_size, width, prefix_length, -(-int(prefix_length) // page_size), 0, 0, 0, 0]
        arr, n = self.ctx._dims(dims)
        out = C.c_size_t(0)
        self.ctx._check(self.ctx.lib.disc_cache_workspace_bytes(self.ctx.h, self.id, arr, n, C.byref(out)))
        return int(out.value)

    def attend(self, q, lengths, table, pages: Sequence, out, workspace=None, prefix_table=None, prefix_length: int = 0,
               stream: Optional[int] = None):
        """out[b] = attention of the query token q[b] ([batch, q_heads, head_dim]) over the shared prefix's tokens and the
        lengths[b] tokens in the pages table[b] (int32 [batch, width])."""
        stream = self._stream(self._device) if stream is None else stream
        quick = getattr(binding._pylaunch, "cache_attend", None)
        if quick is not None:
            rc = quick(self._attend, self.ctx.h.value or 0, self.id, self._dtype, self._device, self.head_dim, self._scaled, self._stored[0],
                       self._i32[0], self._f32[0], q, lengths, table, pages, out, workspace, prefix_table, prefix_length, stream)
            if rc is not None:
                return self.ctx._check(rc)
        count, kv_heads, page_size, _ = self._pages(pages)
        batch, heads, a, b = self._rows(q, "q")
        also, too, c, d = self._rows(out, "out")
        if batch != also or heads != too:
            _refuse(f"q of {batch} x {heads} and out of {also} x {too} rows")
        self._plain(lengths, "lengths", self._i32, (batch,))
        width = table.shape[1] if table.dim() == 2 else -1
        self._plain(table, "table", self._i32, (batch, width))
        inputs = [q, lengths, table, *pages]
        prefix_width = 0
        if prefix_length:
            if prefix_table is None or prefix_table.dim() != 1:
                _refuse("a prefix has a table [pages of the prefix]")
            prefix_width = prefix_table.shape[0]
            self._plain(prefix_table, "prefix_table", self._i32, (prefix_width,))
            inputs.append(prefix_table)
        if workspace is not None and workspace.get_device() != self._device:
            _refuse(f"the workspace is on {workspace.device}, the context on device {self._device}")
        if workspace is not None and not workspace.is_contiguous():
            _refuse(f"the workspace has strides {workspace.stride()}, a dense tensor is wanted")
        self._call(self._attend, [batch, heads, kv_heads, count, page_size, width, prefix_length, prefix_width, a, b, c, d], inputs, [out], workspace, stream)

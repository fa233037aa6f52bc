"""Handles of what a decoder's step runs around its attention: a norm into 8-bit rows and its gradient, products with
4-bit weights, the check of drafted tokens (the functions of the same names in include/disc.h, which says what they
compute).

The handles check the tensors they are given (type, shape, strides, device) and marshal them; a call that does not fit
raises DiscError before anything runs.  Launches go to torch's current stream of the context's device unless `stream` (a
hipStream_t as a number) says otherwise.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

from . import binding, decoder
from .binding import DiscError
from .decoder import _refuse, _stream_of, _types


class _Handle:
    def __init__(self, ctx, oid: int, dtype: str):
        self.ctx, self.id = ctx, oid
        self._dtype = _types()[dtype]
        self._device = ctx.device
        self._stream = _stream_of(ctx.device)
        torch = decoder._torch
        self._f32, self._i32, self._u8 = torch.float32, torch.int32, torch.uint8

    def _is(self, t, what: str, dtype):
        if t.dtype is not dtype:
            _refuse(f"{what} is {t.dtype}, {dtype} is wanted")
        if t.get_device() != self._device:
            _refuse(f"{what} is on {t.device}, the context on device {self._device}")

    def _rows(self, t, what: str, dtype, rows=None, width=None):
        """A tensor [rows, width] whose last axis is dense -> (rows, width, row stride)."""
        self._is(t, what, dtype)
        if t.dim() != 2:
            _refuse(f"{what} has {t.dim()} axes, [rows, width] is wanted")
        n, w = t.shape
        if (rows is not None and n != rows) or (width is not None and w != width):
            _refuse(f"{what} is {n} x {w}, {rows if rows is not None else n} x {width if width is not None else w} is wanted")
        a, b = t.stride()
        if b != 1 and w > 1:
            _refuse(f"{what}: the elements of a row are not next to each other")
        return n, w, a

    def _dense(self, t, what: str, dtype, shape):
        self._is(t, what, dtype)
        if tuple(t.shape) != shape or not t.is_contiguous():
            _refuse(f"{what} is {tuple(t.shape)} with strides {t.stride()}, dense {shape} is wanted")

    def _scratch(self, workspace):
        if workspace is not None and workspace.get_device() != self._device:
            _refuse(f"the workspace is on {workspace.device}, the context on device {self._device}")
        if workspace is not None and not workspace.is_contiguous():
            _refuse(f"the workspace has strides {workspace.stride()}, a dense tensor is wanted")

    def _bytes(self, fn, dims) -> int:
        arr, n = self.ctx._dims(dims)
        out = C.c_size_t(0)
        self.ctx._check(fn(self.ctx.h, self.id, arr, n, C.byref(out)))
        return int(out.value)

    def _quickly(self, name: str, fn, number, *rest) -> bool:
        """All of a call that fits, in C; False: through the checks here, which say why it does not."""
        quick = getattr(binding._pylaunch, name, None)
        rc = None if quick is None else quick(fn, self.ctx.h.value or 0, self.id, self._dtype, self._device, number, *rest)
        if rc:
            self.ctx._check(rc)
        return rc is not None

    def _call(self, fn, dims, inputs, outputs, workspace, stream):
        rc = binding._pylaunch.launch(fn, self.ctx.h.value or 0, self.id, dims, inputs, outputs, workspace, 0, stream)
        if rc != 0:
            self.ctx._check(rc)


class NormHandle(_Handle):
    """Root-mean-square norm into 8-bit rows (disc_norm, disc_norm_backward)."""

    def __init__(self, ctx, oid, dtype, storage):
        super().__init__(ctx, oid, dtype)
        self.storage = storage
        self._stored = _types()[storage]
        self._fn = C.cast(ctx.lib.disc_norm, C.c_void_p).value
        self._backward = C.cast(ctx.lib.disc_norm_backward, C.c_void_p).value

    def launch(self, x, weight, codes, scales, residual=None, total=None, stream: Optional[int] = None):
        """codes [rows, width] of the storage's type and scales (fp32 [rows]) of the norm of x [rows, width], or with a residual
        of x + residual, which total gets (it may be x or residual)."""
        stream = self._stream(self._device) if stream is None else stream
        if self._quickly("norm", self._fn, 0, self._stored, self._f32, x, weight, codes, scales, residual, total, stream):
            return
        rows, width, a = self._rows(x, "x", self._dtype)
        self._dense(weight, "weight", self._dtype, (width,))
        _, _, d = self._rows(codes, "codes", self._stored, rows, width)
        self._dense(scales, "scales", self._f32, (rows,))
        if (residual is None) != (total is None):
            _refuse("a residual goes with the total that it makes")
        if residual is None:
            self._call(self._fn, [rows, width, a, 0, 0, d], [x, weight], [codes, scales], None, stream)
            return
        _, _, b = self._rows(residual, "residual", self._dtype, rows, width)
        _, _, c = self._rows(total, "total", self._dtype, rows, width)
        self._call(self._fn, [rows, width, a, b, c, d], [x, weight, residual], [codes, scales, total], None, stream)

    def workspace_bytes(self, rows: int, width: int) -> int:
        """Bytes of workspace that backward takes for up to `rows` rows of this width."""
        return self._bytes(self.ctx.lib.disc_norm_workspace_bytes, [rows, width, 0, 0, 0, 0])

    def backward(self, total, weight, dy, dx, dweight, dtotal=None, workspace=None, stream: Optional[int] = None):
        """dx [rows, width], the gradient of x and of the residual, and dweight (fp32 [width], overwritten), from the rows that were
        normed (total; x where there was no residual), the gradient dy of the norm's result and that of total, dtotal.  dx may be
        total, dy or dtotal."""
        stream = self._stream(self._device) if stream is None else stream
        if self._quickly("norm_backward", self._backward, 0, self._f32, total, weight, dy, dx, dweight, dtotal, workspace, stream):
            return
        rows, width, a = self._rows(total, "total", self._dtype)
        self._dense(weight, "weight", self._dtype, (width,))
        _, _, b = self._rows(dy, "dy", self._dtype, rows, width)
        _, _, d = self._rows(dx, "dx", self._dtype, rows, width)
        self._dense(dweight, "dweight", self._f32, (width,))
        inputs, c = [total, weight, dy], 0
        if dtotal is not None:
            _, _, c = self._rows(dtotal, "dtotal", self._dtype, rows, width)
            inputs.append(dtotal)
        self._scratch(workspace)
        self._call(self._backward, [rows, width, a, b, c, d], inputs, [dx, dweight], workspace, stream)


class Linear4Handle(_Handle):
    """Products of few rows with 4-bit weights (disc_linear4)."""

    def __init__(self, ctx, oid, dtype, group, rows, zeros):
        super().__init__(ctx, oid, dtype)
        self.group, self.rows, self.zeros = group, rows, zeros
        self._scaled = rows in decoder.STORAGE_IDS
        self._row = _types()[rows] if self._scaled else self._dtype
        self._fn = C.cast(ctx.lib.disc_linear4, C.c_void_p).value

    def launch(self, x, weights, scales, out, row_scales=None, zeros=None, bias=None, stream: Optional[int] = None):
        """out [rows, n] = x [rows, k] times the weights (uint8 [n, k / 2], two elements a byte, the even one in the lower four
        bits), their scales [n, k / group] and zero points (uint8, of the same shape), plus bias [n].  8-bit rows come with
        row_scales (fp32 [rows])."""
        stream = self._stream(self._device) if stream is None else stream
        if self._quickly("linear4", self._fn, self.group, self._row, self._f32, self._u8, self._scaled, self.zeros, x, weights, scales, out, row_scales, zeros, bias, stream):
            return
        rows, k, a = self._rows(x, "x", self._row)
        if k % self.group:
            _refuse(f"x has rows of {k} elements, a multiple of the group, {self.group}, is wanted")
        if weights.dim() != 2:
            _refuse(f"weights has {weights.dim()} axes, [n, k / 2] is wanted")
        n = weights.shape[0]
        self._dense(weights, "weights", self._u8, (n, k // 2))
        self._dense(scales, "scales", self._dtype, (n, k // self.group))
        _, _, b = self._rows(out, "out", self._dtype, rows, n)
        inputs = [x, weights, scales]
        if self._scaled != (row_scales is not None):
            _refuse("8-bit rows come with row_scales" if self._scaled else "rows of the registered type have no row_scales")
        if self._scaled:
            self._dense(row_scales, "row_scales", self._f32, (rows,))
            inputs.append(row_scales)
        if self.zeros != (zeros is not None):
            _refuse("the product was registered with zero points" if self.zeros else "the product was registered without zero points")
        if self.zeros:
            self._dense(zeros, "zeros", self._u8, (n, k // self.group))
            inputs.append(zeros)
        if bias is not None:
            self._dense(bias, "bias", self._dtype, (n,))
            inputs.append(bias)
        self._call(self._fn, [rows, n, k, a, b], inputs, [out], None, stream)


class VerifyHandle(_Handle):
    """The check of drafted tokens against the target's probabilities (disc_verify)."""

    def __init__(self, ctx, oid, dtype):
        super().__init__(ctx, oid, dtype)
        self._fn = C.cast(ctx.lib.disc_verify, C.c_void_p).value

    def workspace_bytes(self, batch: int, vocabulary: int) -> int:
        """Bytes of workspace that launch takes for up to `batch` sequences and this vocabulary or a smaller one."""
        return self._bytes(self.ctx.lib.disc_verify_workspace_bytes, [batch, 0, vocabulary, 0, 0, 0, 0, 0, 0])

    def _probabilities(self, t, what: str):
        self._is(t, what, self._dtype)
        if t.dim() != 3:
            _refuse(f"{what} has {t.dim()} axes, [batch, places, vocabulary] is wanted")
        if t.stride(2) != 1 and t.shape[2] > 1:
            _refuse(f"{what}: the probabilities of a place are not next to each other")
        return tuple(t.shape), t.stride(0), t.stride(1)

    def launch(self, target, drafted, uniforms, tokens, accepted, draft=None, lengths=None, workspace=None, stream: Optional[int] = None):
        """tokens (int32 [batch, drafts + 1]: the kept ones, the one drawn behind them, then -1) and accepted (int32 [batch], how many
        were kept) of the drafted tokens (int32 [batch, drafts]), the target's probabilities [batch, drafts + 1, vocabulary], the draft's
        [batch, drafts, vocabulary] (None: it drew each for certain) and uniforms (fp32 [batch, drafts + 1] in [0, 1)).  lengths
        (int32 [batch]): how many of a sequence's drafted tokens there are."""
        stream = self._stream(self._device) if stream is None else stream
        if self._quickly("verify", self._fn, 0, self._f32, self._i32, target, drafted, uniforms, tokens, accepted, draft, lengths, workspace, stream):
            return
        (batch, places, vocabulary), a, b = self._probabilities(target, "target")
        drafts = places - 1
        if drafts < 0:
            _refuse("target has a place behind the drafted tokens")
        self._dense(drafted, "drafted", self._i32, (batch, drafts))
        self._dense(uniforms, "uniforms", self._f32, (batch, places))
        self._dense(tokens, "tokens", self._i32, (batch, places))
        self._dense(accepted, "accepted", self._i32, (batch,))
        inputs, c, d = [target, drafted, uniforms], 0, 0
        if draft is not None:
            shape, c, d = self._probabilities(draft, "draft")
            if shape != (batch, drafts, vocabulary):
                _refuse(f"draft is {shape}, {(batch, drafts, vocabulary)} is wanted")
            inputs.append(draft)
        if lengths is not None:
            self._dense(lengths, "lengths", self._i32, (batch,))
            inputs.append(lengths)
        self._scratch(workspace)
        self._call(self._fn, [batch, drafts, vocabulary, a, b, c, d, int(draft is not None), int(lengths is not None)], inputs, [tokens, accepted], workspace, stream)

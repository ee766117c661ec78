"""Operators of the training step around the aggregation, on torch tensors.

A data-parallel step makes the weight gradients, aggregates them (`cerar.Plan`) and applies them.  This module is
the two outer parts:

  Ops.quantize, Ops.matmul   products in 8-bit floating point with a scale per 128 values (cerar_fp8_quantize, cerar_fp8_matmul)
  linear, linear_backward, Linear8   a linear layer made of them; the weight gradient is added to a binary32 buffer of the
                             caller's (a slice of the vector that is aggregated)
  TensorSet.grad_norm        norm and clip coefficient of many gradients (cerar_grad_norm)
  TensorSet.adamw            AdamW over many tensors, states in 32 or 8 bits (cerar_adamw_step)

Everything runs on the current stream of the current device, without synchronisation.  The formulas, formats and rules
stand in include/cerar.h.
"""
from __future__ import annotations

import ctypes as C
import weakref

import torch
from torch.autograd.function import once_differentiable

from . import cerar
from .cerar import CerarError, Fp8Matrix, lib

BY_ROW, BY_COLUMN, BY_BLOCK = 0, 1, 2
BLOCK = 128            # values that share a scale of an 8-bit matrix
STATE_BLOCK = 256      # elements that share a scale of an 8-bit optimizer state

_TYPES = {torch.float32: 0, torch.bfloat16: 1}
_check = cerar._check
_E4M3, _F32 = torch.float8_e4m3fn, torch.float32
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # the same handle without the Stream object around it
_MATRIX_BYTES = C.sizeof(Fp8Matrix)
_LAYOUTS: dict = {}      # (rows, cols, scalings) -> where the parts of such matrices lie in one allocation
_quantize, _matmul, _norm, _adamw = lib.cerar_fp8_quantize, lib.cerar_fp8_matmul, lib.cerar_grad_norm, lib.cerar_adamw_step


def _stream(device: int | None = None) -> int:
    """The current stream of a device (of the current one)."""
    if _raw_stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(torch.cuda.current_device() if device is None else device)


def _type(t: torch.Tensor, what: str) -> int:
    if t.dtype not in _TYPES:
        raise TypeError(f"{what}: float32 or bfloat16 wanted, got {t.dtype}")
    return _TYPES[t.dtype]


def _matrix(t: torch.Tensor, what: str) -> torch.Tensor:
    """A two-dimensional device tensor whose rows are contiguous (an empty one may have any strides: there is nothing at them)."""
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{what}: a two-dimensional CUDA tensor is wanted")
    if not t.numel():
        return t
    if t.stride(1) != 1 and t.size(1) > 1 or t.stride(0) < t.size(1) and t.size(0) > 1:
        raise ValueError(f"{what}: elements of a row must be contiguous and rows must not overlap")
    return t


def _ld(t: torch.Tensor) -> int:
    """Elements between rows (a tensor of one row may carry any stride)."""
    return t.stride(0) if t.size(0) > 1 else max(t.stride(0), t.size(1))


class Quantized:
    """An 8-bit matrix: `codes` (rows x cols, float8_e4m3fn or uint8, rows a multiple of 16 bytes apart), `scales` (float32,
    [ceil(cols/128), rows] by row, [ceil(rows/128), cols] by column, [ceil(rows/128), ceil(cols/128)] by block).

    pow2: whether all scales are powers of two, as Ops.quantize makes them: products of two such matrices are faster.  None: the
    scales are read once, here, to see (which waits for the device).  Scales that are changed later have to keep to it:
    what they touch becomes NaN otherwise."""

    __slots__ = ("_codes", "_scales", "scaling", "desc", "at", "_buffer", "_parts")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, scaling: int, pow2: bool | None = None):
        if codes.element_size() != 1:
            raise TypeError("codes: float8_e4m3fn or uint8 wanted")
        _matrix(codes, "codes"), _matrix(scales, "scales")
        if scales.dtype != torch.float32 or scales.device != codes.device:
            raise TypeError("scales: float32 on the device of the codes wanted")
        rows, cols = codes.shape
        nr, nc = -(-rows // BLOCK), -(-cols // BLOCK)
        want = {BY_ROW: (nc, rows), BY_COLUMN: (nr, cols), BY_BLOCK: (nr, nc)}.get(scaling)
        if want is None:
            raise ValueError("scaling must be BY_ROW, BY_COLUMN or BY_BLOCK")
        if tuple(scales.shape) != want:
            raise ValueError(f"scales of shape {want} wanted, got {tuple(scales.shape)}")
        ld = codes.stride(0) if rows > 1 else -(-max(codes.stride(0), cols) // 16) * 16
        if pow2 is None:
            bits = scales.contiguous().view(torch.int32)
            pow2 = bool(((bits & 0x7FFFFF == 0) & (bits >= 1 << 23) & (bits < 255 << 23)).all())
        self._set(codes, scales, scaling, rows, cols, ld, _ld(scales), pow2)

    def _set(self, codes, scales, scaling, rows, cols, ld, lds, pow2):
        self._codes, self._scales, self.scaling, self._buffer = codes, scales, scaling, None
        self.desc = Fp8Matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, ld, lds, scaling, pow2)
        self.at = C.addressof(self.desc)

    def _saved(self):
        """(tensors to save for a backward pass, what _restored wants beside them, which holds no memory)."""
        tensors = (self._codes, self._scales) if self._buffer is None else (self._buffer, None)
        return tensors, (self.scaling, self.desc, None if self._buffer is None else self._parts)

    @classmethod
    def _restored(cls, first, second, rest):
        """The matrix of tensors that _saved gave: the same memory, or copies of it (from the host, packed)."""
        scaling, desc, parts = rest
        q = cls.__new__(cls)
        if second is None:
            base = first.data_ptr()
            if base + parts[0] != desc.codes:
                desc = Fp8Matrix(base + parts[0], base + parts[1], desc.rows, desc.cols, desc.ld, desc.lds, scaling, desc.pow2)
            q._codes = q._scales = None
            q.scaling, q.desc, q.at, q._buffer, q._parts = scaling, desc, C.addressof(desc), first, parts
            return q
        rows, cols = first.shape
        if first.data_ptr() == desc.codes and second.data_ptr() == desc.scales and (rows < 2 or first.stride(0) == desc.ld) and \
                (second.size(0) < 2 or second.stride(0) == desc.lds):
            q._codes, q._scales, q.scaling, q.desc, q.at, q._buffer = first, second, scaling, desc, C.addressof(desc), None
            return q
        if rows > 1 and (first.stride(0) & 15 or first.stride(1) != 1) or first.data_ptr() & 15:
            wide = torch.empty(rows, (cols + 15) & -16, dtype=first.dtype, device=first.device)
            first = wide[:, :cols].copy_(first)
        q._set(first, second, scaling, rows, cols, first.stride(0) if rows > 1 else (cols + 15) & -16, _ld(second), desc.pow2)
        return q

    @staticmethod
    def _sizes(rows, cols, scaling):
        """Bytes between rows of codes, and the shape of the scales."""
        ld, nr, nc = (cols + 15) & -16, (rows + 127) >> 7, (cols + 127) >> 7
        if scaling == BY_ROW:
            return ld, nc, rows
        if scaling == BY_COLUMN:
            return ld, nr, cols
        if scaling != BY_BLOCK:
            raise ValueError("scaling must be BY_ROW, BY_COLUMN or BY_BLOCK")
        return ld, nr, nc

    @classmethod
    def empty(cls, rows: int, cols: int, scaling: int, device) -> "Quantized":
        ld, nr, nc = cls._sizes(rows, cols, scaling)
        codes = torch.empty(rows, ld, dtype=_E4M3, device=device)
        q = cls.__new__(cls)
        q._set(codes if ld == cols else codes[:, :cols], torch.empty(nr, nc, dtype=_F32, device=device), scaling, rows, cols, ld, nc, True)
        return q

    @classmethod
    def _several(cls, rows, cols, scalings, device):
        """As many matrices in one allocation; their tensors are made when they are asked for.  Also the descriptors in a row."""
        layout = _LAYOUTS.get((rows, cols, scalings))
        if layout is None:
            layout = cls._layout(rows, cols, scalings)
        size, kind, template, offsets = layout
        arr = kind.from_buffer_copy(template)
        buffer = torch.empty(size, dtype=_E4M3, device=device)
        base, at = buffer.data_ptr(), C.addressof(arr)
        first, out = at, []
        for d, scaling, parts in zip(arr, scalings, offsets):
            d.codes, d.scales = base + parts[0], base + parts[1]
            q = cls.__new__(cls)
            q._codes = q._scales = None
            q.scaling, q.desc, q.at, q._buffer, q._parts = scaling, d, at, buffer, parts
            at += _MATRIX_BYTES
            out.append(q)
        return out, first

    @classmethod
    def _layout(cls, rows, cols, scalings):
        """Where codes and scales of these matrices lie in one allocation (and their shapes and strides), and their descriptors but
        for the addresses."""
        n = len(scalings)
        arr, offsets, size = (Fp8Matrix * n)(), [], 0
        for i, scaling in enumerate(scalings):
            ld, nr, nc = cls._sizes(rows, cols, scaling)
            at = size + ((rows * ld + 255) & -256)                   # the scales start there
            arr[i] = Fp8Matrix(0, 0, rows, cols, ld, nc, scaling, True)
            offsets.append((size, at, (rows, cols), (ld, 1), (nr, nc), (nc, 1)))
            size = (at + 4 * nr * nc + 255) & -256
        if len(_LAYOUTS) >= 1024:
            _LAYOUTS.clear()
        _LAYOUTS[rows, cols, scalings] = layout = (size, Fp8Matrix * n, bytes(arr), offsets)
        return layout

    @property
    def codes(self) -> torch.Tensor:
        if self._codes is None:
            p = self._parts
            self._codes = self._buffer.as_strided(p[2], p[3], p[0])
        return self._codes

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            p = self._parts
            self._scales = self._buffer.view(_F32).as_strided(p[4], p[5], p[1] >> 2)
        return self._scales

    @property
    def device(self) -> torch.device:
        return (self._codes if self._buffer is None else self._buffer).device

    @property
    def shape(self):
        return torch.Size((self.desc.rows, self.desc.cols))

    def dequantize(self) -> torch.Tensor:
        """The values in float32 (for inspection; torch operations)."""
        r, c = self.codes.shape
        s = self.scales.t() if self.scaling == BY_ROW else self.scales
        if self.scaling != BY_ROW:
            s = s.repeat_interleave(BLOCK, 0)[:r]
        if self.scaling != BY_COLUMN:
            s = s.repeat_interleave(BLOCK, 1)[:, :c]
        return self.codes.view(torch.float8_e4m3fn).float() * s


class Ops:
    """Owns a cerar_ops_t of the current device."""

    def __init__(self):
        out = C.c_void_p()
        _check(lib.cerar_ops_create(C.byref(out)))
        self._h = out
        self._index = torch.cuda.current_device()
        self._sets = weakref.WeakSet()

    def destroy(self):
        """Also destroys the sets that were made with it: they hold its address."""
        if self._h:
            for s in list(self._sets):
                s.destroy()
            lib.cerar_ops_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _here(self, device):
        if device.index != self._index:
            raise ValueError(f"a tensor on {device}, but these operators were made on cuda:{self._index}")

    def status(self):
        """Waits for the current stream; raises if a kernel gave up on a bounded wait."""
        _check(lib.cerar_ops_status(self._h, _stream()))

    def launch_count(self) -> int:
        return lib.cerar_ops_launch_count(self._h)

    def quantize(self, x: torch.Tensor, *scalings: int):
        """8-bit matrices of x, one for each of `scalings` (BY_ROW, BY_COLUMN, BY_BLOCK), from one reading of x."""
        t = _TYPES.get(x.dtype)
        shape, strides = x.shape, x.stride()
        if t is None or len(shape) != 2 or not x.is_cuda or strides[1] != 1 or strides[0] < shape[1]:
            t = _type(x, "x")                                       # the whole check, where the short one is not enough
            _matrix(x, "x")
        rows, cols = shape
        device = x.device
        if device.index != self._index:
            self._here(device)
        if len(scalings) == 1 and not cols & 15:                    # two allocations cost the host less than two views of one
            out = [Quantized.empty(rows, cols, scalings[0], device)]
            at = out[0].at
        else:
            out, at = Quantized._several(rows, cols, scalings, device)
        st = _quantize(self._h, x.data_ptr(), t, strides[0] if rows > 1 else max(strides[0], cols), at, len(out), _stream(device.index))
        if st:
            _check(st)
        return out

    def matmul(self, a: Quantized, b: Quantized, *, trans_a=False, trans_b=False, out: torch.Tensor | None = None,
               dtype: torch.dtype = torch.bfloat16, accumulate=False) -> torch.Tensor:
        """op(a) op(b), into `out` if given (added to it with accumulate)."""
        da, db = a.desc, b.desc
        m, n = (da.cols if trans_a else da.rows), (db.rows if trans_b else db.cols)
        device = a.device
        self._here(device)
        if b.device != device:
            raise ValueError("the operands are on different devices")
        if out is None:
            if accumulate:
                raise ValueError("accumulate wants an `out` to add to")
            out = torch.empty(m, n, dtype=dtype, device=device)
            ld = n
        else:
            _matrix(out, "out")
            self._here(out.device)
            if tuple(out.shape) != (m, n):
                raise ValueError(f"out of shape {(m, n)} wanted, got {tuple(out.shape)}")
            ld = _ld(out)
        st = _matmul(self._h, a.at, trans_a, b.at, trans_b, out.data_ptr(), _type(out, "out"), ld, accumulate, _stream(device.index))
        if st:
            _check(st)
        return out


# ------------------------------------------------------------------------------------------------ a linear layer


def linear(ops: Ops, x: torch.Tensor, w: Quantized):
    """y = x w^T for x (tokens x inputs) and weights quantized by block.  Returns (y, what linear_backward wants of x)."""
    xr, xc = ops.quantize(x, BY_ROW, BY_COLUMN)
    return ops.matmul(xr, w, trans_b=True, dtype=x.dtype), xc


def linear_backward(ops: Ops, dy: torch.Tensor, xc: Quantized, w: Quantized, dw: torch.Tensor | None, *, accumulate=True, need_dx=True):
    """dx = dy w, and dw (outputs x inputs, float32 or bfloat16, e.g. a slice of the gradient vector) += dy^T x."""
    if dw is None:
        dr, = ops.quantize(dy, BY_ROW)
    elif need_dx:
        dr, dc = ops.quantize(dy, BY_ROW, BY_COLUMN)
    else:
        dc, = ops.quantize(dy, BY_COLUMN)
    if dw is not None:
        ops.matmul(dc, xc, trans_a=True, out=dw, accumulate=accumulate)
    return ops.matmul(dr, w, dtype=dy.dtype) if need_dx else None


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t (..., columns) as a matrix whose rows the conversion can read: a copy where a row's elements are not contiguous or rows overlap
    (transposed inputs, gradients that autograd expands from one element)."""
    if t.dim() != 2:
        t = t.unsqueeze(0) if t.dim() == 1 else t.flatten(0, -2)
    (rows, cols), (row, col) = t.shape, t.stride()
    return t.contiguous() if col != 1 and cols > 1 or row < cols and rows > 1 else t


class Linear8(torch.autograd.Function):
    """linear and linear_backward for torch.autograd: y = Linear8.apply(x, w, ops, dw), x (..., inputs) with any strides.  w: quantized
    weights (no gradient of their own: it is added to `dw`, which may be None).  y has a gradient wherever x or dw wants one, so `dw` is
    served too where x is data or comes from frozen layers.  Every pass backward through the layer adds to dw, torch.autograd.grad's
    too; second derivatives are refused."""

    @classmethod
    def apply(cls, x, w, ops, dw):
        # Neither w nor dw is a tensor that autograd follows.  Where x is not one either, an empty one takes that place: without it y
        # would have no gradient and backward would not be called.  It lies on x's device, so that the stream dw is written on
        # is among those that the end of the backward pass waits for.
        anchor = None
        if dw is not None and not x.requires_grad and torch.is_grad_enabled():
            anchor = torch.empty(0, device=x.device, requires_grad=True)
        return super().apply(x, w, ops, dw, anchor)

    @staticmethod
    def forward(ctx, x, w, ops, dw, anchor):
        y, xc = linear(ops, _rows(x), w)
        # Saved as autograd saves tensors: freed by the backward pass, within reach of saved-tensor hooks, and refused if changed in between.
        # (Weights made in inference mode cannot be saved; they are held as they are.)
        ctx.ops, ctx.dw, ctx.x_rest, ctx.w_rest, ctx.w = ops, dw, None, None, None
        xs = ws = (None, None)
        if dw is not None:
            xs, ctx.x_rest = xc._saved()
        if ctx.needs_input_grad[0]:
            ws, ctx.w_rest = w._saved()
            if any(t is not None and t.is_inference() for t in ws):
                ws, ctx.w_rest, ctx.w = (None, None), None, w
        ctx.save_for_backward(*xs, *ws)
        return y.view(*x.shape[:-1], y.shape[-1])

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        saved = ctx.saved_tensors
        xc = None if ctx.x_rest is None else Quantized._restored(saved[0], saved[1], ctx.x_rest)
        w = ctx.w if ctx.w_rest is None else Quantized._restored(saved[2], saved[3], ctx.w_rest)
        dx = linear_backward(ctx.ops, _rows(dy), xc, w, ctx.dw, need_dx=ctx.needs_input_grad[0])
        return None if dx is None else dx.view(*dy.shape[:-1], dx.shape[-1]), None, None, None, None


# ------------------------------------------------------------------------------------------------ norm and optimizer


def _flat(tensors, what, n=None, device=None):
    tensors = list(tensors)
    for t in tensors:
        if not t.is_cuda or not t.is_contiguous() or (device is not None and t.device != device):
            raise ValueError(f"{what}: contiguous tensors on one CUDA device are wanted")
    if n is not None and [t.numel() for t in tensors] != n:
        raise ValueError(f"{what}: the sizes differ from the gradients'")
    return tensors


class TensorSet:
    """Parameters, gradients and optimizer states of a step (cerar_tensors_t).

    grads              tensors of float32 or bfloat16, e.g. views into the aggregated vector
    params, masters    the parameters (float32 or bfloat16), and for bfloat16 ones optional float32 copies (None where one has none)
    state_bits         32 or 8; with no params the set serves grad_norm only
    m, v               states of all tensors in one flat tensor each (zeros are made where none are given), tensor i at
                       state_offsets[i]: float32 of both moments, or e4m3 codes of the first moment and of the second one's
                       root with m_scale, v_scale, one float32 per 256 elements.  Every tensor starts at a multiple of 256.
    weight_decay, lr_scale   one number, or one for each tensor
    """

    def __init__(self, ops: Ops, grads, params=None, masters=None, *, state_bits=32, m=None, v=None, m_scale=None, v_scale=None,
                 weight_decay=0.0, lr_scale=1.0):
        grads = _flat(grads, "grads")
        n = [t.numel() for t in grads]
        dev = grads[0].device if grads else torch.device("cuda", torch.cuda.current_device())
        _flat(grads, "grads", device=dev)
        ops._here(dev)
        self.ops, self.grads = ops, grads
        self.params = None if params is None else _flat(params, "params", n, dev)
        self.masters = None if masters is None else list(masters)
        if self.masters is not None:
            if len(self.masters) != len(n):
                raise ValueError("masters: one for each tensor, or None in its place")
            there = [i for i, t in enumerate(self.masters) if t is not None]
            _flat([self.masters[i] for i in there], "masters", [n[i] for i in there], dev)
            if any(self.masters[i].dtype != torch.float32 for i in there):
                raise TypeError("masters: float32 wanted")
        self.state_bits = state_bits if params is not None else 0
        self.state_offsets = [0]
        for k in n:
            self.state_offsets.append(self.state_offsets[-1] + -(-k // STATE_BLOCK) * STATE_BLOCK)
        total = self.state_offsets[-1]
        if self.state_bits:
            if state_bits not in (8, 32):
                raise ValueError("state_bits must be 8 or 32")
            dt = torch.float32 if state_bits == 32 else torch.float8_e4m3fn

            def state(t, size, dtype, fill=0):
                if t is None:
                    return torch.full((size,), fill, dtype=torch.uint8, device=dev).view(dtype) if dtype.itemsize == 1 else \
                        torch.full((size,), fill, dtype=dtype, device=dev)
                if t.device != dev or not t.is_contiguous() or t.numel() != size or t.element_size() != dtype.itemsize or \
                        (dtype.itemsize == 4 and t.dtype != dtype):
                    raise ValueError(f"state: {size} contiguous values of {dtype} on {dev} wanted")
                return t

            self.m, self.v = state(m, total, dt), state(v, total, dt)
            if state_bits == 8:
                self.m_scale = state(m_scale, total // STATE_BLOCK, torch.float32, 1)
                self.v_scale = state(v_scale, total // STATE_BLOCK, torch.float32, 1)
        wd = list(weight_decay) if hasattr(weight_decay, "__iter__") else [weight_decay] * len(n)
        lr = list(lr_scale) if hasattr(lr_scale, "__iter__") else [lr_scale] * len(n)
        if len(wd) != len(n) or len(lr) != len(n):
            raise ValueError("weight_decay and lr_scale: one number, or one for each tensor")
        desc = (cerar.TensorDesc * len(n))()
        for i, k in enumerate(n):
            d = desc[i]
            d.numel, d.grad, d.grad_type = k, grads[i].data_ptr(), _type(grads[i], "grads")
            if self.state_bits:
                at, size = self.state_offsets[i], state_bits // 8
                d.param, d.param_type = self.params[i].data_ptr(), _type(self.params[i], "params")
                d.master = None if self.masters is None or self.masters[i] is None else self.masters[i].data_ptr()
                d.m, d.v = self.m.data_ptr() + at * size, self.v.data_ptr() + at * size
                if state_bits == 8:
                    d.m_scale = self.m_scale.data_ptr() + at // STATE_BLOCK * 4
                    d.v_scale = self.v_scale.data_ptr() + at // STATE_BLOCK * 4
                d.lr_scale, d.weight_decay = lr[i], wd[i]
        out = C.c_void_p()
        _check(lib.cerar_tensors_create(ops._h, len(n), desc, self.state_bits, C.byref(out)))
        self._h = out
        ops._sets.add(self)
        self._device = dev
        self._opt = cerar.AdamwOptions()
        self._opt_at = C.addressof(self._opt)

    def destroy(self):
        if getattr(self, "_h", None):
            lib.cerar_tensors_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def set_grads(self, grads):
        """Points the set at other gradients of the same sizes and types, in stream order."""
        grads = _flat(grads, "grads", [t.numel() for t in self.grads], self.grads[0].device if self.grads else None)
        if any(a.dtype != b.dtype for a, b in zip(grads, self.grads)):
            raise TypeError("grads: the types differ from those the set was made with")
        _check(lib.cerar_tensors_set_grads(self._h, (C.c_void_p * len(grads))(*[t.data_ptr() for t in grads]), _stream()))
        self.grads = grads

    def grad_norm(self, max_norm: float = 0.0, out: torch.Tensor | None = None) -> torch.Tensor:
        """[norm, clip coefficient, 1 if finite] on the device; the third argument of a step that skips itself otherwise."""
        if out is None:
            out = torch.empty(3, dtype=_F32, device=self._device)
        elif out.dtype != _F32 or out.numel() != 3 or out.device != self._device or not out.is_contiguous():
            raise ValueError("out: three contiguous floats on the set's device are wanted")
        st = _norm(self._h, max_norm, out.data_ptr(), _stream(self._device.index))
        if st:
            _check(st)
        return out

    def adamw(self, *, lr: float, betas=(0.9, 0.95), eps: float = 1e-8, step: int, clip: torch.Tensor | None = None, seed: int = 0):
        """One AdamW step, in place.  clip: what grad_norm returned; seed: of the random rounding (8-bit states, bfloat16
        parameters without masters), another one for every step.  All of these are values of the call: a CUDA graph that captured it
        repeats them."""
        o = self._opt
        o.lr, o.beta1, o.beta2, o.eps, o.step, o.seed = lr, betas[0], betas[1], eps, step, seed
        if clip is not None and (clip.dtype != _F32 or clip.numel() != 3 or clip.device != self._device or not clip.is_contiguous()):
            raise ValueError("clip: the three floats that grad_norm returned are wanted")
        st = _adamw(self._h, self._opt_at, None if clip is None else clip.data_ptr(), _stream(self._device.index))
        if st:
            _check(st)

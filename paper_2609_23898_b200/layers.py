"""Layers around the linear ones, on torch tensors: what else of a model has weights whose gradients are aggregated.

  embed, embed_backward, Embed              embedding lookup with scaling, and its gradient by sorted tokens (cerar_embed, cerar_embed_grad)
  rotation_table, head_norm, head_norm_backward, HeadNorm
                                            norms of queries and keys for each head, with the rotation by position in the same pass
                                            (cerar_rotation_table, cerar_head_norm, cerar_head_norm_grad)
  matmul, gated, gated_backward, Gated      bfloat16 products, and a gated feed-forward block made of them (cerar_matmul_bf16, cerar_gated_forward,
                                            cerar_gated_backward)

As with training.Linear8 the gradients of weights are added to buffers of the caller's (slices of the vector that is aggregated) and the
weights have none of their own.  Everything runs on the current stream of the tensors' device, without synchronisation.
The formulas and rules stand in include/cerar.h.
"""
from __future__ import annotations

import ctypes as C
import struct

import torch
from torch.autograd.function import once_differentiable

from . import cerar
from .cerar import lib
from .training import _TYPES, Ops, _check, _matrix, _raw_stream, _rows, _stream, _type

HALVES, NEIGHBOURS = "halves", "neighbours"
_raw = _stream if _raw_stream is None else _raw_stream
_IDS = {torch.int32: 4, torch.int64: 8}


def _whole(t: torch.Tensor, what: str) -> int:
    size = _IDS.get(t.dtype)
    if size is None:
        raise TypeError(f"{what}: int32 or int64 wanted, got {t.dtype}")
    return size


def _kind(t: torch.Tensor, what: str) -> int:
    kind = _TYPES.get(t.dtype)
    return _type(t, what) if kind is None else kind


def _here(ops: Ops, tensors, names: str):
    """All of them (but None) on the operators' device; `names` are looked at only to say which one is not."""
    index = ops._index
    for i, t in enumerate(tensors):
        if t is not None and t.get_device() != index:
            if not t.is_cuda:
                raise ValueError(f"{names.split()[i]}: a CUDA tensor is wanted")
            ops._here(t.device)


def _stride(t: torch.Tensor) -> int:
    """Elements between rows of a matrix that _matrix has let pass (one row, or none: its length)."""
    rows, cols = t.shape
    return t.stride(0) if rows > 1 and cols else cols


def _no_gradient(**tensors):
    for what, t in tensors.items():
        if t is not None and t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{what} has no gradient of its own (it is added to d{what}): it must not require one")


def _anchor(device, wanted: bool):
    """Where no input is a tensor that autograd follows, an empty one takes that place (see training.Linear8)."""
    return torch.empty(0, device=device, requires_grad=True) if wanted and torch.is_grad_enabled() else None


def _save(ctx, *tensors):
    """Saved as autograd saves tensors: freed by the backward pass, within reach of saved-tensor hooks, and refused if changed in between.
    (Those made in inference mode cannot be saved; they are held as they are.)"""
    ctx.held = tuple(t if t is not None and t.is_inference() else None for t in tensors)
    ctx.save_for_backward(*(t if h is None else None for t, h in zip(tensors, ctx.held)))


def _saved(ctx) -> list:
    return [t if h is None else h for t, h in zip(ctx.saved_tensors, ctx.held)]


# ------------------------------------------------------------------------------------------------ embedding


def embed(ops: Ops, table: torch.Tensor, ids: torch.Tensor, *, scale: float = 1.0, dtype: torch.dtype | None = None) -> torch.Tensor:
    """scale * table[ids], of `dtype` (the table's): shape of ids, then the table's width.  An id below zero is padding and gives zeros;
    one beyond the table does so too, and Ops.status raises."""
    _here(ops, (table, ids), "table ids")
    _matrix(table, "table")
    kind, size = _kind(table, "table"), _whole(ids, "ids")
    if not ids.is_contiguous():
        ids = ids.contiguous()
    vocab, width = table.shape
    y = torch.empty(*ids.shape, width, dtype=dtype or table.dtype, device=table.device)      # (numbers: a torch.Size takes twice as long)
    st = lib.cerar_embed(ops._h, table.data_ptr(), kind, vocab, width, _stride(table), ids.data_ptr(), size, ids.numel(), scale, y.data_ptr(),
                         _kind(y, "dtype"), width, _raw(ops._index))
    if st:
        _check(st)
    return y


def embed_backward(ops: Ops, dy: torch.Tensor, ids: torch.Tensor, dtable: torch.Tensor, *, scale: float = 1.0, accumulate=True):
    """dtable[v] += scale * the sum of dy over the tokens v (without accumulate: = that, and zeros for tokens that ids has none of).
    Deterministic."""
    _here(ops, (dy, ids, dtable), "dy ids dtable")
    _matrix(dtable, "dtable")
    vocab, width = dtable.shape
    if dy.shape != (*ids.shape, width):
        raise ValueError(f"dy of shape {(*ids.shape, width)} wanted, got {tuple(dy.shape)}")
    kind, size = _kind(dy, "dy"), _whole(ids, "ids")
    dy = _rows(dy)
    if not ids.is_contiguous():
        ids = ids.contiguous()
    n = ids.numel()
    need = lib.cerar_embed_grad_workspace(n, vocab, width)
    ws = torch.empty(need, dtype=torch.uint8, device=dtable.device)
    st = lib.cerar_embed_grad(ops._h, dy.data_ptr(), kind, _stride(dy), ids.data_ptr(), size, n, scale, dtable.data_ptr(),
                              _kind(dtable, "dtable"), vocab, width, _stride(dtable), accumulate, ws.data_ptr(), need, _raw(ops._index))
    if st:
        _check(st)


class Embed(torch.autograd.Function):
    """embed and embed_backward for torch.autograd: y = Embed.apply(table, ids, ops, dtable, scale).  Every pass backward adds to `dtable`
    (None: no gradient); second derivatives are refused."""

    @classmethod
    def apply(cls, table, ids, ops, dtable, scale=1.0):
        _no_gradient(table=table)
        return super().apply(table, ids, ops, dtable, scale, _anchor(table.device, dtable is not None))

    @staticmethod
    def forward(ctx, table, ids, ops, dtable, scale, anchor):
        ctx.ops, ctx.dtable, ctx.scale = ops, dtable, scale
        _save(ctx, ids)
        return embed(ops, table, ids, scale=scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        ids, = _saved(ctx)
        embed_backward(ctx.ops, dy, ids, ctx.dtable, scale=ctx.scale)
        return None, None, None, None, None, None


# ------------------------------------------------------------------------------------------------ head norms


def rotation_table(ops: Ops, rows: int, dim: int, *, base: float = 10000.0, freqs=None, first: int = 0) -> torch.Tensor:
    """Cosine and sine of the angles of positions first .. first + rows - 1, float32 (rows, dim / 2, 2); pair j turns by freqs[j]
    (base ** (-2 j / dim)) per position.  The angles are worked out in 64 bits."""
    freqs = [base ** (-2.0 * j / dim) for j in range(dim // 2)] if freqs is None else [float(f) for f in freqs]
    if dim < 0 or dim % 2 or len(freqs) != dim // 2:
        raise ValueError("rotation_table: an even dim and dim / 2 frequencies are wanted")
    table = torch.empty(rows, dim // 2, 2, dtype=torch.float32, device=torch.device("cuda", ops._index))
    _check(lib.cerar_rotation_table(ops._h, (C.c_double * len(freqs))(*freqs), len(freqs), first, rows, table.data_ptr(), _raw(ops._index)))
    return table


def _heads(t: torch.Tensor, what: str) -> torch.Tensor:
    """t (..., heads, dim) as (tokens, heads, dim) with a head's values next to one another: a copy only where there is no such view."""
    if t.dim() != 3:
        if t.dim() < 3:
            raise ValueError(f"{what}: (tokens, heads, values) or more dimensions are wanted")
        t = t.flatten(0, -3)
    return t if t.stride(2) == 1 or t.size(2) < 2 else t.contiguous()


_PARTS, _ROTATION = struct.Struct("24q"), struct.Struct("4q3i4x")         # two cerar_heads_t, one cerar_rotation_t
assert _PARTS.size == 2 * C.sizeof(cerar.Heads) and _ROTATION.size == C.sizeof(cerar.Rotation)


def _rotation(table, positions, lead, pairs) -> bytes:
    """(positions: contiguous)"""
    if pairs != HALVES and pairs != NEIGHBOURS:
        raise ValueError("pairs must be 'halves' or 'neighbours'")
    period, at, size, first, rows, rotated = lead[-1], 0, 8, 0, 0, 0
    if positions is not None:
        size = _whole(positions, "positions")
        if positions.shape != lead and positions.shape != lead[-1:]:
            raise ValueError(f"positions of shape {tuple(lead)} or {tuple(lead[-1:])} wanted, got {tuple(positions.shape)}")
        at, period = positions.data_ptr(), positions.numel()
    if table is not None:
        if table.dtype != torch.float32 or table.dim() != 3 or table.size(2) != 2 or not table.is_contiguous():
            raise ValueError("table: contiguous float32 of shape (positions, pairs, 2) wanted, as rotation_table makes it")
        first, rows, rotated = table.data_ptr(), table.size(0), 2 * table.size(1)
    return _ROTATION.pack(first, rows, at, period or 1, size, rotated, pairs == NEIGHBOURS)


def _part(what, x, w, y, dy, dw, like, types):
    """One group of heads: its fields of the descriptor, the result, its numbers, and what has to live until the call has been made.
    types: those of the weights and of their gradients so far."""
    shape, dtype = x.shape, x.dtype
    x3 = _heads(x, what)
    n, h, d = x3.shape
    if like is not None and (n != like[0] or d != like[1] or dtype != like[2] or (len(like[3]) != 1 if x3 is x else shape[:-2] != like[3])):
        raise ValueError("q and k: the same tokens, values per head and type are wanted")
    sx = x3.stride()
    if y is None:
        y = torch.empty(*shape, dtype=dtype, device=x.device)
        y3, ty, hy = y, h * d, d
    else:
        if y.shape != shape or y.dtype != dtype:
            raise ValueError("out: tensors of the shapes and type of q and k are wanted")
        y3 = y if y.dim() == 3 else y.flatten(0, -3)
        ty, hy, cy = y3.stride()
        if y3.data_ptr() != y.data_ptr() or (cy != 1 and d > 1):
            raise ValueError("out: leading dimensions that can be flattened and contiguous heads are wanted")
    pw = pdw = pdy = tdy = hdy = 0
    dy3 = None
    if w is not None:
        if w.shape != (d,) or not w.is_contiguous():
            raise ValueError(f"w{what}: {d} contiguous weights wanted")
        kind = _kind(w, "w" + what)
        if types[0] is not None and types[0] != kind:
            raise TypeError("wq and wk: one type is wanted")
        pw, types[0] = w.data_ptr(), kind
    if dy is not None:
        if dy.shape != shape or dy.dtype != dtype:
            raise ValueError(f"d{what}: the shape and type of {what} wanted")
        dy3 = _heads(dy, "d" + what)
        pdy, (tdy, hdy, _) = dy3.data_ptr(), dy3.stride()
    if dw is not None:
        if dw.shape != (d,) or not dw.is_contiguous():
            raise ValueError(f"dw{what}: {d} contiguous values wanted")
        kind = _kind(dw, "dw" + what)
        if types[1] is not None and types[1] != kind:
            raise TypeError("dwq and dwk: one type is wanted")
        pdw, types[1] = dw.data_ptr(), kind
    return (x3.data_ptr(), y3.data_ptr(), pw, pdy, pdw, sx[0], sx[1], ty, hy, tdy, hdy, h), y, n, d, (x3, dy3)


_NO_PART = (0,) * 12


def head_norm(ops: Ops, q: torch.Tensor, k: torch.Tensor | None, wq, wk, table: torch.Tensor | None, positions: torch.Tensor | None = None, *,
              eps: float = 1e-6, pairs: str = HALVES, out=None):
    """Every head of q and k (..., heads, values; k may be None) divided by its root mean square, times wq, wk (None: one), its first values turned
    by the token's position: those that `table` (rotation_table; None: no rotation) has pairs for.  positions: of every token, or of
    the last dimension of the tokens, for all sequences alike (None: 0, 1, ...); below zero: padding, whose result is zero; beyond the
    table: the same, and Ops.status raises.  q and k may be slices of one projection's result.  Returns both (in `out`, if given: q and k
    themselves for results in place)."""
    _here(ops, (q, k, wq, wk, table, positions), "q k wq wk table positions")
    kind, types = _kind(q, "q"), [None, None]
    yq, yk = (None, None) if out is None else out
    first, yq, n, d, kept = _part("q", q, wq, yq, None, None, None, types)
    second, yk, _, _, kept2 = (_NO_PART, None, 0, 0, None) if k is None else _part("k", k, wk, yk, None, None, (n, d, q.dtype, q.shape[:-2]), types)
    if positions is not None and not positions.is_contiguous():
        positions = positions.contiguous()
    rotation = _rotation(table, positions, q.shape[:-2], pairs)
    st = lib.cerar_head_norm(ops._h, kind, _PARTS.pack(*first, *second), 1 if k is None else 2, types[0] or 0, n, d, eps, rotation, _raw(ops._index))
    if st:
        _check(st)
    return yq, yk


def head_norm_backward(ops: Ops, dq: torch.Tensor, dk: torch.Tensor | None, q: torch.Tensor, k: torch.Tensor | None, wq, wk, table, positions=None, *,
                       dwq=None, dwk=None, accumulate=True, eps: float = 1e-6, pairs: str = HALVES, out=None):
    """Gradients of q and k (in `out`, if given, e.g. dq and dk themselves) from those of head_norm's results; dwq, dwk (float32 or bfloat16,
    None: not wanted; the same one where q and k share their weights) += those of the weights.  Deterministic."""
    _here(ops, (dq, dk, q, k, wq, wk, table, positions, dwq, dwk), "dq dk q k wq wk table positions dwq dwk")
    kind, types = _kind(q, "q"), [None, None]
    if (dk is None) != (k is None) or (k is None and dwk is not None):
        raise ValueError("dk and dwk belong to k")
    yq, yk = (None, None) if out is None else out
    first, yq, n, d, kept = _part("q", q, wq, yq, dq, dwq, None, types)
    second, yk, _, _, kept2 = (_NO_PART, None, 0, 0, None) if k is None else _part("k", k, wk, yk, dk, dwk, (n, d, q.dtype, q.shape[:-2]), types)
    if positions is not None and not positions.is_contiguous():
        positions = positions.contiguous()
    rotation = _rotation(table, positions, q.shape[:-2], pairs)
    count = 1 if k is None else 2
    need = lib.cerar_head_norm_grad_workspace(count, d)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    st = lib.cerar_head_norm_grad(ops._h, kind, _PARTS.pack(*first, *second), count, types[0] or 0, types[1] or 0, accumulate, n, d, eps, rotation,
                                  ws.data_ptr(), need, _raw(ops._index))
    if st:
        _check(st)
    return yq, yk


class HeadNorm(torch.autograd.Function):
    """head_norm and head_norm_backward for torch.autograd: q, k = HeadNorm.apply(q, k, wq, wk, ops, table, positions, dwq, dwk, eps, pairs).
    Every pass backward adds to dwq and dwk (None: not wanted); second derivatives are refused."""

    @classmethod
    def apply(cls, q, k, wq, wk, ops, table, positions=None, dwq=None, dwk=None, eps=1e-6, pairs=HALVES):
        _no_gradient(wq=wq, wk=wk)
        followed = q.requires_grad or (k is not None and k.requires_grad)
        anchor = _anchor(q.device, (dwq is not None or dwk is not None) and not followed)
        return super().apply(q, k, wq, wk, ops, table, positions, dwq, dwk, eps, pairs, anchor)

    @staticmethod
    def forward(ctx, q, k, wq, wk, ops, table, positions, dwq, dwk, eps, pairs, anchor):
        ctx.ops, ctx.dw, ctx.rest = ops, (dwq, dwk), (eps, pairs)
        _save(ctx, q, k, wq, wk, table, positions)
        return head_norm(ops, q, k, wq, wk, table, positions, eps=eps, pairs=pairs)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        q, k, wq, wk, table, positions = _saved(ctx)
        eps, pairs = ctx.rest
        dxq, dxk = head_norm_backward(ctx.ops, dq, dk, q, k, wq, wk, table, positions, dwq=ctx.dw[0], dwk=ctx.dw[1], eps=eps, pairs=pairs)
        need = ctx.needs_input_grad
        return (dxq if need[0] else None, dxk if need[1] else None) + (None,) * 10


# ------------------------------------------------------------------------------------------------ bfloat16 products, gated block

_ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}
_BF16 = torch.bfloat16


_ROWS = struct.Struct("6q")          # cerar_rows_t
_BLOCK = struct.Struct("25q")        # cerar_gated_t
assert _BLOCK.size == C.sizeof(cerar.GatedBlock)


def _bf16(t: torch.Tensor, what: str) -> torch.Tensor:
    """A bfloat16 matrix whose rows are contiguous: a copy where they are not."""
    if t.dtype != _BF16:
        raise TypeError(f"{what}: bfloat16 wanted, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{what}: a two-dimensional tensor is wanted")
    return _rows(t)


def _operands(ops: Ops, *given):
    """bfloat16 matrices (as _bf16 gives them) with rows on 16-byte boundaries, as tensor-map copies read them: copies, one launch for all of them, of
    those that are not.  Each as (tensor, address, elements between rows)."""
    out, copies = [], b""
    for t in given:
        rows, cols = t.shape
        row, at, ld = t.stride(0), t.data_ptr(), (cols + 7) & -8
        if not (rows and cols) or not at & 15 and (rows == 1 or not row & 7):
            out.append((t, at, row if rows > 1 and cols else ld))
            continue
        wide = torch.empty(rows, ld, dtype=_BF16, device=t.device)
        to = wide.data_ptr()
        copies += _ROWS.pack(at, to, rows, cols, row if rows > 1 else cols, ld)
        out.append((wide, to, ld))
    if copies:
        st = lib.cerar_align_bf16(ops._h, copies, len(copies) // _ROWS.size, _raw(ops._index))
        if st:
            _check(st)
    return out


def _meet(p, rows, width, pitch, q, rows2, cols2, ld2) -> bool:
    """Whether two matrices share a byte: address, rows, bytes of a row, bytes between rows; the second one, of bfloat16, with its columns and elements between rows."""
    width2, pitch2 = 2 * cols2, 2 * ld2
    if q + (rows2 - 1) * pitch2 + width2 <= p or p + (rows - 1) * pitch + width <= q or not (rows and width and rows2 and width2):
        return False
    if rows == 1:
        pitch = pitch2
    elif rows2 == 1:
        pitch2 = pitch
    if pitch == pitch2:      # two rows lie apart as the first one does from some row of a longer matrix
        starts, q, rows2 = (p,), q - (rows - 1) * pitch, rows + rows2 - 1
    else:
        starts = range(p, p + rows * pitch, pitch)
    # for each row: the numbers of the other matrix's rows that end behind its start, and that start in front of its end
    return any(max(0, (at - width2 - q) // pitch2 + 1) <= min(rows2 - 1, (at + width - 1 - q) // pitch2) for at in starts)


def matmul(ops: Ops, a: torch.Tensor, b: torch.Tensor, *, trans_a=False, trans_b=False, out: torch.Tensor | None = None,
           dtype: torch.dtype = torch.bfloat16, accumulate=False) -> torch.Tensor:
    """op(a) op(b) of bfloat16 matrices, into `out` (float32 or bfloat16, over neither of them) if given, added to it with accumulate."""
    _here(ops, (a, b, out), "a b out")
    a, b = _bf16(a, "a"), _bf16(b, "b")
    m, k = (a.size(1), a.size(0)) if trans_a else a.shape
    k2, n = (b.size(1), b.size(0)) if trans_b else b.shape
    if k != k2:
        raise ValueError("the summed dimensions of a and b differ")
    fresh = out is None
    if fresh:
        if accumulate:
            raise ValueError("accumulate wants an `out` to add to")
        out = torch.empty(m, n, dtype=dtype, device=a.device)
    else:
        _matrix(out, "out")
        if tuple(out.shape) != (m, n):
            raise ValueError(f"out of shape {(m, n)} wanted, got {tuple(out.shape)}")
    (a, pa, lda), (b, pb, ldb) = _operands(ops, a, b)
    pc, ldc = out.data_ptr(), _stride(out)
    if not fresh:
        size = out.element_size()
        end = pc + m * ldc * size                    # (where the ranges lie apart there is no more to do)
        if (pa < end and _meet(pc, m, n * size, ldc * size, pa, *a.shape, lda)) or (pb < end and _meet(pc, m, n * size, ldc * size, pb, *b.shape, ldb)):
            raise ValueError("out lies over a or b")
    st = lib.cerar_matmul_bf16(ops._h, pa, lda, trans_a, pb, ldb, trans_b, m, n, k, pc, _kind(out, "out"), ldc, accumulate, _raw(ops._index))
    if st:
        _check(st)
    return out


def _gated_sizes(x, w_in, w_out, activation):
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(_ACTIVATIONS)}")
    if w_in.dim() != 2 or w_out.dim() != 2 or w_in.size(0) != 2 * w_out.size(1):
        raise ValueError("w_in (2 hidden x inputs: the gate's rows, then the others) and w_out (outputs x hidden) are wanted")
    if x.dim() < 1 or x.size(-1) != w_in.size(1):
        raise ValueError(f"x: {w_in.size(1)} values in the last dimension wanted")


def gated(ops: Ops, x: torch.Tensor, w_in: torch.Tensor, w_out: torch.Tensor, *, activation: str = "silu", keep=False):
    """(act(x w_g^T) * (x w_u^T)) w_out^T for x (..., inputs), w_in = w_g over w_u (2 hidden x inputs) and w_out (outputs x hidden), all bfloat16.
    activation: silu, gelu, gelu_tanh or relu.  With keep also what gated_backward wants of it: (x, g and u in 24 bits, the activation)."""
    _here(ops, (x, w_in, w_out), "x w_in w_out")
    _gated_sizes(x, w_in, w_out, activation)
    xm, wi, wo = _bf16(_rows(x), "x"), _bf16(w_in, "w_in"), _bf16(w_out, "w_out")
    (t, d), (o, f), device = xm.shape, wo.shape, x.device
    gu = torch.empty(lib.cerar_gated_kept_bytes(t, f), dtype=torch.uint8, device=device) if keep else None
    y = torch.empty(t, o, dtype=_BF16, device=device)
    block = _BLOCK.pack(t, d, f, o, _ACTIVATIONS[activation], 0, xm.data_ptr(), _stride(xm), wi.data_ptr(), _stride(wi), wo.data_ptr(), _stride(wo),
                        gu.data_ptr() if keep else 0, y.data_ptr(), o, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    need = lib.cerar_gated_workspace(block, 0)
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    st = lib.cerar_gated_forward(ops._h, block, ws.data_ptr(), need, _raw(ops._index))
    if st:
        _check(st)
    if x.dim() != 2:
        y = y.view(*x.shape[:-1], o)
    return (y, (xm, gu, activation)) if keep else y


def gated_backward(ops: Ops, dy: torch.Tensor, kept, w_in: torch.Tensor, w_out: torch.Tensor, dw_in: torch.Tensor | None, dw_out: torch.Tensor | None, *,
                   accumulate=True, need_dx=True):
    """dx from dy and what gated kept; dw_in and dw_out (float32 or bfloat16, e.g. slices of the gradient vector; None: not wanted) += the
    gradients of the weights."""
    x, gu, activation = kept
    _here(ops, (dy, x, gu, w_in, w_out, dw_in, dw_out), "dy x kept w_in w_out dw_in dw_out")
    _gated_sizes(x, w_in, w_out, activation)
    dym, wi, wo = _bf16(_rows(dy), "dy"), _bf16(w_in, "w_in"), _bf16(w_out, "w_out")
    (t, d), (o, f), device = x.shape, wo.shape, x.device
    if gu.numel() != lib.cerar_gated_kept_bytes(t, f):
        raise ValueError("kept does not belong to weights of these sizes")
    if dym.shape != (t, o):
        raise ValueError(f"dy: {t} rows of {o} values wanted")
    grads = []
    for what, dw, w in (("dw_in", dw_in, w_in), ("dw_out", dw_out, w_out)):
        if dw is None:
            grads += (0, 0, 0)
            continue
        _matrix(dw, what)
        if dw.shape != w.shape:
            raise ValueError(f"{what} of shape {tuple(w.shape)} wanted, got {tuple(dw.shape)}")
        grads += (dw.data_ptr(), _stride(dw), _kind(dw, what))
    dx = torch.empty(t, d, dtype=_BF16, device=device) if need_dx else None
    block = _BLOCK.pack(t, d, f, o, _ACTIVATIONS[activation], bool(accumulate), x.data_ptr(), _stride(x), wi.data_ptr(), _stride(wi), wo.data_ptr(), _stride(wo),
                        gu.data_ptr(), 0, 0, dym.data_ptr(), _stride(dym), dx.data_ptr() if need_dx else 0, d, *grads)
    need = lib.cerar_gated_workspace(block, 1)
    ws = torch.empty(need, dtype=torch.uint8, device=device)
    st = lib.cerar_gated_backward(ops._h, block, ws.data_ptr(), need, _raw(ops._index))
    if st:
        _check(st)
    return dx if not need_dx or dy.dim() == 2 else dx.view(*dy.shape[:-1], d)


class Gated(torch.autograd.Function):
    """gated and gated_backward for torch.autograd: y = Gated.apply(x, w_in, w_out, ops, dw_in, dw_out, activation).  Every pass backward adds to
    dw_in and dw_out (None: not wanted); second derivatives are refused."""

    @classmethod
    def apply(cls, x, w_in, w_out, ops, dw_in, dw_out, activation="silu"):
        _no_gradient(w_in=w_in, w_out=w_out)
        wanted = dw_in is not None or dw_out is not None
        # (forward does not see the caller's mode: under no_grad needs_input_grad still says what x requires)
        keep = torch.is_grad_enabled() and (wanted or x.requires_grad)
        return super().apply(x, w_in, w_out, ops, dw_in, dw_out, activation, _anchor(x.device, wanted and not x.requires_grad), keep)

    @staticmethod
    def forward(ctx, x, w_in, w_out, ops, dw_in, dw_out, activation, anchor, keep):
        if not keep:
            return gated(ops, x, w_in, w_out, activation=activation)
        y, kept = gated(ops, x, w_in, w_out, activation=activation, keep=True)
        ctx.ops, ctx.dw, ctx.activation = ops, (dw_in, dw_out), activation
        _save(ctx, *kept[:2], w_in, w_out)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        *kept, w_in, w_out = _saved(ctx)
        dx = gated_backward(ctx.ops, dy, (*kept, ctx.activation), w_in, w_out, *ctx.dw, need_dx=ctx.needs_input_grad[0])
        return (dx,) + (None,) * 8

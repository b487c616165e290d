"""Thin binding of the C ABI in include/rb_block.h: what a block of a model computes between its matrix products.

As in train.py every function has the name and argument order of its C counterpart, and the classes only own device memory, keep a handle, look at
what they are given and raise RbError on a non-zero status.  There is no fallback: if librb_block.so is missing the import fails.
"""
import ctypes as C
import os
import struct
from typing import NamedTuple, Optional

import torch

from .binding import Call, HERE, _check, _ptr, _stream
from .train import _CODES, _OnStream, _current_stream, _fits, _written

BLOCK_LIB_PATH = os.environ.get("RB_BLOCK_LIBRARY") or os.path.join(HERE, "librb_block.so")   # RB_BLOCK_LIBRARY: another build of the same library

RB_MAX_NORM_ROWS, RB_MAX_NORM_WIDTH, RB_MAX_DROP_WIDTH = 1 << 23, 32768, 1 << 27
RB_MAX_HEADS, RB_MAX_HEAD_DIM, RB_MAX_TOKENS, RB_MAX_HEAD_ROWS, RB_MAX_DOCUMENTS = 1024, 128, 1 << 22, 1 << 30, 1 << 22

BLOCK_EXPORTS = (
    "rb_dropout", "rb_norm_create", "rb_norm_query", "rb_norm_bind", "rb_norm_forward", "rb_norm_grad", "rb_norm_destroy",
    "rb_attention_create", "rb_attention_query", "rb_attention_bind", "rb_attention_forward", "rb_attention_grad", "rb_attention_destroy",
)

__all__ = ["BLOCK_EXPORTS", "BLOCK_LIB_PATH", "RB_MAX_NORM_ROWS", "RB_MAX_NORM_WIDTH", "RB_MAX_DROP_WIDTH", "RB_MAX_HEADS", "RB_MAX_HEAD_DIM", "RB_MAX_TOKENS",
           "RB_MAX_HEAD_ROWS", "RB_MAX_DOCUMENTS", "RbRows", "RbHeads", "RbDrop", "RbDocuments", "Drop", "Normed", "NormGrads", "Documents", "Attended", "dropout",
           "LayerNorm", "DocumentAttention", *BLOCK_EXPORTS]


class RbDrop(C.Structure):
    _fields_ = [("p", C.c_double), ("seed", C.c_uint64), ("step", C.c_uint64)]


class RbRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64)]


class RbHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class RbDocuments(C.Structure):
    _fields_ = [("offsets", C.c_void_p), ("lengths", C.c_void_p), ("prefixes", C.c_void_p), ("count", C.c_int64)]


def _load():
    if not os.path.exists(BLOCK_LIB_PATH):
        raise ImportError(
            f"{BLOCK_LIB_PATH} is missing: build it with `python paper_2406_03285_amd/build.py` "
            "(there is no fallback path)")
    L = C.CDLL(BLOCK_LIB_PATH)
    vp, i64, i32, sz, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t, C.c_float
    rows = heads = drop = docs = vp            # (addresses of structures)
    L.rb_dropout.argtypes = [vp, i64, i64, i64, i32, drop, vp, i64, vp]
    L.rb_norm_create.argtypes = [C.POINTER(vp), i64, i32, i32, f32]
    L.rb_norm_query.argtypes = [vp, C.POINTER(sz)]
    L.rb_norm_bind.argtypes = [vp, vp]
    L.rb_norm_forward.argtypes = [vp, rows, rows, drop, i64, vp, vp, rows, rows, vp, vp, vp]
    L.rb_norm_grad.argtypes = [vp, rows, rows, rows, vp, vp, drop, i64, vp, rows, rows, vp, vp, vp]
    L.rb_norm_destroy.argtypes = [vp]
    L.rb_attention_create.argtypes = [C.POINTER(vp), i64, i64, i64, i64, i32, f32, f32]
    L.rb_attention_query.argtypes = [vp, C.POINTER(sz)]
    L.rb_attention_bind.argtypes = [vp, vp]
    L.rb_attention_forward.argtypes = [vp, heads, heads, heads, i64, docs, vp, heads, vp, vp]
    L.rb_attention_grad.argtypes = [vp, heads, heads, heads, i64, docs, vp, heads, vp, heads, heads, heads, heads, vp]
    L.rb_attention_destroy.argtypes = [vp]
    for name in BLOCK_EXPORTS:
        getattr(L, name).restype = C.c_int
    return L


_L = _load()


def _at(structure):
    """The address of RbRows, RbHeads, RbDrop or RbDocuments, which an address itself may stand for (None: null)."""
    return C.addressof(structure) if isinstance(structure, C.Structure) else structure


def _native(general, layout):
    """As in binding.py: the same function with its usual arguments - here structures by their addresses - marshalled natively."""
    if Call is None:
        return general
    return Call(C.cast(getattr(_L, general.__name__), C.c_void_p).value, layout, general)


def rb_dropout(x, x_stride, rows, width, dtype, drop, out, out_stride, hip_stream=None):
    return _L.rb_dropout(_ptr(x), int(x_stride), int(rows), int(width), int(dtype), _at(drop), _ptr(out), int(out_stride), _stream(hip_stream))


def rb_norm_create(width, dtype, weight_dtype, eps):
    h = C.c_void_p()
    rc = _L.rb_norm_create(C.byref(h), int(width), int(dtype), int(weight_dtype), float(eps))
    return rc, h.value


def rb_norm_query(n):
    size = C.c_size_t()
    rc = _L.rb_norm_query(n, C.byref(size))
    return rc, size.value


def rb_norm_bind(n, workspace):
    return _L.rb_norm_bind(n, _ptr(workspace))


def rb_norm_forward(n, x, residual, drop, rows, weight, bias, total, y, mean, rstd, hip_stream=None):
    return _L.rb_norm_forward(n, _at(x), _at(residual), _at(drop), int(rows), _ptr(weight), _ptr(bias), _at(total), _at(y), _ptr(mean), _ptr(rstd), _stream(hip_stream))


def rb_norm_grad(n, grad_y, total, grad_total, mean, rstd, drop, rows, weight, grad_sum, grad_x, grad_weight, grad_bias, hip_stream=None):
    return _L.rb_norm_grad(n, _at(grad_y), _at(total), _at(grad_total), _ptr(mean), _ptr(rstd), _at(drop), int(rows), _ptr(weight), _at(grad_sum), _at(grad_x),
                           _ptr(grad_weight), _ptr(grad_bias), _stream(hip_stream))


def rb_norm_destroy(n):
    return _L.rb_norm_destroy(n)


def rb_attention_create(heads, kv_heads, head_dim, max_tokens, causal, scale, cap):
    h = C.c_void_p()
    rc = _L.rb_attention_create(C.byref(h), int(heads), int(kv_heads), int(head_dim), int(max_tokens), int(causal), float(scale), float(cap))
    return rc, h.value


def rb_attention_query(a):
    size = C.c_size_t()
    rc = _L.rb_attention_query(a, C.byref(size))
    return rc, size.value


def rb_attention_bind(a, workspace):
    return _L.rb_attention_bind(a, _ptr(workspace))


def rb_attention_forward(a, q, k, v, tokens, documents, slopes, out, lse, hip_stream=None):
    return _L.rb_attention_forward(a, _at(q), _at(k), _at(v), int(tokens), _at(documents), _ptr(slopes), _at(out), _ptr(lse), _stream(hip_stream))


def rb_attention_grad(a, q, k, v, tokens, documents, slopes, out, lse, grad_out, grad_q, grad_k, grad_v, hip_stream=None):
    return _L.rb_attention_grad(a, _at(q), _at(k), _at(v), int(tokens), _at(documents), _ptr(slopes), _at(out), _ptr(lse), _at(grad_out), _at(grad_q), _at(grad_k),
                                _at(grad_v), _stream(hip_stream))


def rb_attention_destroy(a):
    return _L.rb_attention_destroy(a)


rb_dropout = _native(rb_dropout, "piiiihpis")
rb_norm_forward = _native(rb_norm_forward, "hhhhipphhpps")
rb_norm_grad = _native(rb_norm_grad, "hhhhpphiphhpps")
rb_attention_forward = _native(rb_attention_forward, "hhhhihphps")
rb_attention_grad = _native(rb_attention_grad, "hhhhihphphhhhs")


class _Structures:
    """Memory for the structures of a handle's calls, which are read before a call returns."""

    def __init__(self, layout):
        self._pack = struct.Struct(layout)
        self._memory = C.create_string_buffer(self._pack.size)
        self.address = C.addressof(self._memory)

    def fill(self, *values):
        self._pack.pack_into(self._memory, 0, *values)
        return self.address


# ---- dropout -------------------------------------------------------------------

class Drop(NamedTuple):
    """Dropout with probability p; the mask is a function of seed, step, row and column.  Every layer of a training step has a step (or a seed) of its own.  Both are
    numbers of the host: a call that was captured into a graph has the same mask in every replay."""
    p: float
    seed: int
    step: int

    def structure(self):
        return RbDrop(self.p, self.seed & (2 ** 64 - 1), self.step & (2 ** 64 - 1))


def _rows_of(t, width, dtype, index, what):
    """(rows, elements between them) of a tensor of rows, looked at first."""
    shape, (stride, step) = t.shape, t.stride()
    assert len(shape) == 2 and shape[1] == width and t.dtype == dtype and t.get_device() == index, what
    assert step == 1 or width == 1 or shape[0] == 0, what
    return shape[0], stride if shape[0] > 1 else max(stride, width)


def _drop_rows(x, drop, out):
    index, dtype = x.get_device(), x.dtype
    assert index >= 0 and dtype in _CODES, "x"
    rows, stride = _rows_of(x, x.shape[-1], dtype, index, "x")
    width = x.shape[1]
    out_rows, out_stride = (rows, stride) if out is x else _rows_of(out, width, dtype, index, "out")
    assert out_rows == rows, "out"
    if rows == 0:
        return out
    structure = drop.structure()
    if torch.cuda.current_device() == index:
        rc = rb_dropout(x, stride, rows, width, _CODES[dtype], C.addressof(structure), out, out_stride, _current_stream(index))
    else:
        with torch.cuda.device(index):
            rc = rb_dropout(x, stride, rows, width, _CODES[dtype], C.addressof(structure), out, out_stride, _current_stream(index))
    _check(rc, "rb_dropout")
    return out


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, drop):
        ctx.drop = drop
        return _drop_rows(x, drop, torch.empty(x.shape, dtype=x.dtype, device=x.device))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        if grad.stride(-1) != 1 or grad.stride(0) < grad.shape[1]:
            grad = grad.contiguous()
        return _drop_rows(grad, ctx.drop, torch.empty(grad.shape, dtype=grad.dtype, device=grad.device)), None


def dropout(x, drop, out=None):
    """Dropout of x [rows, width] (rows may be strided), binary32 or bfloat16, as `drop` says: a differentiable call; into `out` if given (which x may be),
    without gradient."""
    if out is None:
        return _Dropout.apply(x, drop)
    assert not (torch.is_grad_enabled() and (x.requires_grad or out.requires_grad)), "out= has no gradient"
    _drop_rows(x, drop, out)
    _written(out)
    return out


# ---- layer norm ------------------------------------------------------------------

class Normed(NamedTuple):
    """What LayerNorm.forward gives; total is None without residual and drop."""
    y: torch.Tensor                        # [rows, width]
    total: Optional[torch.Tensor]          # [rows, width]: the residual and what was left of x
    mean: torch.Tensor                     # [rows], binary32, as rstd
    rstd: torch.Tensor


class NormGrads(NamedTuple):
    """What LayerNorm.grad gives; x is None without drop (the gradient of x is total's then), bias where none was asked for."""
    total: torch.Tensor                    # [rows, width]: of the sum, so of the residual
    x: Optional[torch.Tensor]
    weight: Optional[torch.Tensor]         # [width]
    bias: Optional[torch.Tensor]


class _NormOutputs(Normed):
    """Normed's tensors that LayerNorm.outputs has made: `norm` and `rows` say for what (of one that was changed since: for none)."""
    norm = rows = None


class _NormGradients(NormGrads):
    norm = rows = None


_M64 = 2 ** 64 - 1


class LayerNorm(_OnStream):
    """Layer norm of rows, alone or of residual + dropout(x), and its gradients.  One handle serves all layers of a width (it holds no weights), and one host thread
    at a time.

    norm = LayerNorm(1024, torch.bfloat16, weight_dtype=torch.float32)
    o = norm.forward(x, weight, bias, residual=r, drop=Drop(0.1, seed, step))      # Normed; x, r [rows, width], rows may be strided
    o = norm(x, weight, bias, residual=r, drop=d)                                  # the same within autograd: o.y and o.total carry gradients
    """

    def __init__(self, width, dtype=torch.float32, weight_dtype=None, eps=1e-5, device="cuda"):
        self.weight_dtype = dtype if weight_dtype is None else weight_dtype
        rc, self.handle = rb_norm_create(width, _CODES[dtype], _CODES[self.weight_dtype], eps)
        _check(rc, "rb_norm_create")
        self.width, self.dtype = int(width), dtype
        self._bind_device(device)
        rc, size = rb_norm_query(self.handle)
        _check(rc, "rb_norm_query")
        self.workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(rb_norm_bind(self.handle, self.workspace), "rb_norm_bind")
        self._structures = _Structures("=QqQqQqQqQqdQQ")       # five rb_rows, one rb_drop

    def _new(self, *shape, dtype=None):
        return torch.empty(shape, dtype=dtype or self.dtype, device=self.device)

    def outputs(self, rows, total=False):
        """Tensors for forward(..., out=...), which looks at these no further."""
        f32 = torch.float32
        out = _NormOutputs(self._new(rows, self.width), self._new(rows, self.width) if total else None, self._new(rows, dtype=f32), self._new(rows, dtype=f32))
        out.norm, out.rows = self, rows
        return out

    def gradients(self, rows, bias=True, drop=False):
        """Tensors for grad(..., out=...), which looks at these no further."""
        out = _NormGradients(self._new(rows, self.width), self._new(rows, self.width) if drop else None, self._new(self.width, dtype=self.weight_dtype),
                             self._new(self.width, dtype=self.weight_dtype) if bias else None)
        out.norm, out.rows = self, rows
        return out

    def _rows(self, t, rows, what):
        """Elements between the rows of a tensor that is looked at first."""
        n, stride = _rows_of(t, self.width, self.dtype, self._index, what)
        assert n == rows, what
        return stride

    def _weights(self, t, what):
        assert t is None or _fits(t, self.weight_dtype, self._index, (self.width,)), what
        return t

    def forward(self, x, weight, bias=None, residual=None, drop=None, out=None):
        """Normed of x, or of residual + dropout(x); into `out` if given (see outputs; its y or total may be x, its total the residual)."""
        rows, width = x.shape[0], self.width
        theirs, sums = out is not None, residual is not None or drop is not None
        if out is None:
            out = self.outputs(rows, total=sums)
        assert (out[1] is not None) == sums, "out.total"
        y, total, mean, rstd = out
        if type(out) is _NormOutputs and out.norm is self and out.rows == rows:
            y_stride = total_stride = width
        else:
            y_stride = self._rows(y, rows, "out.y")
            total_stride = self._rows(total, rows, "out.total") if sums else 0
            for t, name in ((mean, "out.mean"), (rstd, "out.rstd")):
                assert t is None or _fits(t, torch.float32, self._index, (rows,)), name
        x_stride = self._rows(x, rows, "x")
        self._weights(weight, "weight")
        self._weights(bias, "bias")
        residual_stride = 0 if residual is None else self._rows(residual, rows, "residual")
        if rows == 0:
            return out
        p, seed, step = (0.0, 0, 0) if drop is None else drop
        at = self._structures.fill(x.data_ptr(), x_stride, 0 if residual is None else residual.data_ptr(), residual_stride, total.data_ptr() if sums else 0, total_stride,
                                   y.data_ptr(), y_stride, 0, 0, p, seed & _M64, step & _M64)
        _check(self._on_stream(rb_norm_forward, self.handle, at, None if residual is None else at + 16, None if drop is None else at + 80, rows, weight, bias,
                               at + 32 if sums else None, at + 48, mean, rstd), "rb_norm_forward")
        if theirs:
            _written([t for t in out if t is not None])
        return out

    def grad(self, grad_y, total, weight, mean, rstd, grad_total=None, drop=None, bias=True, out=None):
        """NormGrads from the derivatives with respect to y and (or None) total; total: forward's, or x where that was None.  bias: whether that gradient is
        wanted; into `out` if given (see gradients; its total or x may be grad_y or grad_total, its weight or bias None)."""
        rows, width = total.shape[0], self.width
        theirs = out is not None
        if out is None:
            out = self.gradients(rows, bias=bias, drop=drop is not None)
        assert (out[1] is not None) == (drop is not None), "out.x"
        g_total, g_x, g_weight, g_bias = out
        if type(out) is _NormGradients and out.norm is self and out.rows == rows:
            g_stride = x_stride = width
        else:
            g_stride = self._rows(g_total, rows, "out.total")
            x_stride = 0 if g_x is None else self._rows(g_x, rows, "out.x")
            self._weights(g_weight, "out.weight")
            self._weights(g_bias, "out.bias")
        strides = self._rows(grad_y, rows, "grad_y"), self._rows(total, rows, "total"), 0 if grad_total is None else self._rows(grad_total, rows, "grad_total")
        self._weights(weight, "weight")
        for t, name in ((mean, "mean"), (rstd, "rstd")):
            assert _fits(t, torch.float32, self._index, (rows,)), name
        if rows == 0:
            for t in (g_weight, g_bias):
                if t is not None:
                    t.zero_()
            return out
        p, seed, step = (0.0, 0, 0) if drop is None else drop
        at = self._structures.fill(grad_y.data_ptr(), strides[0], total.data_ptr(), strides[1], 0 if grad_total is None else grad_total.data_ptr(), strides[2],
                                   g_total.data_ptr(), g_stride, 0 if g_x is None else g_x.data_ptr(), x_stride, p, seed & _M64, step & _M64)
        _check(self._on_stream(rb_norm_grad, self.handle, at, at + 16, None if grad_total is None else at + 32, mean, rstd, None if drop is None else at + 80, rows, weight,
                               at + 48, None if g_x is None else at + 64, g_weight, g_bias), "rb_norm_grad")
        if theirs:
            _written([t for t in out if t is not None])
        return out

    def __call__(self, x, weight, bias=None, residual=None, drop=None):
        return Normed(*_Norm.apply(x, weight, bias, residual, drop, self))

    def close(self):
        if getattr(self, "handle", None):
            rb_norm_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, drop, norm):
        o = norm.forward(x, weight, bias, residual, drop)
        ctx.norm, ctx.drop, ctx.residual, ctx.bias = norm, drop, residual is not None, bias is not None
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(x if o.total is None else o.total, weight, o.mean, o.rstd)
        ctx.mark_non_differentiable(o.mean, o.rstd)
        return tuple(o)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_y, grad_total, _mean, _rstd):
        total, weight, mean, rstd = ctx.saved_tensors
        norm = ctx.norm
        if grad_y is None and grad_total is None:
            return (None,) * 6
        if grad_y is None:
            grad_y = torch.zeros(total.shape, dtype=norm.dtype, device=norm.device)
        grad_y, grad_total = (t if t is None or (t.stride(1) == 1 and t.stride(0) >= t.shape[1]) else t.contiguous() for t in (grad_y, grad_total))
        wanted = ctx.needs_input_grad
        g = norm.grad(grad_y, total, weight, mean, rstd, grad_total, ctx.drop, bias=ctx.bias and wanted[2])
        return g.total if ctx.drop is None else g.x, g.weight if wanted[1] else None, g.bias, g.total if ctx.residual else None, None, None


# ---- attention of packed documents -------------------------------------------------

class Documents(NamedTuple):
    """Where the documents of packed rows lie, int64 on the device: document d begins at position offsets[d] and ends before offsets[d + 1] (or after lengths[d]
    positions); all of it sees its first prefixes[d] positions.  Empty documents are documents: with more than one for each 128 positions (padded offsets) a call
    takes the forms for short ones, which are slower for long ones."""
    offsets: torch.Tensor                      # [documents + 1]
    lengths: Optional[torch.Tensor] = None     # [documents]
    prefixes: Optional[torch.Tensor] = None    # [documents]


class Attended(NamedTuple):
    """What DocumentAttention.forward gives."""
    out: torch.Tensor                      # [tokens, heads, head_dim], bfloat16
    lse: torch.Tensor                      # [heads, tokens], binary32


class _AttendedOutputs(Attended):
    """Attended's tensors that DocumentAttention.outputs has made: `attention` and `tokens` say for what."""
    attention = tokens = None


_NO_HEADS = (0, 0, 0) * 4


class DocumentAttention(_OnStream):
    """Attention of packed documents, and its gradients.  One handle serves all layers of a form, and one host thread at a time.

    attention = DocumentAttention(16, 128, kv_heads=4, max_tokens=8192)            # bfloat16; causal, no cap
    documents = Documents(torch.tensor([0, 700, 1500], device="cuda"))
    out = attention(q, k, v, documents)                                             # [tokens, heads, head_dim], with gradients of q, k and v
    o = attention.forward(q, k, v, documents)                                       # Attended; q, k, v [tokens, heads, head_dim] may be views of one tensor
    """

    def __init__(self, heads, head_dim, kv_heads=None, max_tokens=8192, causal=True, scale=None, cap=0.0, device="cuda"):
        kv_heads = heads if kv_heads is None else kv_heads
        scale = float(head_dim) ** -0.5 if scale is None else scale
        rc, self.handle = rb_attention_create(heads, kv_heads, head_dim, max_tokens, causal, scale, cap)
        _check(rc, "rb_attention_create")
        self.heads, self.kv_heads, self.head_dim, self.max_tokens = int(heads), int(kv_heads), int(head_dim), int(max_tokens)
        self._bind_device(device)
        rc, size = rb_attention_query(self.handle)
        _check(rc, "rb_attention_query")
        self.workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(rb_attention_bind(self.handle, self.workspace), "rb_attention_bind")
        self._structures = _Structures("=" + "Qqq" * 8 + "QQQq")       # eight rb_heads, one rb_documents

    def outputs(self, tokens):
        """Tensors for forward(..., out=...), which looks at these no further."""
        out = _AttendedOutputs(torch.empty((tokens, self.heads, self.head_dim), dtype=torch.bfloat16, device=self.device),
                               torch.empty((self.heads, tokens), dtype=torch.float32, device=self.device))
        out.attention, out.tokens = self, tokens
        return out

    def _heads(self, t, tokens, heads, what):
        """The structure's numbers of a tensor that is looked at first."""
        assert t.shape == (tokens, heads, self.head_dim) and t.dtype is torch.bfloat16 and t.get_device() == self._index, what
        a, b, step = t.stride()
        assert step == 1 or tokens == 0, what
        # (strides that are never used may be anything)
        return t.data_ptr(), a if tokens > 1 else heads * self.head_dim, b if heads > 1 else self.head_dim

    def _documents(self, d):
        offsets, lengths, prefixes = d
        count, index, i64 = offsets.shape[0] - 1, self._index, torch.int64
        assert count >= 0 and _fits(offsets, i64, index, (count + 1,)), "documents.offsets"
        assert lengths is None or _fits(lengths, i64, index, (count,)), "documents.lengths"
        assert prefixes is None or _fits(prefixes, i64, index, (count,)), "documents.prefixes"
        return offsets.data_ptr(), 0 if lengths is None else lengths.data_ptr(), 0 if prefixes is None else prefixes.data_ptr(), count

    def _slopes(self, slopes):
        assert slopes is None or _fits(slopes, torch.float32, self._index, (self.heads,)), "slopes"
        return slopes

    def forward(self, q, k, v, documents, slopes=None, out=None):
        """Attended; into `out` if given (see outputs; its lse may be None)."""
        tokens, heads, kv = q.shape[0], self.heads, self.kv_heads
        theirs = out is not None
        if out is None:
            out = self.outputs(tokens)
        result, lse = out
        if type(out) is _AttendedOutputs and out.attention is self and out.tokens == tokens:
            to = result.data_ptr(), heads * self.head_dim, self.head_dim
        else:
            assert lse is None or _fits(lse, torch.float32, self._index, (heads, tokens)), "out.lse"
            to = self._heads(result, tokens, heads, "out.out")
        at = self._structures.fill(*self._heads(q, tokens, heads, "q"), *self._heads(k, tokens, kv, "k"), *self._heads(v, tokens, kv, "v"), *to, *_NO_HEADS,
                                   *self._documents(documents))
        self._slopes(slopes)
        if tokens == 0:
            return out
        _check(self._on_stream(rb_attention_forward, self.handle, at, at + 24, at + 48, tokens, at + 192, slopes, at + 72, lse), "rb_attention_forward")
        if theirs:
            _written([t for t in out if t is not None])
        return out

    def grad(self, q, k, v, documents, out_, lse, grad_out, slopes=None, out=None):
        """The gradients of q, k and v from the derivatives with respect to out; out_, lse: forward's.  Into the three tensors `out` if given."""
        tokens, heads, kv = q.shape[0], self.heads, self.kv_heads
        theirs = out is not None
        if out is None:
            out = tuple(torch.empty((tokens, n, self.head_dim), dtype=torch.bfloat16, device=self.device) for n in (heads, kv, kv))
        assert _fits(lse, torch.float32, self._index, (heads, tokens)), "lse"
        at = self._structures.fill(*self._heads(q, tokens, heads, "q"), *self._heads(k, tokens, kv, "k"), *self._heads(v, tokens, kv, "v"),
                                   *self._heads(out_, tokens, heads, "out_"), *self._heads(grad_out, tokens, heads, "grad_out"),
                                   *self._heads(out[0], tokens, heads, "out[0]"), *self._heads(out[1], tokens, kv, "out[1]"), *self._heads(out[2], tokens, kv, "out[2]"),
                                   *self._documents(documents))
        self._slopes(slopes)
        if tokens == 0:
            return out
        _check(self._on_stream(rb_attention_grad, self.handle, at, at + 24, at + 48, tokens, at + 192, slopes, at + 72, lse, at + 96, at + 120, at + 144, at + 168),
               "rb_attention_grad")
        if theirs:
            _written(list(out))
        return out

    def __call__(self, q, k, v, documents, slopes=None):
        return _Attend.apply(q, k, v, *documents, slopes, self)

    def close(self):
        if getattr(self, "handle", None):
            rb_attention_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


class _Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, offsets, lengths, prefixes, slopes, attention):
        o = attention.forward(q, k, v, Documents(offsets, lengths, prefixes), slopes)
        ctx.attention = attention
        ctx.save_for_backward(q, k, v, offsets, lengths, prefixes, slopes, *o)
        return o.out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_out):
        q, k, v, offsets, lengths, prefixes, slopes, out, lse = ctx.saved_tensors
        if grad_out.stride(2) != 1 or grad_out.data_ptr() % 16 or any(s % 8 for s in grad_out.stride()[:2]):
            grad_out = grad_out.contiguous()
        g = ctx.attention.grad(q, k, v, Documents(offsets, lengths, prefixes), out, lse, grad_out, slopes)
        return (*g, None, None, None, None, None)

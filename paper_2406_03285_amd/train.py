"""Thin binding of the C ABI in include/rb_train.h: what a training program computes at the augmented mini-batch.

As in binding.py every function has the name and argument order of its C counterpart, and the classes only own device memory, keep a
handle, look at what they are given and raise RbError on a non-zero status.  There is no fallback: if librb_train.so is missing the import fails.
"""
import ctypes as C
import math
import os
from typing import NamedTuple, Optional

import torch

from .binding import Call, HERE, RB_BF16, RB_F32, _check, _ptr, _stream

TRAIN_LIB_PATH = os.environ.get("RB_TRAIN_LIBRARY") or os.path.join(HERE, "librb_train.so")   # RB_TRAIN_LIBRARY: another build of the same library

RB_MAX_VOCAB, RB_MAX_ROWS, RB_MAX_GIVEN, RB_MAX_TOP = 1 << 28, 1 << 23, 64, 64
RB_MAX_DIM, RB_MAX_MATRICES, RB_MAX_ORTHO_STEPS = 65536, 65535, 16

TRAIN_EXPORTS = (
    "rb_scorer_create", "rb_scorer_query", "rb_scorer_bind", "rb_scorer_score", "rb_scorer_grad", "rb_scorer_destroy",
    "rb_ortho_create", "rb_ortho_query", "rb_ortho_bind", "rb_ortho_apply", "rb_ortho_step", "rb_ortho_destroy",
)

__all__ = ["TRAIN_EXPORTS", "TRAIN_LIB_PATH", "RB_MAX_VOCAB", "RB_MAX_ROWS", "RB_MAX_GIVEN", "RB_MAX_TOP", "RB_MAX_DIM", "RB_MAX_MATRICES",
           "RB_MAX_ORTHO_STEPS", "NEWTON_SCHULZ", "Scores", "TokenScorer", "Orthogonalizer", *TRAIN_EXPORTS]


def _load():
    if not os.path.exists(TRAIN_LIB_PATH):
        raise ImportError(
            f"{TRAIN_LIB_PATH} is missing: build it with `python paper_2406_03285_amd/build.py` "
            "(there is no fallback path)")
    L = C.CDLL(TRAIN_LIB_PATH)
    vp, i64, i32, sz, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t, C.c_float
    L.rb_scorer_create.argtypes = [C.POINTER(vp), i64, i32, i64, i64]
    L.rb_scorer_query.argtypes = [vp, C.POINTER(sz)]
    L.rb_scorer_bind.argtypes = [vp, vp, vp]
    L.rb_scorer_score.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, vp]
    L.rb_scorer_grad.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, i64, vp]
    L.rb_scorer_destroy.argtypes = [vp]
    L.rb_ortho_create.argtypes = [C.POINTER(vp), i64, i64, i64, i32, i32, C.POINTER(f32), i64, f32]
    L.rb_ortho_query.argtypes = [vp, C.POINTER(sz)]
    L.rb_ortho_bind.argtypes = [vp, vp]
    L.rb_ortho_apply.argtypes = [vp, vp, i64, i64, vp, i64, i64, vp]
    L.rb_ortho_step.argtypes = [vp, vp, i64, i64, vp, i64, i64, vp, f32, f32, i32, f32, f32, vp]
    L.rb_ortho_destroy.argtypes = [vp]
    for name in TRAIN_EXPORTS:
        getattr(L, name).restype = C.c_int
    return L


_L = _load()


def _native(general, layout):
    """As in binding.py: the same function with its usual arguments marshalled natively."""
    if Call is None:
        return general
    return Call(C.cast(getattr(_L, general.__name__), C.c_void_p).value, layout, general)


def rb_scorer_create(vocab, dtype, given, top):
    h = C.c_void_p()
    rc = _L.rb_scorer_create(C.byref(h), int(vocab), int(dtype), int(given), int(top))
    return rc, h.value


def rb_scorer_query(s):
    n = C.c_size_t()
    rc = _L.rb_scorer_query(s, C.byref(n))
    return rc, n.value


def rb_scorer_bind(s, workspace, hip_stream=None):
    return _L.rb_scorer_bind(s, _ptr(workspace), _stream(hip_stream))


def rb_scorer_score(s, logits, rows, row_stride, tokens, logp, lse, entropy, top_logp, top_ids, hip_stream=None):
    return _L.rb_scorer_score(s, _ptr(logits), int(rows), int(row_stride), _ptr(tokens), _ptr(logp), _ptr(lse), _ptr(entropy),
                              _ptr(top_logp), _ptr(top_ids), _stream(hip_stream))


def rb_scorer_grad(s, logits, rows, row_stride, tokens, lse, entropy, grad_logp, grad_entropy, grad_logits, grad_stride, hip_stream=None):
    return _L.rb_scorer_grad(s, _ptr(logits), int(rows), int(row_stride), _ptr(tokens), _ptr(lse), _ptr(entropy), _ptr(grad_logp),
                             _ptr(grad_entropy), _ptr(grad_logits), int(grad_stride), _stream(hip_stream))


def rb_scorer_destroy(s):
    return _L.rb_scorer_destroy(s)


def rb_ortho_create(matrices, m, n, dtype, out_dtype, coefficients, eps):
    """coefficients: a sequence of (a, b, c), one per step."""
    h = C.c_void_p()
    flat = [float(v) for abc in coefficients for v in abc]
    rc = _L.rb_ortho_create(C.byref(h), int(matrices), int(m), int(n), int(dtype), int(out_dtype), (C.c_float * len(flat))(*flat),
                            len(flat) // 3, float(eps))
    return rc, h.value


def rb_ortho_query(o):
    n = C.c_size_t()
    rc = _L.rb_ortho_query(o, C.byref(n))
    return rc, n.value


def rb_ortho_bind(o, workspace):
    return _L.rb_ortho_bind(o, _ptr(workspace))


def rb_ortho_apply(o, update, update_matrix_stride, update_row_stride, out, out_matrix_stride, out_row_stride, hip_stream=None):
    return _L.rb_ortho_apply(o, _ptr(update), int(update_matrix_stride), int(update_row_stride), _ptr(out), int(out_matrix_stride),
                             int(out_row_stride), _stream(hip_stream))


def rb_ortho_step(o, weight, weight_matrix_stride, weight_row_stride, grad, grad_matrix_stride, grad_row_stride, momentum, lr, beta,
                  nesterov, weight_decay, scale, hip_stream=None):
    return _L.rb_ortho_step(o, _ptr(weight), int(weight_matrix_stride), int(weight_row_stride), _ptr(grad), int(grad_matrix_stride),
                            int(grad_row_stride), _ptr(momentum), float(lr), float(beta), int(nesterov), float(weight_decay),
                            float(scale), _stream(hip_stream))


def rb_ortho_destroy(o):
    return _L.rb_ortho_destroy(o)


rb_scorer_score = _native(rb_scorer_score, "hpiipppppps")
rb_scorer_grad = _native(rb_scorer_grad, "hpiippppppis")
rb_ortho_apply = _native(rb_ortho_apply, "hpiipiis")

try:
    from torch._C import _cuda_getCurrentRawStream as _current_stream      # (the address alone: a Stream object takes the host some us)
except ImportError:
    def _current_stream(index):
        return torch.cuda.current_stream(index).cuda_stream


def _fits(t, dtype, index, shape):
    """Whether t is a contiguous tensor of that type and shape on the device of that index."""
    return t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous()


_CODES = {torch.float32: RB_F32, torch.bfloat16: RB_BF16}


_written = torch.autograd.graph.increment_version       # tells autograd, which may have saved them, of tensors that a call has written


class _OnStream:
    """Calls go to the current stream of the handle's device; a call on another stream than the last one's waits for that, since the two
    share the workspace.  The allocator is told of every stream that the workspace was used on, so that it is not another tensor's before these are
    done with it.  A captured call is ordered by its graph: whoever replays it orders the replays and the handle's other calls, and keeps the
    handle as long as the graph."""

    def _bind_device(self, device):
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        self._index = self.device.index
        self._last = torch.cuda.current_stream(self.device)
        self._last_address = self._last.cuda_stream

    def _on_stream(self, call, *args):
        address = _current_stream(self._index)
        if address != self._last_address and not torch.cuda.is_current_stream_capturing():
            stream = torch.cuda.current_stream(self.device)
            stream.wait_stream(self._last)
            self.workspace.record_stream(stream)
            self._last, self._last_address = stream, address
        if torch.cuda.current_device() == self._index:
            return call(*args, address)
        with torch.cuda.device(self.device):
            return call(*args, address)


class Scores(NamedTuple):
    """What TokenScorer.score gives, binary32 but for the indices; the last two are None without alternatives, logp without given tokens."""
    logp: Optional[torch.Tensor]           # [rows, given]
    lse: torch.Tensor                      # [rows]
    entropy: torch.Tensor                  # [rows]
    top_logp: Optional[torch.Tensor]       # [rows, top]
    top_ids: Optional[torch.Tensor]        # [rows, top] int64


class _Outputs(Scores):
    """Scores' tensors that TokenScorer.outputs has made: `scorer` and `rows` say for what (of one that was changed since: for none)."""
    scorer = rows = None


class TokenScorer(_OnStream):
    """Log probabilities of given tokens under rows of logits, the rows' entropy and top alternatives, and their gradient.

    scorer = TokenScorer(vocab, torch.bfloat16, given=1, top=8)
    s = scorer.score(logits, tokens)                # Scores; logits [rows, vocab], rows may be strided; tokens [rows, given] (or [rows])
    s = scorer(logits, tokens)                      # the same within autograd: s.logp and s.entropy carry gradients
                                                    # (s.lse, s.top_logp and s.top_ids carry none: what a loss adds of them changes no gradient)
    """

    def __init__(self, vocab, dtype=torch.float32, given=1, top=0, device="cuda"):
        rc, self.handle = rb_scorer_create(vocab, _CODES[dtype], given, top)
        _check(rc, "rb_scorer_create")
        self.vocab, self.dtype, self.given, self.top = int(vocab), dtype, int(given), int(top)
        self._bind_device(device)
        rc, size = rb_scorer_query(self.handle)
        _check(rc, "rb_scorer_query")
        self.workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(self._on_stream(rb_scorer_bind, self.handle, self.workspace), "rb_scorer_bind")

    def outputs(self, rows):
        """Tensors for score(..., out=...), which looks at these no further."""
        def new(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=self.device)
        out = _Outputs(new(rows, self.given) if self.given else None, new(rows), new(rows), new(rows, self.top) if self.top else None,
                       new(rows, self.top, dtype=torch.int64) if self.top else None)
        out.scorer, out.rows = self, rows
        return out

    def _rows(self, logits, what):
        """(rows, elements between them) of a tensor of the logits' form, looked at first."""
        shape, (stride, step) = logits.shape, logits.stride()
        assert len(shape) == 2 and shape[1] == self.vocab and logits.dtype == self.dtype and logits.get_device() == self._index, what
        assert step == 1 or self.vocab == 1, what
        return shape[0], stride if shape[0] > 1 else max(stride, self.vocab)

    def _given(self, t, rows, dtype, what):
        """A tensor of given tokens' form: [rows, given], or [rows] of one."""
        assert _fits(t, dtype, self._index, (rows, self.given)) or (self.given == 1 and _fits(t, dtype, self._index, (rows,))), what
        return t

    def score(self, logits, tokens=None, out=None):
        """Scores of every row of logits; into `out` if given (see outputs)."""
        rows, stride = self._rows(logits, "logits")
        if self.given:
            self._given(tokens, rows, torch.int64, "tokens")
        theirs = out is not None
        if out is None:
            out = self.outputs(rows)
        elif type(out) is not _Outputs or out.scorer is not self or out.rows != rows:
            f32, index = torch.float32, self._index
            assert out.lse is None or _fits(out.lse, f32, index, (rows,)), "out.lse"
            assert out.entropy is None or _fits(out.entropy, f32, index, (rows,)), "out.entropy"
            assert not self.given or _fits(out.logp, f32, index, (rows, self.given)), "out.logp"
            assert not self.top or (_fits(out.top_logp, f32, index, (rows, self.top)) and _fits(out.top_ids, torch.int64, index, (rows, self.top))), "out.top"
        if rows == 0:
            return out
        logp, lse, entropy, top_logp, top_ids = out
        if not self.given:
            tokens = logp = None
        if not self.top:
            top_logp = top_ids = None
        _check(self._on_stream(rb_scorer_score, self.handle, logits, rows, stride, tokens, logp, lse, entropy, top_logp, top_ids), "rb_scorer_score")
        if theirs:
            _written([t for t in (logp, lse, entropy, top_logp, top_ids) if t is not None])
        return out

    def grad(self, logits, tokens, lse, entropy, grad_logp, grad_entropy=None, out=None):
        """The gradient with respect to the logits, from the derivatives with respect to logp [rows, given] and entropy [rows] (or None).
        out: a tensor shaped as the logits (rows may be strided), which the logits themselves may be.  Without it the rows lie behind each other, as in
        backward: where those of the logits lie otherwise relative to 16 bytes, a tensor laid out like the logits is written faster."""
        rows, stride = self._rows(logits, "logits")
        theirs = out is not None
        if out is None:
            out = torch.empty((rows, self.vocab), dtype=self.dtype, device=self.device)
        out_rows, out_stride = self._rows(out, "out")
        assert out_rows == rows, "out"
        assert _fits(lse, torch.float32, self._index, (rows,)), "lse"
        if self.given:
            self._given(tokens, rows, torch.int64, "tokens")
            self._given(grad_logp, rows, torch.float32, "grad_logp")
        else:
            tokens = grad_logp = None
        if grad_entropy is None:
            entropy = None
        else:
            assert _fits(entropy, torch.float32, self._index, (rows,)), "entropy"
            assert _fits(grad_entropy, torch.float32, self._index, (rows,)), "grad_entropy"
        if rows == 0:
            return out
        _check(self._on_stream(rb_scorer_grad, self.handle, logits, rows, stride, tokens, lse, entropy, grad_logp, grad_entropy, out, out_stride),
               "rb_scorer_grad")
        if theirs:
            _written(out)
        return out

    def __call__(self, logits, tokens=None):
        return Scores(*_Score.apply(logits, tokens, self))

    def close(self):
        if getattr(self, "handle", None):
            rb_scorer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()


class _Score(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, scorer):
        s = scorer.score(logits, tokens)
        ctx.scorer = scorer
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, tokens, s.lse, s.entropy)
        ctx.mark_non_differentiable(*[t for t in (s.lse, s.top_logp, s.top_ids) if t is not None])
        return tuple(s)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_logp, _lse, grad_entropy, _top_logp, _top_ids):
        logits, tokens, lse, entropy = ctx.saved_tensors
        scorer = ctx.scorer
        if grad_logp is None and grad_entropy is None:
            return None, None, None
        if grad_logp is None and scorer.given:
            grad_logp = lse.new_zeros((logits.shape[0], scorer.given))
        return scorer.grad(logits, tokens, lse, entropy, None if grad_logp is None else grad_logp.contiguous(),
                           None if grad_entropy is None else grad_entropy.contiguous()), None, None


#: The usual coefficients of one Newton-Schulz step: they bring singular values from about 0.01 to 1 near 1 in five steps.
NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


class Orthogonalizer(_OnStream):
    """Updates orthogonalised by Newton-Schulz products, for `batch` matrices of m x n at a time.

    ortho = Orthogonalizer(1024, 4096, dtype=torch.bfloat16, out_dtype=torch.float32)
    ortho.orthogonalize(update)                                  # [m, n] or [batch, m, n] -> the same of out_dtype
    ortho.step(weight, grad, momentum, lr=0.02)                  # the optimiser step around it, in place
    """

    def __init__(self, m, n, batch=1, dtype=torch.float32, out_dtype=None, coefficients=(NEWTON_SCHULZ,) * 5, eps=1e-7, device="cuda"):
        self.out_dtype = dtype if out_dtype is None else out_dtype
        rc, self.handle = rb_ortho_create(batch, m, n, _CODES[dtype], _CODES[self.out_dtype], coefficients, eps)
        _check(rc, "rb_ortho_create")
        self.m, self.n, self.batch, self.dtype = int(m), int(n), int(batch), dtype
        self._bind_device(device)
        rc, size = rb_ortho_query(self.handle)
        _check(rc, "rb_ortho_query")
        self.workspace = torch.empty(size, dtype=torch.uint8, device=self.device)
        _check(rb_ortho_bind(self.handle, self.workspace), "rb_ortho_bind")

    def _strides(self, t, dtype):
        """(matrix stride, row stride) of a tensor that is looked at first."""
        assert t.dtype == dtype and t.device == self.device
        assert t.shape == (self.batch, self.m, self.n) or (self.batch == 1 and t.shape == (self.m, self.n))
        assert t.stride(-1) == 1 or self.n == 1
        return (t.stride(0) if t.dim() == 3 and self.batch > 1 else 0), (t.stride(-2) if self.m > 1 else self.n)

    def orthogonalize(self, update, out=None):
        a = self._strides(update, self.dtype)
        theirs = out is not None
        if out is None:
            out = torch.empty(update.shape, dtype=self.out_dtype, device=self.device)
        b = self._strides(out, self.out_dtype)
        _check(self._on_stream(rb_ortho_apply, self.handle, update, *a, out, *b), "rb_ortho_apply")
        if theirs:
            _written(out)
        return out

    def step(self, weight, grad, momentum, lr, beta=0.95, nesterov=True, weight_decay=0.0, scale=None):
        """momentum <- beta momentum + grad; weight <- (1 - lr weight_decay) weight - lr scale O, O the orthogonalised grad + beta momentum
        (nesterov) or momentum.  scale: None - sqrt(max(1, m / n))."""
        w, g = self._strides(weight, self.out_dtype), self._strides(grad, self.dtype)
        assert momentum.shape == weight.shape and momentum.dtype == torch.float32 and momentum.is_contiguous() and momentum.device == self.device
        if scale is None:
            scale = math.sqrt(max(1.0, self.m / self.n))
        _check(self._on_stream(rb_ortho_step, self.handle, weight, *w, grad, *g, momentum, lr, beta, nesterov, weight_decay, scale), "rb_ortho_step")
        _written((weight, momentum))

    def close(self):
        if getattr(self, "handle", None):
            rb_ortho_destroy(self.handle)
            self.handle = None

    def __del__(self):
        self.close()

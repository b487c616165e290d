"""What LayerNorm, dropout and DocumentAttention do on the host around a call, without a GPU: the calls themselves do nothing here."""
import ctypes as C
import inspect

import pytest
import torch

import paper_2406_03285_amd as rb
from paper_2406_03285_amd import binding, block

CALLED = []


@pytest.fixture(autouse=True)
def no_device(monkeypatch):
    CALLED.clear()
    for kind in (rb.LayerNorm, rb.DocumentAttention):
        monkeypatch.setattr(kind, "_on_stream", lambda self, call, *args: CALLED.append((call, args)) or rb.RB_OK)


def norm_of(width, dtype=torch.float32, weight_dtype=torch.float32):
    n = object.__new__(rb.LayerNorm)
    n.handle, n.width, n.dtype, n.weight_dtype, n.device, n._index = None, width, dtype, weight_dtype, torch.device("cpu"), -1
    n._structures = block._Structures("=QqQqQqQqQqdQQ")
    return n


def attention_of(heads, kv, dim):
    a = object.__new__(rb.DocumentAttention)
    a.handle, a.heads, a.kv_heads, a.head_dim, a.device, a._index = None, heads, kv, dim, torch.device("cpu"), -1
    a._structures = block._Structures("=" + "Qqq" * 8 + "QQQq")
    return a


def rows_at(address):
    r = rb.RbRows.from_address(address)
    return r.data, r.stride


def test_norm_passes_its_tensors():
    n = norm_of(7)
    x, r, w, b = torch.zeros((4, 9))[:, :7], torch.zeros((4, 7)), torch.zeros(7), torch.zeros(7)
    o = n.forward(x, w, b, residual=r, drop=rb.Drop(0.25, -1, 5))
    (_, args), = CALLED
    assert rows_at(args[1]) == (x.data_ptr(), 9) and rows_at(args[2]) == (r.data_ptr(), 7) and rows_at(args[7]) == (o.total.data_ptr(), 7)
    assert rows_at(args[8]) == (o.y.data_ptr(), 7) and args[4:7] == (4, w, b) and args[9:] == (o.mean, o.rstd)
    d = rb.RbDrop.from_address(args[3])
    assert (d.p, d.seed, d.step) == (0.25, 2 ** 64 - 1, 5)
    CALLED.clear()
    o = n.forward(x, w)
    assert o.total is None and CALLED[0][1][2:4] == (None, None) and CALLED[0][1][7] is None
    CALLED.clear()
    g = n.grad(r, x, w, o.mean, o.rstd, grad_total=r, drop=rb.Drop(0.5, 1, 2), bias=False)
    args = CALLED[0][1]
    assert [rows_at(args[i]) for i in (1, 2, 3, 9, 10)] == [(r.data_ptr(), 7), (x.data_ptr(), 9), (r.data_ptr(), 7), (g.total.data_ptr(), 7), (g.x.data_ptr(), 7)]
    assert args[11] is g.weight and args[12] is None and g.bias is None and args[4:6] == (o.mean, o.rstd)


def test_norm_looks_at_its_arguments():
    n = norm_of(7)
    x, w = torch.zeros((4, 7)), torch.zeros(7)
    o = n.forward(x, w)
    for bad in (dict(x=torch.zeros((4, 8))), dict(x=torch.zeros((4, 7), dtype=torch.bfloat16)), dict(x=torch.zeros((7, 4)).t()), dict(weight=torch.zeros(8)),
                dict(weight=torch.zeros(14)[::2]), dict(bias=torch.zeros(7, dtype=torch.float64)), dict(residual=torch.zeros((5, 7))), dict(out=n.outputs(4, total=True)),
                dict(out=n.outputs(5)), dict(out=n.outputs(4)._replace(mean=torch.zeros(5))), dict(residual=x, out=n.outputs(4)), dict(out=norm_of(7).outputs(5))):
        with pytest.raises(AssertionError):
            n.forward(**{**dict(x=x, weight=w), **bad})
    good = dict(grad_y=x, total=x, weight=w, mean=o.mean, rstd=o.rstd)
    for bad in (dict(grad_y=torch.zeros((4, 8))), dict(total=torch.zeros((3, 7))), dict(mean=torch.zeros(3)), dict(rstd=torch.zeros(4, dtype=torch.float64)), dict(weight=torch.zeros(6)),
                dict(grad_total=torch.zeros((4, 6))), dict(out=n.gradients(4, drop=True)), dict(drop=rb.Drop(0.1, 1, 1), out=n.gradients(4)), dict(out=n.gradients(3)),
                dict(out=n.gradients(4)._replace(weight=torch.zeros(6)))):
        with pytest.raises(AssertionError):
            n.grad(**{**good, **bad})


def test_attention_passes_its_tensors_and_looks_at_them():
    a = attention_of(4, 2, 16)
    whole = torch.zeros((10, 128), dtype=torch.bfloat16)
    q, k, v = (x.unflatten(1, (-1, 16)) for x in whole.split([64, 32, 32], 1))
    docs = rb.Documents(torch.tensor([0, 4, 10]), None, torch.tensor([1, 2]))
    slopes = torch.zeros(4)
    o = a.forward(q, k, v, docs, slopes=slopes)
    args = CALLED[0][1]

    def heads_at(address):
        h = rb.RbHeads.from_address(address)
        return h.data, h.token_stride, h.head_stride
    assert [heads_at(args[i]) for i in (1, 2, 3, 7)] == [(x.data_ptr(), 128, 16) for x in (q, k, v)] + [(o.out.data_ptr(), 64, 16)]
    d = rb.RbDocuments.from_address(args[5])
    assert (d.offsets, d.lengths, d.prefixes, d.count) == (docs.offsets.data_ptr(), None, docs.prefixes.data_ptr(), 2) and args[4] == 10 and args[6] is slopes and args[8] is o.lse
    CALLED.clear()
    g = a.grad(q, k, v, docs, o.out, o.lse, o.out)
    args = CALLED[0][1]
    assert [heads_at(args[i])[0] for i in (1, 2, 3, 7, 9, 10, 11, 12)] == [x.data_ptr() for x in (q, k, v, o.out, o.out, *g)] and args[8] is o.lse
    for bad in (dict(q=k), dict(k=q), dict(q=q.float()), dict(v=v[:9]), dict(documents=rb.Documents(torch.tensor([0, 4], dtype=torch.int32))),
                dict(documents=rb.Documents(torch.tensor([0, 4]), torch.tensor([1, 2]))), dict(documents=rb.Documents(torch.tensor([0, 4, 10]), None, torch.tensor([1]))),
                dict(slopes=torch.zeros(3)), dict(out=a.outputs(9)), dict(q=whole.unflatten(1, (-1, 16))[:, :4].transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(AssertionError):
            a.forward(**{**dict(q=q, k=k, v=v, documents=docs), **bad})
    with pytest.raises(AssertionError):
        a.grad(q, k, v, docs, o.out, o.lse[:, :9], o.out)
    with pytest.raises(AssertionError):
        rb.dropout(torch.zeros((3, 4)), rb.Drop(0.1, 1, 1))            # not on a GPU


def test_what_is_written_is_a_new_version():
    n, a = norm_of(7), attention_of(1, 1, 8)
    x, w = torch.zeros((4, 7)), torch.zeros(7)
    for out in (n.outputs(4, total=True), rb.Normed(*n.outputs(4, total=True))):
        n.forward(x, w, residual=x, out=out)
        assert [t._version for t in out] == [1] * 4 and x._version == w._version == 0
    out = n.gradients(4)
    n.grad(x, x, w, torch.zeros(4), torch.zeros(4), out=out)
    assert [t._version for t in out if t is not None] == [1] * 3
    q, docs = torch.zeros((3, 1, 8), dtype=torch.bfloat16), rb.Documents(torch.tensor([0, 3]))
    o = a.outputs(3)
    a.forward(q, q, q, docs, out=o)
    grads = tuple(torch.zeros_like(q) for _ in range(3))
    a.grad(q, q, q, docs, o.out, o.lse, q, out=grads)
    assert [t._version for t in (*o, *grads)] == [1] * 5 and q._version == 0


@pytest.mark.parametrize("name,count", [("rb_dropout", 9), ("rb_norm_forward", 12), ("rb_norm_grad", 14), ("rb_attention_forward", 10), ("rb_attention_grad", 14)])
def test_native_marshalling_passes_what_ctypes_passes(name, count):
    native = getattr(block, name)
    if binding.Call is None:
        pytest.skip("no native marshalling was built")
    general = native.__wrapped__
    names = list(inspect.signature(general).parameters)
    assert len(names) == count and names[-1] == "hip_stream"
    structures = {"drop", "x", "residual", "total", "y", "grad_y", "grad_total", "grad_sum", "grad_x", "q", "k", "v", "documents", "out", "grad_out", "grad_q", "grad_k", "grad_v"}
    flat = name == "rb_dropout"
    kinds = "".join("s" if n == "hip_stream" else "i" if n in ("rows", "width", "dtype", "tokens") or n.endswith("stride") else
                    "h" if n in ("n", "a") or (n in structures and not (flat and n in ("x", "out"))) else "p" for n in names)
    seen = []
    entry = C.CFUNCTYPE(C.c_int, *[C.c_uint64] * count)(lambda *a: seen.append(a) or 5)
    there = binding.Call(C.cast(entry, C.c_void_p).value, kinds, lambda *a: ("general", a))
    t = torch.zeros(4)
    args = [{"h": 2 ** 46 + i, "p": t, "i": 5 + i, "s": 77}[k] for i, k in enumerate(kinds)]
    assert there(*args) == 5 and seen == [tuple(a.data_ptr() if a is t else a for a in args)]
    assert there(*args[:-1]) == 5 and seen[1] == seen[0][:-1] + (0,)
    args[kinds.index("h")] = rb.RbDrop(0.5, 1, 2)                      # a structure itself: the Python function takes it
    assert there(*args)[0] == "general"
    assert block._at(args[kinds.index("h")]) == C.addressof(args[kinds.index("h")]) and block._at(None) is None and block._at(12) == 12

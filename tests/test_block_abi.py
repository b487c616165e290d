"""The C ABI of include/rb_block.h without a GPU: exports, and every refusal of an argument before any device work."""
import ctypes as C
import os
import re
import subprocess

import pytest

import paper_2406_03285_amd as rb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                          # stands for an aligned device address: the calls below end before it is used
STREAM = None
NAN, INF = float("nan"), float("inf")


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rb_block.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\bint (rb_[a-z_]+)\s*\(", text)))
    assert set(names) == set(rb.BLOCK_EXPORTS)
    lib = C.CDLL(rb.BLOCK_LIB_PATH)
    for name in names:
        assert getattr(lib, name) is not None and callable(getattr(rb, name))


def test_constants_are_the_headers():
    text = open(os.path.join(ROOT, "include", "rb_block.h")).read()
    found = re.findall(r"#define (RB_MAX_[A-Z_]+)\s+(\(1 << \d+\)|\d+)", text)
    assert len(found) == 8
    for name, value in found:
        assert getattr(rb, name) == eval(value), name


@pytest.mark.parametrize("compiler", [["gcc", "-std=c11"], ["g++", "-std=c++17"]])
def test_header_is_c_and_cpp(compiler, tmp_path):
    src = tmp_path / ("t.c" if compiler[0] == "gcc" else "t.cpp")
    src.write_text("#include \"rb_block.h\"\n#include \"rb_train.h\"\nint f(rb_norm *n, rb_attention *a) { return rb_norm_destroy(n) + rb_attention_destroy(a); }\n"
                   "int sizes[sizeof(rb_rows) == 16 && sizeof(rb_heads) == 24 && sizeof(rb_drop) == 24 && sizeof(rb_documents) == 32 ? 1 : -1];\n")
    subprocess.run([*compiler, "-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)], check=True)
    assert (C.sizeof(rb.RbRows), C.sizeof(rb.RbHeads), C.sizeof(rb.RbDrop), C.sizeof(rb.RbDocuments)) == (16, 24, 24, 32)


def refused(call, good, bad, status=None):
    for b in bad:
        assert call(*{**good, **b}.values(), STREAM) == (rb.RB_EINVAL if status is None else status), b


def test_dropout_refuses():
    d = rb.RbDrop(0.5, 1, 2)
    good = dict(x=P, x_stride=100, rows=0, width=100, dtype=rb.RB_BF16, drop=d, out=2 * P, out_stride=100)
    assert rb.rb_dropout(*good.values(), STREAM) == rb.RB_OK                       # no rows: nothing to do
    refused(rb.rb_dropout, good, (
        dict(x=None), dict(x=P + 1), dict(out=None), dict(out=2 * P + 1), dict(x=P + 2, dtype=rb.RB_F32), dict(x_stride=99), dict(out_stride=99), dict(x_stride=1 << 60),
        dict(rows=-1), dict(rows=rb.RB_MAX_NORM_ROWS + 1), dict(width=0), dict(width=rb.RB_MAX_DROP_WIDTH + 1, x_stride=1 << 28, out_stride=1 << 28), dict(dtype=2),
        dict(drop=None), dict(drop=rb.RbDrop(-0.1, 1, 2)), dict(drop=rb.RbDrop(1.1, 1, 2)), dict(drop=rb.RbDrop(NAN, 1, 2)), dict(rows=2, out=P, out_stride=101)))


@pytest.mark.parametrize("args", [(0, 0, 0, 1e-5), (-1, 0, 0, 1e-5), (rb.RB_MAX_NORM_WIDTH + 1, 0, 0, 1e-5), (10, 2, 0, 1e-5), (10, 0, -1, 1e-5), (10, 0, 0, 0.0),
                                  (10, 0, 0, -1e-5), (10, 0, 0, NAN), (10, 0, 0, INF)])
def test_norm_create_refuses(args):
    assert rb.rb_norm_create(*args) == (rb.RB_EINVAL, None)


def rows(data, stride=100):
    return rb.RbRows(data, stride)


def test_norm_calls_refuse():
    rc, n = rb.rb_norm_create(100, rb.RB_BF16, rb.RB_F32, 1e-5)
    assert rc == rb.RB_OK
    assert rb.rb_norm_query(None)[0] == rb.RB_EINVAL and rb.rb_norm_query(n)[1] > 0
    assert rb.rb_norm_bind(n, None) == rb.RB_EINVAL and rb.rb_norm_bind(n, P + 128) == rb.RB_EINVAL and rb.rb_norm_bind(None, P) == rb.RB_EINVAL
    d, bad_d = rb.RbDrop(0.5, 1, 2), rb.RbDrop(2.0, 1, 2)
    wrong = (None, rows(None), rows(9 * P + 1), rows(9 * P, 99), rows(9 * P, -100), rows(9 * P, 1 << 60))
    good = dict(n=n, x=rows(P), residual=rows(2 * P), drop=d, rows=0, weight=3 * P, bias=4 * P, total=rows(5 * P), y=rows(6 * P), mean=7 * P, rstd=8 * P)
    assert rb.rb_norm_forward(*good.values(), STREAM) == rb.RB_OK
    assert rb.rb_norm_forward(*{**good, **dict(bias=None, mean=None, rstd=None)}.values(), STREAM) == rb.RB_OK
    assert rb.rb_norm_forward(*{**good, **dict(residual=None, drop=None, total=None)}.values(), STREAM) == rb.RB_OK
    refused(rb.rb_norm_forward, good, (
        dict(n=None), dict(rows=-1), dict(rows=rb.RB_MAX_NORM_ROWS + 1), dict(drop=bad_d), dict(weight=None), dict(weight=P + 2), dict(bias=P + 2), dict(mean=P + 1), dict(rstd=P + 2),
        dict(residual=None, drop=None), dict(total=rows(6 * P)), dict(rows=2, total=rows(P, 101)), dict(rows=2, total=rows(2 * P, 101)), dict(rows=2, y=rows(P, 101)),
        dict(rows=2, y=rows(2 * P)), *(dict(x=r) for r in wrong), *(dict(y=r) for r in wrong), *(dict(total=r) for r in wrong), *(dict(residual=r) for r in wrong[1:])))
    good = dict(n=n, grad_y=rows(P), total=rows(2 * P), grad_total=rows(3 * P), mean=4 * P, rstd=5 * P, drop=d, rows=2, weight=6 * P, grad_sum=rows(7 * P), grad_x=rows(8 * P),
                grad_weight=10 * P, grad_bias=11 * P)
    assert rb.rb_norm_grad(*good.values(), STREAM) == rb.RB_ESTATE                 # never bound
    refused(rb.rb_norm_grad, good, (
        dict(n=None), dict(rows=-1), dict(rows=rb.RB_MAX_NORM_ROWS + 1), dict(drop=bad_d), dict(drop=None), dict(grad_x=None), dict(mean=None), dict(rstd=None), dict(mean=P + 2),
        dict(rstd=P + 1), dict(weight=None), dict(weight=P + 1), dict(grad_weight=P + 2), dict(grad_bias=P + 1), dict(grad_sum=rows(2 * P)), dict(grad_x=rows(2 * P)),
        dict(grad_x=rows(7 * P)), dict(grad_sum=rows(P, 101)), dict(grad_sum=rows(3 * P, 101)), dict(grad_x=rows(P, 101)), dict(grad_x=rows(3 * P, 101)),
        *(dict(grad_y=r) for r in wrong), *(dict(total=r) for r in wrong), *(dict(grad_sum=r) for r in wrong), *(dict(grad_x=r) for r in wrong[1:]),
        *(dict(grad_total=r) for r in wrong[1:])))
    assert rb.rb_norm_destroy(n) == rb.RB_OK and rb.rb_norm_destroy(None) == rb.RB_OK


@pytest.mark.parametrize("change", [dict(heads=0), dict(heads=rb.RB_MAX_HEADS + 1, kv_heads=1), dict(kv_heads=0), dict(kv_heads=3), dict(kv_heads=16), dict(head_dim=0),
                                    dict(head_dim=4), dict(head_dim=12), dict(head_dim=136), dict(max_tokens=0), dict(max_tokens=rb.RB_MAX_TOKENS + 1),
                                    dict(heads=1024, kv_heads=1, max_tokens=(1 << 20) + 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(cap=-1.0),
                                    dict(cap=NAN), dict(cap=INF)])
def test_attention_create_refuses(change):
    good = dict(heads=8, kv_heads=2, head_dim=64, max_tokens=1000, causal=1, scale=0.125, cap=0.0)
    rc, a = rb.rb_attention_create(*good.values())
    assert rc == rb.RB_OK and rb.rb_attention_destroy(a) == rb.RB_OK
    assert rb.rb_attention_create(*{**good, **change}.values()) == (rb.RB_EINVAL, None)


def test_attention_calls_refuse():
    rc, a = rb.rb_attention_create(8, 2, 64, 1000, 1, 0.125, 0.0)
    assert rc == rb.RB_OK
    assert rb.rb_attention_query(None)[0] == rb.RB_EINVAL and rb.rb_attention_query(a)[1] >= 1000 * 16
    assert rb.rb_attention_bind(a, None) == rb.RB_EINVAL and rb.rb_attention_bind(a, P + 128) == rb.RB_EINVAL and rb.rb_attention_bind(None, P) == rb.RB_EINVAL

    def heads(data, token=512, head=64):
        return rb.RbHeads(data, token, head)

    docs = rb.RbDocuments(P, 2 * P, 3 * P, 5)
    bad_docs = (None, rb.RbDocuments(None, P, P, 5), rb.RbDocuments(P + 4, P, P, 5), rb.RbDocuments(P, P + 4, P, 5), rb.RbDocuments(P, P, P + 4, 5),
                rb.RbDocuments(P, P, P, -1), rb.RbDocuments(P, P, P, rb.RB_MAX_DOCUMENTS + 1))
    read = (None, heads(None), heads(P + 8), heads(P, 508), heads(P, 512, 60), heads(P, -512), heads(P, 512, -64), heads(P, 1 << 40), heads(P, 512, 1 << 50))
    written = read + (heads(P, 56), heads(P, 512, 56), heads(P, 0), heads(P, 64, 64), heads(P, 72, 64), heads(P, 64, 9 * 64 - 8))
    good = dict(a=a, q=heads(P), k=heads(2 * P), v=heads(3 * P), tokens=10, documents=docs, slopes=P, out=heads(4 * P), lse=5 * P)
    assert rb.rb_attention_forward(*good.values(), STREAM) == rb.RB_ESTATE         # never bound
    refused(rb.rb_attention_forward, good, (
        dict(a=None), dict(tokens=-1), dict(tokens=1001), dict(slopes=P + 2), dict(lse=P + 1), *(dict(documents=d) for d in bad_docs),
        *({n: t} for n in "qkv" for t in read), *(dict(out=t) for t in written)))
    good = dict(a=a, q=heads(P), k=heads(2 * P), v=heads(3 * P), tokens=10, documents=docs, slopes=P, out=heads(4 * P), lse=5 * P, grad_out=heads(6 * P), grad_q=heads(7 * P),
                grad_k=heads(8 * P), grad_v=heads(9 * P))
    assert rb.rb_attention_grad(*good.values(), STREAM) == rb.RB_ESTATE
    refused(rb.rb_attention_grad, good, (
        dict(a=None), dict(tokens=-1), dict(tokens=1001), dict(slopes=P + 2), dict(lse=None), dict(lse=P + 1), *(dict(documents=d) for d in bad_docs),
        *({n: t} for n in ("q", "k", "v", "out", "grad_out") for t in read), *({n: t} for n in ("grad_q", "grad_k", "grad_v") for t in written)))
    assert rb.rb_attention_destroy(a) == rb.RB_OK and rb.rb_attention_destroy(None) == rb.RB_OK

"""The C ABI of include/rb_train.h without a GPU: exports, and every refusal of an argument before any device work."""
import ctypes as C
import os
import re

import pytest

import paper_2406_03285_amd as rb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                          # stands for an aligned device address: the calls below end before it is used
STREAM = None


def test_library_exports_every_declared_function():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rb_train.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rb_[a-z_]+)\s*\(", text)))
    assert set(names) == set(rb.TRAIN_EXPORTS)
    lib = C.CDLL(rb.TRAIN_LIB_PATH)
    for name in names:
        assert getattr(lib, name) is not None and callable(getattr(rb, name))


def test_constants_are_the_headers():
    text = open(os.path.join(ROOT, "include", "rb_train.h")).read()
    for name, value in re.findall(r"#define (RB_MAX_[A-Z_]+)\s+(\(1 << \d+\)|\d+)", text):
        assert getattr(rb, name) == eval(value), name


@pytest.mark.parametrize("args", [(0, 0, 1, 0), (-1, 0, 1, 0), (rb.RB_MAX_VOCAB + 1, 0, 1, 0), (10, 2, 1, 0), (10, -1, 1, 0), (10, 0, -1, 0),
                                  (10, 0, rb.RB_MAX_GIVEN + 1, 0), (10, 0, 1, -1), (100, 0, 1, rb.RB_MAX_TOP + 1), (10, 1, 1, 11)])
def test_scorer_create_refuses(args):
    assert rb.rb_scorer_create(*args) == (rb.RB_EINVAL, None)


def test_scorer_calls_refuse():
    rc, s = rb.rb_scorer_create(100, rb.RB_BF16, 2, 3)
    assert rc == rb.RB_OK
    assert rb.rb_scorer_query(None)[0] == rb.RB_EINVAL and rb.rb_scorer_query(s)[1] > 0
    assert rb.rb_scorer_bind(s, None) == rb.RB_EINVAL and rb.rb_scorer_bind(s, P + 8) == rb.RB_EINVAL and rb.rb_scorer_bind(None, P) == rb.RB_EINVAL
    good = dict(s=s, logits=P, rows=4, row_stride=100, tokens=P, logp=P, lse=P, entropy=P, top_logp=P, top_ids=P)
    assert rb.rb_scorer_score(*good.values(), STREAM) == rb.RB_ESTATE            # never bound
    for bad in (dict(s=None), dict(logits=None), dict(logits=P + 1), dict(rows=-1), dict(rows=rb.RB_MAX_ROWS + 1), dict(row_stride=99), dict(tokens=None),
                dict(tokens=P + 4), dict(logp=None), dict(logp=P + 2), dict(lse=P + 1), dict(entropy=P + 2), dict(top_logp=None), dict(top_ids=None),
                dict(top_ids=P + 4)):
        assert rb.rb_scorer_score(*{**good, **bad}.values(), STREAM) == rb.RB_EINVAL, bad
    good = dict(s=s, logits=P, rows=0, row_stride=100, tokens=P, lse=P, entropy=P, grad_logp=P, grad_entropy=P, grad_logits=2 * P, grad_stride=100)
    assert rb.rb_scorer_grad(*good.values(), STREAM) == rb.RB_OK                  # no rows: nothing to do
    for bad in (dict(s=None), dict(logits=None), dict(logits=P + 1), dict(rows=-1), dict(row_stride=99), dict(tokens=None), dict(lse=None), dict(lse=P + 2),
                dict(entropy=None), dict(grad_logp=None), dict(grad_logp=P + 1), dict(grad_entropy=P + 2), dict(grad_logits=None),
                dict(grad_logits=2 * P + 1), dict(grad_stride=99), dict(rows=2, grad_logits=P, grad_stride=101)):
        assert rb.rb_scorer_grad(*{**good, **bad}.values(), STREAM) == rb.RB_EINVAL, bad
    assert rb.rb_scorer_destroy(s) == rb.RB_OK and rb.rb_scorer_destroy(None) == rb.RB_OK


FIVE = [rb.NEWTON_SCHULZ] * 5
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("args", [
    (0, 4, 4, 0, 0, FIVE, 0.0), (rb.RB_MAX_MATRICES + 1, 4, 4, 0, 0, FIVE, 0.0), (1, 0, 4, 0, 0, FIVE, 0.0), (1, 4, 0, 0, 0, FIVE, 0.0),
    (1, rb.RB_MAX_DIM + 1, 4, 0, 0, FIVE, 0.0), (1, 4, rb.RB_MAX_DIM + 1, 0, 0, FIVE, 0.0), (1, 4, 4, 2, 0, FIVE, 0.0), (1, 4, 4, 0, -1, FIVE, 0.0),
    (1, 4, 4, 0, 0, [], 0.0), (1, 4, 4, 0, 0, [(1.5, -0.5, 0.0)] * (rb.RB_MAX_ORTHO_STEPS + 1), 0.0), (1, 4, 4, 0, 0, FIVE, -1e-7),
    (1, 4, 4, 0, 0, FIVE, NAN), (1, 4, 4, 0, 0, FIVE, INF), (1, 4, 4, 0, 0, [(NAN, 0, 0)], 0.0), (1, 4, 4, 0, 0, [(1, INF, 0)], 0.0),
    (1, 4, 4, 0, 0, [(4.5, 0, 0)], 0.0), (1, 4, 4, 0, 0, [(2, 0, 0)] * 3, 0.0), (1, 4, 4, 0, 0, [(1, -70, 68)], 0.0)])
def test_ortho_create_refuses(args):
    assert rb.rb_ortho_create(*args) == (rb.RB_EINVAL, None)


def test_ortho_calls_refuse():
    rc, o = rb.rb_ortho_create(2, 6, 10, rb.RB_BF16, rb.RB_F32, FIVE, 1e-7)
    assert rc == rb.RB_OK
    assert rb.rb_ortho_query(None)[0] == rb.RB_EINVAL and rb.rb_ortho_query(o)[1] > 0
    assert rb.rb_ortho_bind(o, None) == rb.RB_EINVAL and rb.rb_ortho_bind(o, P + 128) == rb.RB_EINVAL and rb.rb_ortho_bind(None, P) == rb.RB_EINVAL
    good = dict(o=o, update=P, ums=60, urs=10, out=2 * P, oms=60, ors=10)
    assert rb.rb_ortho_apply(*good.values(), STREAM) == rb.RB_ESTATE
    for bad in (dict(o=None), dict(update=None), dict(update=P + 1), dict(out=None), dict(out=P + 2), dict(ums=-1), dict(urs=9), dict(oms=9), dict(oms=-60),
                dict(ors=9), dict(ors=2 ** 62)):
        assert rb.rb_ortho_apply(*{**good, **bad}.values(), STREAM) == rb.RB_EINVAL, bad
    good = dict(o=o, weight=P, wms=60, wrs=10, grad=2 * P, gms=60, grs=10, momentum=3 * P, lr=0.1, beta=0.9, nesterov=1, weight_decay=0.0, scale=1.0)
    assert rb.rb_ortho_step(*good.values(), STREAM) == rb.RB_ESTATE
    for bad in (dict(o=None), dict(weight=None), dict(weight=P + 2), dict(grad=None), dict(grad=P + 1), dict(momentum=None), dict(momentum=P + 2), dict(wms=5),
                dict(wrs=9), dict(gms=-1), dict(grs=9), dict(lr=NAN), dict(beta=INF), dict(weight_decay=NAN), dict(scale=-INF)):
        assert rb.rb_ortho_step(*{**good, **bad}.values(), STREAM) == rb.RB_EINVAL, bad
    assert rb.rb_ortho_destroy(o) == rb.RB_OK and rb.rb_ortho_destroy(None) == rb.RB_OK


@pytest.mark.parametrize("compiler", [["gcc", "-std=c11"], ["g++", "-std=c++17"]])
def test_header_is_c_and_cpp(compiler, tmp_path):
    import subprocess
    src = tmp_path / ("t.c" if compiler[0] == "gcc" else "t.cpp")
    src.write_text("#include \"rb_train.h\"\nint f(rb_scorer *s) { return rb_scorer_destroy(s); }\n")
    subprocess.run([*compiler, "-Wall", "-Werror", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(src)], check=True)


@pytest.mark.parametrize("name", ["rb_scorer_score", "rb_scorer_grad", "rb_ortho_apply"])
def test_native_marshalling_passes_what_ctypes_passes(name):
    """Streams, tensors, None and numbers, and what goes to the Python function instead."""
    import inspect

    import torch

    from paper_2406_03285_amd import binding, train
    native = getattr(train, name)
    if binding.Call is None:
        pytest.skip("no native marshalling was built")
    general = native.__wrapped__
    names = list(inspect.signature(general).parameters)
    kinds = "".join("h" if n in ("s", "o") else "s" if n == "hip_stream" else "i" if n == "rows" or n.endswith("stride") else "p" for n in names)
    assert {"rb_scorer_score": 11, "rb_scorer_grad": 12, "rb_ortho_apply": 8}[name] == len(kinds)
    seen = []
    entry = C.CFUNCTYPE(C.c_int, *[C.c_uint64] * len(kinds))(lambda *a: seen.append(a) or 3)
    there = binding.Call(C.cast(entry, C.c_void_p).value, kinds, lambda *a: ("general", a))

    class Stream:
        cuda_stream = 77

    t = torch.zeros(4)
    args = [{"h": 2 ** 46, "p": t, "i": 5 + i, "s": Stream()}[k] for i, k in enumerate(kinds)]
    assert there(*args) == 3
    assert seen == [tuple({"h": 2 ** 46, "p": t.data_ptr(), "i": 5 + i, "s": 77}[k] for i, k in enumerate(kinds))]
    assert there(*args[:-1]) == 3 and seen[1] == seen[0][:-1] + (0,)              # the stream left out: null
    args[kinds.index("p")] = None
    assert there(*args) == 3 and seen[2][kinds.index("p")] == 0
    args[kinds.index("i")] = 2.5
    assert there(*args)[0] == "general"

"""What positions of packed documents see (csrc/rb_kernels_attention.h), on the CPU: the function that the kernel calls, compiled for the host."""
import ctypes as C
import os
import random
import subprocess

import pytest

import block_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def spans_of(tmp_path_factory):
    where = tmp_path_factory.mktemp("spans")
    src = where / "spans.hip"
    src.write_text('''#include "rb_kernels_attention.h"
extern "C" void spans_of(const int64_t* offsets, const int64_t* lengths, const int64_t* prefixes, int64_t count, int32_t tokens, int32_t causal, int32_t* out)
{
    const SpanArgs a{offsets, lengths, prefixes, count, nullptr, tokens, causal};
    for (int32_t t = 0; t < tokens; ++t) {
        const Spans s = at_spans_of(a, a.offsets, t);
        out[4 * t] = s.sees.lo; out[4 * t + 1] = s.sees.hi; out[4 * t + 2] = s.seen.lo; out[4 * t + 3] = s.seen.hi;
    }
}
''')
    hipcc = os.environ.get("HIPCC", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc"))
    subprocess.run([hipcc, "-std=c++17", "-O1", "--offload-host-only", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2406_03285_amd", "csrc"), str(src), "-o",
                    str(where / "spans.so")], check=True)
    lib = C.CDLL(str(where / "spans.so"))

    def call(offsets, lengths, prefixes, tokens, causal):
        def array(x):
            return None if x is None else (C.c_int64 * len(x))(*x)
        out = (C.c_int32 * (4 * tokens))()
        lib.spans_of(array(offsets), array(lengths), array(prefixes), C.c_int64(len(offsets) - 1), tokens, int(causal), out)
        return [tuple(out[4 * t:4 * t + 4]) for t in range(tokens)]
    return call


def test_positions_see_what_the_definition_says(spans_of):
    rng = random.Random(1)
    for _ in range(300):
        tokens, count = rng.randrange(1, 40), rng.randrange(0, 9)
        offsets = sorted(rng.randrange(0, tokens + 1) for _ in range(count + 1))
        lengths = [rng.randrange(0, 12) for _ in range(count)] if rng.random() < 0.5 else None
        prefixes = [rng.randrange(0, 12) for _ in range(count)] if rng.random() < 0.5 else None
        causal = rng.random() < 0.7
        mask = ref.seen(tokens, offsets, lengths, prefixes, causal)
        spans = spans_of(offsets, lengths, prefixes, tokens, causal)
        for t, (lo, hi, seen_lo, seen_hi) in enumerate(spans):
            assert mask[t].nonzero().flatten().tolist() == list(range(lo, hi))
            assert mask[:, t].nonzero().flatten().tolist() == list(range(seen_lo, seen_hi))
        for a, b in zip(spans, spans[1:]):
            assert all(x <= y for x, y in zip((a[0], a[2]), (b[0], b[2])))


def test_offsets_that_cannot_be_stay_within_the_positions(spans_of):
    rng = random.Random(2)
    pool = [0, 1, 5, 20, 39, 40, 41, 1000, -1, -7, 2 ** 31 - 1, 2 ** 31, 2 ** 62, 2 ** 63 - 1, -2 ** 31, -2 ** 62, -2 ** 63]
    for _ in range(2000):
        tokens, count = 40, rng.randrange(0, 7)
        offsets, lengths, prefixes = ([rng.choice(pool) for _ in range(n)] for n in (count + 1, count, count))
        for t, (lo, hi, seen_lo, seen_hi) in enumerate(spans_of(offsets, lengths if rng.random() < 0.7 else None, prefixes, tokens, rng.random() < 0.5)):
            for a, b in ((lo, hi), (seen_lo, seen_hi)):
                assert 0 <= a <= t and t <= b <= tokens and (a == b or t < b)

"""CPU tests of csrc/overlap.h: whether two arrays with strides share an element, against every element's bytes."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
APART, SHARED, UNKNOWN = 0, 1, 2


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(pairs of arrays) -> answers; an array is (begin, bytes of a run, [(stride, count)])."""
    tmp = tmp_path_factory.mktemp("overlap")
    src, exe = tmp / "ask.cpp", tmp / "ask"
    src.write_text("""#include "overlap.h"
#include <cstdio>
int main()
{
    auto array = [](overlap::Array *a) {
        long long p, run, dims, s, n;
        if (scanf("%lld %lld %lld", &p, &run, &dims) != 3) return false;
        a->p = (uintptr_t)p;
        a->run = run;
        for (int k = 0; k < dims; ++k) {
            if (scanf("%lld %lld", &s, &n) != 2) return false;
            a->dim(s, n);
        }
        return true;
    };
    for (;;) {
        overlap::Array a, b;
        if (!array(&a) || !array(&b)) return 0;
        printf("%d %d\\n", (int)overlap::of(a, b), (int)overlap::of(b, a));
    }
}
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2211_00839_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True, timeout=60)

    def run(pairs):
        text = "\n".join("%d %d %d %s" % (p, n, len(dims), " ".join("%d %d" % d for d in dims)) for pair in pairs for p, n, dims in pair)
        out = subprocess.run([str(exe)], input=text, check=True, stdout=subprocess.PIPE, text=True, timeout=60).stdout.split()
        assert len(out) == 2 * len(pairs)
        return [(int(a), int(b)) for a, b in zip(out[::2], out[1::2])]
    return run


def bytes_of(array):
    p, run, dims = array
    begins = {p}
    for stride, count in dims:
        begins = {x + i * stride for x in begins for i in range(count)}
    return {x + i for x in begins for i in range(run)}


def test_against_every_byte(ask):
    rng = random.Random(5)

    def any_array():
        dims = [(rng.choice([0, 1, 2, 3, 4, 8, 12, 16, 24, 40, 64, 100]), rng.choice([0, 1, 1, 2, 3, 5])) for _ in range(rng.randint(0, 3))]
        return rng.randint(0, 120), rng.choice([0, 1, 2, 4, 8]), dims

    pairs = [(any_array(), any_array()) for _ in range(6000)]
    wanted = [SHARED if bytes_of(a) & bytes_of(b) else APART for a, b in pairs]
    assert sum(wanted) > 300
    assert ask(pairs) == [(w, w) for w in wanted]


def test_views_of_one_buffer(ask):
    """What programs have, at their sizes: parts of one projection's rows, a row further on, halves of a buffer, a transposed view."""
    rows, heads, d = 100000, 24, 128
    pitch = heads * d * 2

    def part(first, count, row=0, n=rows):
        return (1 << 40) + row * pitch + first * d * 2, d * 2, [(pitch, n), (d * 2, count)]

    def turned(first, count):
        return (1 << 40) + first * d * 2, d * 2, [(d * 2, count), (pitch, rows)]

    cases = [(part(0, 16), part(16, 4), APART), (part(16, 4), part(20, 4), APART), (part(0, 16), part(15, 4), SHARED), (part(0, 16), part(0, 16, 1, rows - 1), SHARED),
             (part(0, 16, 0, 50000), part(0, 16, 50000, 50000), APART), (part(0, 16, 0, 50001), part(0, 16, 50000, 50000), SHARED), (turned(0, 16), part(16, 8), APART),
             (turned(0, 17), part(16, 8), SHARED), (part(0, 16), ((1 << 40) - 8, 16, []), SHARED), (part(0, 16), ((1 << 40) - 8, 8, []), APART),
             # every other row of two interleaved tensors, and half a row of d elements
             ((0, 256, [(512, 1000)]), (256, 256, [(512, 1000)]), APART), ((0, 256, [(512, 1000)]), (257, 256, [(512, 1000)]), SHARED),
             ((0, 256, [(2 ** 40, 2 ** 20), (512, 1000)]), (2 ** 59 + 256, 256, [(2 ** 40, 2 ** 10), (512, 1000)]), APART)]
    assert ask([c[:2] for c in cases]) == [(c[2], c[2]) for c in cases]


def test_what_is_not_settled(ask):
    """Strides made to be hard end in an answer all the same."""
    a = (0, 1, [(6 * (i + 1000003), 4000) for i in range(3)])
    b = (3000001, 1, [(6 * (i + 1000033), 4000) for i in range(3)])
    assert all(x in (APART, UNKNOWN) for pair in ask([(a, b)]) for x in pair)

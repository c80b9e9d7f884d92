"""CPU tests of the rules that cut attention's calls into workgroups (csrc/attention_rules.h)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MOST = 2 ** 24 - 8


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(statements) -> the numbers they print, in C++ with the rules at hand."""
    def run(body):
        tmp = tmp_path_factory.mktemp("rules")
        src, exe = tmp / "ask.cpp", tmp / "ask"
        src.write_text('#include "attention_rules.h"\n#include <cstdio>\nusing namespace attn_rules;\n'
                       "static void put(double x) { printf(\"%%.17g\\n\", x); }\nint main()\n{\n%s\n    return 0;\n}\n" % body)
        subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2211_00839_amd", "csrc"), str(src), "-o", str(exe)], check=True, timeout=60)
        out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True, timeout=60).stdout
        return [float(x) for x in out.split()]
    return run


# batch, heads, group, longest_q, longest_k, fp32, bias's width, uneven
CALLS = [(b, kv * g, g, q, k, f, w, u) for b in (1, 7, 64, 5000) for kv in (1, 3, 8) for g in (1, 4, 32) for q in (1, 2, 33, 65, 129, 5000)
         for k in (1, 300, 4096, 100003, 2 ** 29) for f, w, u in ((0, 0, 0), (1, 449, 1), (0, 2241, 1))]


def test_forward_calls(ask):
    """Every row has its workgroup or one that goes on to it, parts of keys are wanted only where there are keys for them, and what is packed
    side by side fits."""
    got = iter(ask("\n".join("{ const Cut c = cut_of(%d, %d, %d, %d, %d, %d, %d, %d, %d); put(c.shared); put(c.pack); put(c.tiles); put(c.splits); put(c.least); }" %
                             (b, h, g, q, k, q, f, w, u) for b, h, g, q, k, f, w, u in CALLS)))
    for b, h, g, q, k, f, w, u in CALLS:
        shared, pack, tiles, splits, least = (int(next(got)) for _ in range(5))
        assert pack in (1, g) and (pack == 1 or (q * g <= 64 and w * g <= 7168))
        assert tiles >= 1 and (tiles == -(-q * pack // (32 if shared else 128)) or tiles * b * h // pack > MOST // 2)
        assert 1 <= splits <= 512
        units = -(-(b + 1) * (h // g) // 8) * 8
        assert tiles * splits * units * (g // pack) <= MOST or tiles == 1
        if splits > 1:
            assert tiles * b * (h // pack) * splits <= (4096 if u else 1024)
            assert splits * 128 <= k and least * splits * (32 if shared else 64) <= k


def test_longest_sequence_that_is_not_said(ask):
    got = ask("put(longest_of(0, 1000, 10, true)); put(longest_of(0, 1000, 2, true)); put(longest_of(77, 1000, 10, true)); "
              "put(longest_of(5000, 1000, 10, true)); put(longest_of(77, 1000, 10, false)); put(longest_of(0, 0, 0, true));")
    assert got == [400, 1000, 77, 1000, 1000, 0]


def test_parts_of_the_gradients(ask):
    """Queries are cut into parts only where workgroups are few, and each part has 256 rows at least."""
    cases = [(groups, uneven, q, g) for groups in (1, 40, 511, 512, 513, 1023, 1024, 10 ** 6) for uneven in (0, 1) for q in (1, 300, 4096) for g in (1, 4)]
    got = iter(ask("\n".join("put(parts_of(%d, %d, %d, %d));" % c for c in cases)))
    for groups, uneven, q, g in cases:
        parts = int(next(got))
        assert 1 <= parts <= 8 and (parts == 1 or parts * 256 <= q * g)
        assert parts == 1 or groups < (1024 if uneven else 512)
        assert parts * groups < 2048 or parts == 1


def test_rows_of_no_sequence(ask):
    """A token of one sequence in a tensor with room for many: parts of the keys where their sums stay small, none where they would be
    as large as all that room."""
    got = ask("\n".join("put(cut_of(1, 32, 4, 1, 100000, %d, false, 0, false, true).splits);" % rows for rows in (1, 4096, 4097, 2 ** 29)))
    assert got[0] > 1 and got[1] == got[0] and got[2:] == [1, 1]


def test_even_calls_have_no_more_parts_than_fill_the_device(ask):
    cases = [(b, h, q, k, f) for b in (1, 4) for h in (1, 8, 24, 64) for q in (128, 2048, 8192) for k in (2048, 30000) for f in (0, 1)]
    got = iter(ask("\n".join("{ const Cut c = cut_of(%d, %d, 1, %d, %d, %d, %d, 0, false); put(c.tiles); put(c.splits); }" % (b, h, q, k, q, f) for b, h, q, k, f in cases)))
    for b, h, q, k, f in cases:
        tiles, splits = int(next(got)), int(next(got))
        assert splits == 1 or tiles * b * h * splits <= 256, (b, h, q, k, f)

"""CPU tests of the rules that choose how the encoder's products run (csrc/encoder_rules.h), against points measured on both
sides, and of which routes the GPU tests' sizes reach."""
import os
import subprocess

import pytest

from encoder_shapes import TILES, TILES_8_BITS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(statements) -> the numbers they print, in C++ with the rules at hand."""
    def run(body):
        tmp = tmp_path_factory.mktemp("rules")
        src, exe = tmp / "ask.cpp", tmp / "ask"
        src.write_text('#include "encoder_rules.h"\n#include <cstdio>\nusing namespace enc_rules;\n'
                       "static void put(double x) { printf(\"%%.9g\\n\", x); }\nint main()\n{\n%s\n    return 0;\n}\n" % body)
        subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2211_00839_amd", "csrc"), str(src), "-o", str(exe)],
                       check=True, timeout=60)
        out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True, timeout=60).stdout
        return [float(x) for x in out.split()]
    return run


# (M, N, stages of k, gated): {(half a tile's side, parts): us}
MEASURED = {
    (16384, 2048, 32, 0): {(128, 1): 117, (64, 1): 132, (128, 2): 216, (64, 2): 236},
    (2048, 2048, 256, 0): {(128, 1): 278, (128, 3): 125, (128, 4): 121, (64, 1): 165, (64, 2): 132, (64, 8): 162},
    (1000, 2048, 128, 0): {(128, 1): 146, (128, 6): 47, (64, 1): 69, (64, 2): 48, (64, 4): 43, (64, 8): 50},
    (1000, 512, 8, 0): {(128, 1): 25, (64, 1): 11, (64, 2): 14},
    (5000, 512, 8, 0): {(128, 1): 25, (64, 1): 11, (64, 2): 21},
    (256, 2048, 32, 0): {(128, 1): 40, (64, 1): 19, (64, 3): 15, (64, 4): 15, (64, 16): 23},
    (300, 4096, 16, 1): {(128, 1): 28, (64, 1): 14, (64, 2): 23},
    (2000, 2048, 32, 1): {(128, 1): 55, (128, 2): 50, (64, 1): 35, (64, 2): 51},
    (16384, 8192, 32, 1): {(128, 1): 920, (64, 1): 1010, (128, 2): 1630},
    (2500, 1365, 48, 1): {(128, 1): 87, (64, 1): 63, (128, 2): 68, (64, 2): 73},
    (8000, 2048, 192, 0): {(128, 1): 345, (64, 1): 420, (128, 2): 382},
}


def test_products_are_cut_within_a_tenth_of_the_fastest_way_measured(ask):
    keys = sorted(MEASURED)
    got = ask("\n".join("{ Cut c = cut_of(%d, %d, %d, %s); put(c.wt); put(c.splits); }" % (m, n, s, "true" if g else "false")
                        for m, n, s, g in keys))
    for i, key in enumerate(keys):
        cut = (int(got[2 * i]), int(got[2 * i + 1]))
        points = MEASURED[key]
        if cut in points:
            assert points[cut] <= 1.1 * min(points.values()), (key, cut)
        else:       # parts between two that were measured
            wt, parts = cut
            below, above = max(p for w, p in points if w == wt and p < parts), min(p for w, p in points if w == wt and p > parts)
            assert min(points[(wt, below)], points[(wt, above)]) <= 1.1 * min(points.values()), (key, cut)


def test_cuts_cover_the_result_and_leave_every_part_some_work(ask):
    sizes = [(1, 1, 1), (17, 1, 1), (65, 129, 3), (300, 70000, 5), (1 << 20, 64, 2), (100000, 100000, 1), (64, 64, 100000), (2147483392, 1, 1)]
    body = []
    for m, n, s in sizes:
        for g in ("true", "false"):
            for f in ("cut_of", "direct_cut_of"):
                body.append("{ Cut c = %s(%d, %d, %d, %s); put(c.wt); put(c.splits); put(c.tiles_m); put(c.tiles_n); }" % (f, m, n, s, g))
    got = iter(ask("\n".join(body)))
    for m, n, s in sizes:
        for gated in (True, False):
            for direct in (False, True):
                wt, splits, tm, tn = (int(next(got)) for _ in range(4))
                side = 64 if direct else 2 * wt
                cols = 64 if direct else (wt if gated else 2 * wt)
                assert 1 <= splits <= s and (tm - 1) * side < m <= tm * side and (tn - 1) * cols < n <= tn * cols
                assert splits == 1 or tm * tn * splits <= 512


def test_few_rows_go_past_the_tiles_only_where_that_is_faster(ask):
    # (rows, columns, k, fp32, 8 bits, us straight from the weights, us in tiles)
    measured = [(17, 2048, 2048, 0, 0, 7.5, 11.6), (17, 8192, 2048, 0, 0, 10.9, 15.3), (32, 8192, 2048, 0, 0, 13.5, 15.3),
                (17, 2048, 8192, 0, 0, 28.4, 17.6), (33, 2048, 2048, 0, 0, 9.7, 11.6), (33, 8192, 2048, 0, 0, 15.6, 15.3),
                (64, 8192, 2048, 0, 0, 21.0, 15.3), (64, 512, 512, 0, 0, 4.7, 9.7), (64, 2048, 8192, 0, 0, 38.5, 17.6),
                (32, 2048, 2048, 0, 1, 9.1, 9.6), (64, 2048, 2048, 0, 1, 13.7, 9.6), (16, 2048, 2048, 1, 0, 7.7, 15.4),
                (16, 8192, 2048, 1, 0, 25.9, 39.7), (16, 2048, 8192, 1, 0, 22.9, 41.3)]
    got = ask("\n".join("put(few_rows(%d, %d, %d, %d, %d));" % m[:5] for m in measured))
    for m, few in zip(measured, got):
        assert bool(few) == (m[5] < m[6]), m


def test_small_fp32_products_go_without_pieces_where_that_is_faster(ask):
    # (M, N, K, us directly, us by pieces)
    measured = [(999, 511, 300, 12.7, 21.7), (2048, 2048, 640, 60.9, 52.3), (8000, 2048, 2048, 700, 345)]
    got = ask("\n".join("put(direct_forward(%d, %d, %d, false));" % m[:3] for m in measured))
    for m, direct in zip(measured, got):
        assert bool(direct) == (m[3] < m[4]), m


# (M, N, K): {parts: us}, fp32 directly
MEASURED_DIRECT = {
    (64, 8192, 2048): {1: 61.1, 2: 36.4, 3: 38.3, 4: 31.3, 6: 33.7},
    (960, 512, 640): {1: 21.5, 2: 16.4, 3: 17.5, 4: 16.5, 6: 19.0},
    (999, 511, 300): {1: 12.7, 2: 12.1, 3: 13.2, 4: 13.2},
    (2048, 1024, 640): {1: 33.2, 2: 42.2},
    (300, 300, 1200): {1: 37.0, 2: 22.6, 3: 17.4, 4: 15.0, 6: 13.0},
}


def test_direct_products_are_cut_within_a_fifth_of_the_fastest_way_measured(ask):
    keys = sorted(MEASURED_DIRECT)
    got = ask("\n".join("put(direct_cut_of(%d, %d, ceil_div(%d, DIRECT_STAGE), false).splits);" % key for key in keys))
    for key, parts in zip(keys, got):
        points = MEASURED_DIRECT[key]
        parts = max(p for p in points if p <= parts)
        assert points[parts] <= 1.2 * min(points.values()), (key, parts)


def test_the_gpu_tests_sizes_reach_every_route(ask):
    """Forward products of both tile sizes, whole and in parts, linear and gated, in bf16, 8 bits and pieces; backward products
    of both orders in both tile sizes, whole and in parts, side by side and one after the other."""
    body = []
    for m, n, k in TILES_8_BITS:
        n2 = 2 * (-(-n // 64) * 64)
        for per, times in ((64, 1), (128, 1), (64, 6)):
            for g in ("false", "true"):
                body.append("{ Cut c = cut_of(%d, %d, ceil_div(%d, %d) * %d, %s); put(c.wt); put(c.splits > 1); }" % (m, n, k, per, times, g))
        body.append("put(direct_forward(%d, %d, %d, false)); put(direct_forward(%d, %d, %d, true));" % (m, n, k, m, n, k))
        for times in (1, 6):
            body.append("{ Both b = both_of(%d, %d, ceil_div(%d, 64) * %d, %d, %d, ceil_div(%d, 64) * %d); put(b.together); put(b.first.wt); "
                        "put(b.first.splits > 1); put(b.second.wt); put(b.second.splits > 1); }" % (m, k, n, times, n, k, m, times))
            body.append("{ Both b = both_of(%d, %d, ceil_div(%d, 64) * %d, %d, %d, ceil_div(%d, 64) * %d); put(b.together); put(b.first.wt); "
                        "put(b.first.splits > 1); put(b.second.wt); put(b.second.splits > 1); }" % (m, k, n, 2 * times, n2, k, m, times))
    got = iter([int(x) for x in ask("\n".join(body))])
    forward, backward = set(), set()
    for m, n, k in TILES_8_BITS:
        cuts = {(kind, g): (next(got), next(got)) for kind in ("bf16", "mx8", "f32") for g in (0, 1)}
        direct = {0: next(got), 1: next(got)}
        for (kind, g), cut in cuts.items():
            if kind == "mx8":
                if k >= 2048:
                    forward.add((kind, g) + cut)
            elif (m, n, k) not in TILES:
                pass
            elif kind == "f32" and direct[g]:
                forward.add(("direct", g))
            else:
                forward.add((kind, g) + cut)
        for kind in ("bf16", "f32"):
            for g in (0, 1):
                found = (kind, next(got), ("first", next(got), next(got)), ("second", next(got), next(got)))
                if (m, n, k) in TILES:
                    backward.add(found)
    for kind in ("bf16", "mx8", "f32"):
        for g in (0, 1):
            assert {(kind, g, 128, 0), (kind, g, 64, 0)} <= forward or kind == "f32", (kind, g, forward)
            assert (kind, g, 64, 1) in forward, (kind, g)
    assert ("f32", 0, 128, 0) in forward and ("f32", 1, 128, 1) in forward and ("f32", 1, 64, 0) in forward
    assert {("direct", 0), ("direct", 1)} <= forward
    for which in (2, 3):
        seen = {b[which][1:] for b in backward}
        assert {(128, 0), (128, 1), (64, 0), (64, 1)} <= seen, (which, seen)
    assert {b[1] for b in backward} == {0, 1}

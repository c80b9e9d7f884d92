"""CPU test: of every kernel variant that a call of the encoder's products can launch, some GPU test's size launches it, for each
type, linear and gated, forward and backward on its own."""
from encoder_shapes import TILES, TILES_8_BITS
from encoder_shapes_more import FEW, MORE
from test_encoder_rules import ask  # noqa: F401
from test_gpu_encoder import SIZES

# one number for each call that a size makes: what its launches are, digit by digit
PROGRAM = """
    auto cut = [](Cut c) { return (c.wt == 128 ? 10 : 0) + (c.splits > 1 ? 1 : 0); };
    auto forward = [&](int64_t M, int64_t N, int64_t K, int type, bool gated) {
        if (few_rows(M, N, K, type == 2, type == 1)) {
            if (type == 2) return 1000 + (M == 1 ? 1 : M <= 4 ? 4 : 8);
            return 2000 + (M <= 16 ? (ceil_div(N, 16) < 256 ? 16 : 8) : M <= 32 ? 2 : 4);
        }
        if (type == 2 && direct_forward(M, N, K, gated)) return 3000 + cut(direct_cut_of(M, N, ceil_div(K, DIRECT_STAGE), gated));
        return 4000 + cut(cut_of(M, N, ceil_div(K, type == 1 ? 128 : 64) * (type == 2 ? 6 : 1), gated));
    };
    auto backward = [&](int64_t M, int64_t N, int64_t K, int type, bool gated) {
        const int w = gated ? 2 : 1, pieces = type == 2 ? 6 : 1;
        if (type == 2 && direct_backward(M, N, K, gated)) {
            const Both b = direct_both(M, N, K, gated);
            return 50000 + cut(b.first) * 100 + cut(b.second);
        }
        const Both b = both_of(M, K, ceil_div(N, 64) * pieces * w, gated ? 2 * ceil_div(N, 64) * 64 : N, K, ceil_div(M, 64) * pieces);
        return (b.together ? 60000 : 70000) + cut(b.first) * 100 + cut(b.second);
    };
"""

BF16, MX8, F32 = 0, 1, 2


def calls(sizes, types):
    return [(m, n, k, t, g) for m, n, k in sizes for t in types for g in (0, 1)]


def test_every_variant_is_launched_by_some_test(ask):  # noqa: F811
    asked = calls(SIZES + TILES + FEW + MORE, (BF16, F32)) + calls(SIZES + TILES_8_BITS + FEW + MORE, (MX8,))
    body = "".join("    put(forward(%d, %d, %d, %d, %d));\n" % c + ("    put(backward(%d, %d, %d, %d, %d));\n" % c if c[3] != MX8 else "    put(0);\n")
                   for c in asked)
    got = iter(int(x) for x in ask(PROGRAM + body))
    seen = set()
    for m, n, k, t, g in asked:
        f, b = next(got), next(got)
        if not (t == MX8 and f // 1000 == 4 and k < 2048):         # (those are bf16 products of widened copies)
            seen.add((t, g, "forward", f))
        if b // 10000 == 7:
            seen |= {(t, g, "first", b % 10000 // 100), (t, g, "second", b % 100)}
        elif b:
            seen.add((t, g, "both", b))
    tiles = (0, 1, 10, 11)          # small and large, whole and in parts
    want = {(t, g, "forward", 4000 + c) for t in (BF16, MX8, F32) for g in (0, 1) for c in tiles}
    want |= {(F32, g, "forward", 3000 + parts) for g in (0, 1) for parts in (0, 1)}
    want |= {(F32, g, "forward", 1000 + rows) for g in (0, 1) for rows in (1, 4, 8)}
    want |= {(t, g, "forward", 2000 + waves) for t in (BF16, MX8) for g in (0, 1) for waves in (16, 8, 2, 4)}
    want |= {(t, g, which, c) for t in (BF16, F32) for g in (0, 1) for which in ("first", "second") for c in tiles}
    for kind, types in ((60000, (BF16, F32)), (50000, (F32,))):
        want |= {(t, g, "both", kind + 100 * first + second) for t in types for g in (0, 1) for first in (0, 1) for second in (0, 1)}
    assert want <= seen, sorted(want - seen)

"""CPU tests of the three bf16 pieces that stand for an fp32 number in products (csrc/encoder_pieces.h)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "encoder_pieces.h"
#include <cmath>
#include <cstdio>
#include <cstring>
#include <random>
using namespace enc;

static bool adds_up(float v)
{
    const Piece3 p = pieces_of(v);
    return std::isfinite(of_bf16(p.a)) && (double)of_bf16(p.a) + of_bf16(p.b) + of_bf16(p.c) == (double)v;
}
// what the taken products leave out, as a share of the product
static double left_out(float x, float y)
{
    const Piece3 p = pieces_of(x), q = pieces_of(y);
    const double a[3] = {of_bf16(p.a), of_bf16(p.b), of_bf16(p.c)}, b[3] = {of_bf16(q.a), of_bf16(q.b), of_bf16(q.c)};
    double sum = 0;
    for (auto &pair : PIECE_PAIRS) sum += a[pair[0]] * b[pair[1]];     // (exact: 16 bits each, within 53 in all)
    return (sum - (double)x * y) / std::fabs((double)x * y);
}
int main()
{
    std::mt19937 gen(1);
    int wrong = 0;
    double worst = 0, mean = 0;
    const uint32_t mantissas[] = {0, 1, 0x7f, 0x80, 0x81, 0x7fff, 0x8000, 0x8001, 0xff7f, 0xff80, 0xffff, 0x10000, 0x17fff, 0x18000, 0x7fffff, 0x7f8000, 0x7f7fff, 0x7eff80};
    for (uint32_t e = 40; e < 255; ++e)             // (least pieces above bf16's least number)
        for (uint32_t m : mantissas)
            for (uint32_t s : {0u, 1u}) wrong += !adds_up(__builtin_bit_cast(float, s << 31 | e << 23 | m));
    const int n = 2000000;
    for (int i = 0; i < n; ++i) {
        const float x = __builtin_bit_cast(float, 127u << 23 | ((uint32_t)gen() & 0x7fffff)), y = __builtin_bit_cast(float, 127u << 23 | ((uint32_t)gen() & 0x7fffff));
        wrong += !adds_up(x) || !adds_up(-y);
        const double d = left_out(x, y);
        worst = std::fmax(worst, std::fabs(d));
        mean += d / n;
    }
    for (uint32_t m : mantissas)
        for (uint32_t k : mantissas)
            worst = std::fmax(worst, std::fabs(left_out(__builtin_bit_cast(float, 127u << 23 | m), __builtin_bit_cast(float, 127u << 23 | k))));
    const float inf = INFINITY;
    const Piece3 p = pieces_of(inf), q = pieces_of(-inf), r = pieces_of(__builtin_bit_cast(float, 0x7f800001u));
    const bool special = of_bf16(p.a) == inf && p.b == 0 && p.c == 0 && of_bf16(q.a) == -inf && q.b == 0 && std::isnan(of_bf16(r.a)) &&
                         adds_up(3.402823466e38f) && adds_up(-3.402823466e38f) && adds_up(0.f);
    std::printf("%d %.9g %.9g %d\n", wrong, worst, mean, special);
}
"""


def test_pieces_add_up_and_leave_out_little_of_either_sign(tmp_path):
    """Derived: pieces of at most 1, 2^-8 and 2^-17 of a number's power of two, so what is left out is at most 2 * 2^-25 + 2^-34; over two
    million random pairs its mean is within 2^-24 / 1000 of 0 (its rms is below 2^-25, a thousandth of which per root of two million)."""
    src, exe = tmp_path / "pieces.cpp", tmp_path / "pieces"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-I", os.path.join(ROOT, "paper_2211_00839_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True, timeout=60)
    wrong, worst, mean, special = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True, timeout=60).stdout.split()
    assert int(wrong) == 0 and int(special) == 1
    assert float(worst) <= 2.0 ** -24 * (1 + 2.0 ** -10), worst
    assert abs(float(mean)) <= 2.0 ** -24 / 1000, mean

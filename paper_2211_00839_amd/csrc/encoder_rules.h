// Rules of the encoder's products that are a matter of sizes alone: plain host code, so that the measured points behind
// them can be tested without a device.
#pragma once
#include <algorithm>
#include <cstdint>

namespace enc_rules {

// The cut of a product into workgroups: tiles of 2 wt x 2 wt sums, k in `splits` parts.
struct Cut {
    int wt, splits;
    int64_t tiles_m, tiles_n;
};

constexpr int64_t UNITS = 256;      // compute units of the device

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// What one launch may hold: the runtime takes fewer than 2^32 threads, and all of these kernels' large grids are of
// workgroups of 256.
constexpr int64_t MOST_WORKGROUPS = (((int64_t)1 << 32) - 1) / 256;
// Of `left` rows, `per` to a workgroup, those that go into the next launch.
inline int64_t rows_of_launch(int64_t left, int per) { return std::min(left, MOST_WORKGROUPS * per); }

inline int64_t workgroups_of(const Cut &c) { return c.tiles_m * c.tiles_n * c.splits; }
inline int64_t grid_of(const Cut &c) { return ceil_div(workgroups_of(c), 8) * 8; }      // (the same number for each of the 8 XCDs)
inline bool launchable(const Cut &c) { return grid_of(c) <= MOST_WORKGROUPS; }

// What a cut takes, in microseconds, from what was measured on full and on part-full devices (bf16, k contiguous):
//   a stage of a 256 x 256 tile      1.0 with few workgroups, 1.5 with one on every unit (the clock falls with the load)
//   a stage of a 128 x 128 tile      0.55 alone on its unit, 0.88 with a second one beside it
//   start, filling and epilogue      6 and 4 per round of workgroups
//   parts                            written and read again at 7 TB/s (they stay in the last-level cache), and a launch of 3.5
// Measured / by this rule: 16384 x 2048 x 2048 large tiles 115 / 108, small 132 / 129; the weights' gradient of it large in 4
// parts 121 / 125, in 1 278 / 294, small in 2 132 / 131; 1000 x 2048 x 8192 small in 4 43 / 41, in 1 69 / 75; 256 x 2048 x
// 2048 small in 3 15 / 15, large in 1 40 / 42.
inline double time_of(const Cut &c, int64_t M, int64_t N, int64_t stages, bool gated, int64_t units = UNITS)
{
    const int64_t workgroups = c.tiles_m * c.tiles_n * c.splits, deep = ceil_div(stages, c.splits);
    double t;
    if (c.wt == 128) {
        const int64_t rounds = ceil_div(workgroups, units);
        t = (double)rounds * ((double)deep * (1.0 + 0.5 * std::min(1.0, (double)workgroups / (double)units)) + 6.0);
    } else {
        const int64_t full = workgroups / (2 * units), rest = workgroups % (2 * units);
        t = (double)full * ((double)deep * 0.88 + 4.0);
        if (rest) t += (double)deep * (rest > units ? 0.88 : 0.55) + 4.0;
    }
    if (c.splits > 1) t += 3.5 + 0.25 * c.splits + 2e-6 / 7 * (double)c.splits * (double)M * (double)N * 4 * (gated ? 2 : 1);
    return t;
}

// M x N: the result (gated: N columns of each of two products); stages: of k, 64 bf16 or 128 8-bit elements each, three
// pieces of fp32 make six products.  units: what of the device it has to itself.
inline Cut cut_of(int64_t M, int64_t N, int64_t stages, bool gated, int64_t units = UNITS)
{
    Cut best{};
    double least = 0.0;
    for (int wt : {128, 64}) {
        Cut c;
        c.wt = wt;
        c.tiles_m = ceil_div(M, 2 * wt);
        c.tiles_n = ceil_div(N, gated ? wt : 2 * wt);
        for (int splits : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16}) {
            // (a part of fewer than four stages is all start and end)
            if (splits > 1 && (splits * 4 > stages || c.tiles_m * c.tiles_n * splits > 2 * units)) break;
            c.splits = splits;
            const double t = time_of(c, M, N, stages, gated, units);
            if (best.splits == 0 || (t < least && launchable(c))) {      // (large tiles come first: if they are too many, all are)
                best = c;
                least = t;
            }
        }
    }
    return best;
}

// A backward call's two products, side by side in one launch where each is small enough to leave room for the other: both in
// small tiles, all workgroups on the device at once.  The whole backward call in us, side by side / one after the other, bf16:
// 128 x 512 x 512 13.5 / 18.9, 1000 x 1024 x 1024 21.8 / 31.6 (gated 31.2 / 42.4), 2500 x 1365 x 512 41.5 / 48.3 (gated 53.0 / 56.8);
// fp32: 960 x 1280 x 512 41.1 / 57.2, 2000 x 1024 x 1024 79.5 / 97.2.
struct Both {
    bool together;
    Cut first, second;
};
inline Both both_of(int64_t M1, int64_t N1, int64_t stages1, int64_t M2, int64_t N2, int64_t stages2)
{
    Both b{true, cut_of(M1, N1, stages1, false, UNITS / 2), cut_of(M2, N2, stages2, false, UNITS / 2)};
    if (b.first.wt == 64 && b.second.wt == 64 && workgroups_of(b.first) + workgroups_of(b.second) <= 2 * UNITS) return b;
    return Both{false, cut_of(M1, N1, stages1, false), cut_of(M2, N2, stages2, false)};
}

// Whether a product has so few rows that each weight is best read once, straight into registers.  In us, that way / in
// tiles: bf16, 17 rows, 2048 x 2048 7.5 / 11.6, 8192 x 2048 10.9 / 15.3, 2048 x 8192 28.4 / 17.6; 33 rows, 2048 x 2048 9.7 / 11.6, 8192 x
// 2048 15.6 / 15.3; 64 rows, 512 x 512 4.7 / 9.7, 8192 x 2048 21.0 / 15.3; 8 bits, 32 rows, 2048 x 2048 9.1 / 9.6, 64 rows 13.7 / 9.6;
// fp32, 16 rows here / 17 in tiles, 2048 x 2048 7.7 / 15.4, 8192 x 2048 25.9 / 39.7, 2048 x 8192 22.9 / 41.3.
inline bool few_rows(int64_t M, int64_t N, int64_t K, bool f32, bool mx)
{
    if (M <= 16) return true;
    if (f32) return false;
    if (M <= 32) return K <= 4096;
    return M <= 64 && K <= 2048 && N * K <= (mx ? (int64_t)1 << 20 : (int64_t)1 << 22);
}

// fp32 products go to the fp32 matrix instruction directly (wt 32: tiles of 64 x 64, k in stages of 32) where that takes less
// than pieces do, whose launch and trip through memory come on top.
constexpr int DIRECT_STAGE = 32;
inline double direct_time_of(const Cut &c, int64_t M, int64_t N, int64_t stages, bool gated, int64_t units = UNITS)
{
    const int64_t workgroups = c.tiles_m * c.tiles_n * c.splits, deep = ceil_div(stages, c.splits);
    // a stage takes a unit 0.85 us, whether one workgroup has it to itself or two share it (measured, in 1 / 2 / 4 parts: 64 x 8192 over
    // 2048 61.1 / 36.4 / 31.3 us, 960 x 512 over 640 21.5 / 16.4 / 16.5, 999 x 511 over 300 12.7 / 12.1 / 13.2, 300 x 300 over 1200 37.0 / 22.6 /
    // 15.0, 2048 x 1024 over 640 33.2 / 42.2 / 46.9)
    double t = 5.0 + (double)ceil_div(workgroups, units) * (double)deep * (gated ? 1.5 : 0.85);
    if (c.splits > 1) t += 3.5 + 0.25 * c.splits + 2e-6 / 7 * (double)c.splits * (double)M * (double)N * 4 * (gated ? 2 : 1);
    return t;
}
inline Cut direct_cut_of(int64_t M, int64_t N, int64_t stages, bool gated, int64_t units = UNITS)
{
    Cut best{};
    double least = 0.0;
    Cut c;
    c.wt = 32;
    c.tiles_m = ceil_div(M, 64);
    c.tiles_n = ceil_div(N, 64);
    for (int splits : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16}) {
        if (splits > 1 && (splits * 2 > stages || c.tiles_m * c.tiles_n * splits > 2 * units)) break;
        c.splits = splits;
        const double t = direct_time_of(c, M, N, stages, gated, units);
        if (best.splits == 0 || t < least) {
            best = c;
            least = t;
        }
    }
    return best;
}

// Whole fp32 calls, both ways, in us: fitted to 560 calls measured both ways, of 64 .. 16384 rows, 64 .. 8192 columns and k of 64 .. 4096, up to
// 30 GFLOP a product, epilogues included (bias, activation, residual and z; g and u).  The estimates are off by a tenth (rms); over 860 calls, 300 of
// them long and narrow and not fitted to, the way they choose takes 0.6 % more than the faster one in the mean, at worst three tenths, where the two
// lie close together.
struct Ways {
    double direct, pieces;
};
inline Ways forward_ways(int64_t M, int64_t N, int64_t K, bool gated)
{
    const double w = gated ? 2 : 1, results = 1e-6 * w * (double)M * (double)N, operands = 1e-6 * (double)(M + (gated ? 2 : 1) * N) * (double)K;
    const int64_t stages = ceil_div(K, DIRECT_STAGE), deep = ceil_div(K, 64) * 6;
    const Cut cut = cut_of(M, N, deep, gated);
    const double direct = direct_time_of(direct_cut_of(M, N, stages, gated), M, N, stages, gated), pieces = time_of(cut, M, N, deep, gated);
    // large tiles at the result's edge take their epilogue with every check: 4097 x 2056 x 200 62.7 / 91.8, 4096 x 2048 x 200 55.6 / 56.0
    const bool edge = cut.wt == 128 && cut.splits == 1 && N % (gated ? 128 : 256) != 0;
    return gated ? Ways{0.88 * direct + 1.0 + 0.7 * results, 7.6 + 0.9 * pieces + 1.6 * operands + 0.9 * results + (edge ? 14.0 : 0.0)}
                 : Ways{0.88 * direct + 0.6 + 1.5 * results, 10.0 + 0.72 * pieces + 2.1 * operands + 2.7 * results + (edge ? 22.0 : 0.0)};
}
inline bool direct_forward(int64_t M, int64_t N, int64_t K, bool gated)
{
    const Ways t = forward_ways(M, N, K, gated);
    return launchable(direct_cut_of(M, N, ceil_div(K, DIRECT_STAGE), gated)) && t.direct < t.pieces;
}
// The direct kernel's two products of a backward call always run side by side, each cut for half of the device.
inline Both direct_both(int64_t M, int64_t N, int64_t K, bool gated)
{
    const int w = gated ? 2 : 1;
    return Both{true, direct_cut_of(M, K, ceil_div(N, DIRECT_STAGE) * w, false, UNITS / 2),
                direct_cut_of(gated ? 2 * ceil_div(N, 64) * 64 : N, K, ceil_div(M, DIRECT_STAGE), false, UNITS / 2)};
}
// Both gradients.  Directly: what all workgroups have to do, shared among the units, and the longest one's own way; by pieces: the products
// as they are cut, side by side or one after the other.  dz is made on the way in both, in four or in six bytes.
inline Ways backward_ways(int64_t M, int64_t N, int64_t K, bool gated)
{
    const int w = gated ? 2 : 1;
    const int64_t rows = gated ? 2 * ceil_div(N, 64) * 64 : N;
    const double slopes = 1e-6 * w * (double)M * (double)N, operands = 1e-6 * (double)(M + w * N) * (double)K, result = 1e-6 * (double)M * (double)K;
    const Both d = direct_both(M, N, K, gated);
    const double deep1 = 0.85 * (double)ceil_div(ceil_div(N, DIRECT_STAGE) * w, d.first.splits), deep2 = 0.85 * (double)ceil_div(ceil_div(M, DIRECT_STAGE), d.second.splits);
    const double load = ((double)workgroups_of(d.first) * deep1 + (double)workgroups_of(d.second) * deep2) / (double)UNITS;
    const int64_t stages1 = ceil_div(N, 64) * 6 * w, stages2 = ceil_div(M, 64) * 6;
    const Both p = both_of(M, K, stages1, rows, K, stages2);
    const int64_t units = p.together ? UNITS / 2 : UNITS;
    const double t1 = time_of(p.first, M, K, stages1, false, units), t2 = time_of(p.second, rows, K, stages2, false, units);
    return Ways{13.0 + 0.73 * load + 0.6 * std::max(deep1, deep2) + 2.0 * slopes + 3.2 * result,
                15.0 + 0.85 * (p.together ? std::max(t1, t2) : t1 + t2) + 3.5 * operands + 2.7 * slopes + 0.2 * result};
}
inline bool direct_backward(int64_t M, int64_t N, int64_t K, bool gated)
{
    const Both cut = direct_both(M, N, K, gated);
    const Ways t = backward_ways(M, N, K, gated);
    return grid_of(cut.first) + grid_of(cut.second) <= MOST_WORKGROUPS && t.direct < t.pieces;
}

} // namespace enc_rules

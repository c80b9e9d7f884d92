// How calls of attention are cut into workgroups (host code without a device, tested as such).
#pragma once
#include <algorithm>
#include <cstdint>

namespace attn_rules {

constexpr int64_t MOST_WORKGROUPS = ((int64_t)1 << 24) - 8;     // a launch stays below 2^32 threads
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int64_t MOST_SPLITS = 512;

// How long a sequence is taken to be where the caller does not say: four times the mean, all there is at most.  (Longer ones are
// gone through all the same, by fewer workgroups.)
inline int64_t longest_of(int64_t said, int64_t rows, int64_t batch, bool ragged)
{
    if (!ragged) return rows;
    return std::min(rows, said > 0 ? said : 4 * ceil_div(rows, std::max<int64_t>(batch, 1)));
}

struct Cut {
    bool keys;          // few rows of q: the waves share them and divide the keys
    int pack;           // heads that share their keys, side by side in a tile of rows
    int blocks;         // blocks of 32 rows in each wave
    int64_t tiles;      // workgroups for each sequence and (packed) head
    int64_t splits;     // parts of the keys
    int64_t least;      // tiles of 32 keys (keys false: 64) in a part, unless there are fewer
};

// bias_entries: floats of the bias for each head, 0 without one.  resident: a workgroup's tiles take an unpacked compute unit each.
inline Cut cut_of(int64_t batch, int64_t heads, int64_t group, int64_t longest_q, int64_t longest_k, int64_t q_rows, bool f32, int64_t bias_entries)
{
    Cut c{};
    const bool packable = group > 1 && q_rows * group <= ((int64_t)1 << 29) && bias_entries * group <= 7680;
    c.pack = packable && longest_q * group <= 64 ? (int)group : 1;
    c.keys = longest_q * c.pack <= 64;
    c.blocks = 1;
    const int64_t rows = c.keys ? 32 : 128 * c.blocks;
    c.tiles = std::max<int64_t>(1, ceil_div(longest_q * c.pack, rows));
    const int64_t across = batch * (heads / c.pack);
    c.tiles = std::max<int64_t>(1, std::min(c.tiles, MOST_WORKGROUPS / std::max<int64_t>(across, 1)));
    const int64_t groups = c.tiles * across;
    c.splits = 1;
    c.least = 1;
    if (groups < 1024 && groups > 0) {
        const int64_t least = c.keys ? (f32 ? 128 : 512) : 1024;            // keys of a part
        // as many parts as fill the compute units once; more where sequences may differ in length, since the longest is what is waited for
        const int64_t wanted = std::max<int64_t>(256 / groups, longest_k / 1024);
        c.splits = std::max<int64_t>(1, std::min({wanted, longest_k / least, 1024 / groups, MOST_SPLITS}));
        c.least = least / (c.keys ? 32 : 64);
    }
    return c;
}

} // namespace attn_rules

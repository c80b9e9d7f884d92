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

// Few rows, or few workgroups of 128 rows for each sequence and head: then the waves share 32 rows and divide what those go along.  Where the two meet was
// measured with 1024 rows of 64, us shared / 128 rows, by workgroups of 128 rows: bf16 forward 64: 14.0 / 20.9, 128: 23.5 / 20.9, 240: 41.8 / 22.1; gradients
// 128: 54 / 58, 192: 76 / 74, 240: 96 / 78; fp32 forward 128: 52 / 80, 192: 78 / 80, 240: 103 / 83; gradients 192: 256 / 281, 240: 340 / 300.
constexpr int64_t FEW_WORKGROUPS = 200, FEW_WORKGROUPS_BF16_FORWARD = 112;
inline bool shared_rows(int64_t across, int64_t longest, int64_t few) { return longest <= 64 || across * ceil_div(longest, 128) < few; }

// Workgroups for each sequence and head; a kernel goes on to the rows that these leave.
inline int64_t tiles_of(int64_t across, int64_t longest, bool shared)
{
    const int64_t tiles = std::max<int64_t>(1, ceil_div(longest, shared ? 32 : 128));
    return std::max<int64_t>(1, std::min(tiles, MOST_WORKGROUPS / std::max<int64_t>(across, 1)));
}

// Parts of the queries that a workgroup of the gradients of k and v goes along, added up behind: two workgroups fit a compute unit, and where some are
// longer than others twice that many are wanted, so that the short ones fill the gaps.  At most 8, of 256 rows at least.
inline int64_t parts_of(int64_t groups, bool uneven, int64_t longest_q, int64_t group)
{
    const int64_t wanted = uneven ? 1024 : 512;
    if (groups <= 0 || groups >= wanted) return 1;
    return std::max<int64_t>(1, std::min<int64_t>({ceil_div(wanted, groups), longest_q * group / 256, 8}));
}

// Sequences (and one for the rows outside them) times heads of k and v, in whole rounds over the eight dies.
inline int64_t units_of(int64_t batch, int64_t kv_heads) { return ceil_div((batch + 1) * kv_heads, 8) * 8; }

struct Cut {
    bool shared;
    int pack;           // heads that share their keys, side by side in a tile of rows
    int64_t tiles;      // workgroups for each sequence and (packed) head
    int64_t splits;     // parts of the keys
    int64_t least;      // tiles in a part, unless there are fewer
};

// The forward call.  uneven: sequences have lengths of their own.  width: floats of the bias for each head, 0 without one; a workgroup has room for 7168.
// (q_rows: of a sequence, or where they lie end to end, ragged, of all of them.)
inline Cut cut_of(int64_t batch, int64_t heads, int64_t group, int64_t longest_q, int64_t longest_k, int64_t q_rows, bool f32, int64_t width, bool uneven,
                  bool ragged = false)
{
    Cut c{};
    c.pack = group > 1 && longest_q * group <= 64 && q_rows * group <= ((int64_t)1 << 29) && width * group <= 7168 ? (int)group : 1;
    const int64_t across = batch * (heads / c.pack), most = units_of(batch, heads / group) * (group / c.pack);
    // (fp32: a compute unit has room for one workgroup of 128 rows, so that 257 of them take as long as 512.  1024 rows of 64, us shared / 128 rows, by
    // workgroups of 128 rows: 320: 127 / 160, 384: 151 / 159, 400: 174 / 159, 512: 200 / 162, 520: 220 / 234, 576: 226 / 238, 592: 246 / 238, 640: 249 / 238, 752: 297 / 239,
    // 776: 318 / 312, 792: 319 / 313, 832: 322 / 317: the rule is 3 percent off at most, just under 600 and 800.)
    const int64_t rounds = ceil_div(across * ceil_div(longest_q * c.pack, 128), 256);
    c.shared = shared_rows(across, longest_q * c.pack, f32 ? FEW_WORKGROUPS * std::max<int64_t>(rounds, 1) : FEW_WORKGROUPS_BF16_FORWARD);
    c.tiles = tiles_of(most, longest_q * c.pack, c.shared);
    c.splits = c.least = 1;
    const int64_t groups = c.tiles * across;
    // Parts of the keys cost a second launch, some 7 us: not for bf16 where a wave has fewer than eight tiles of them anyway (fp32 takes 3 us a tile).
    // Nor where there are far more rows than the lengths say: their parts are memory too.
    const int64_t slots = (ragged ? q_rows : q_rows * batch) * heads;
    if (groups < 1024 && groups > 0 && longest_k >= (f32 ? 256 : 2048) && slots <= 1024 * 128) {
        const int64_t least = c.shared ? (f32 ? 128 : 512) : 1024;          // keys of a part
        // as many parts as fill the compute units once; more where sequences differ in length, since the longest is what is waited for (and the short
        // ones' missing parts cost nothing)
        const int64_t wanted = std::max<int64_t>(256 / groups, uneven ? longest_k / 1024 : 0);
        c.splits = std::max<int64_t>(1, std::min({wanted, longest_k / least, (uneven ? 4096 : 1024) / groups, MOST_SPLITS}));
        c.least = least / (c.shared ? 32 : 64);
    }
    return c;
}

// Sums of parts are joined by a wave for each row and head where there are many, by a workgroup's eight where there are few and parts may be many.
// Whole calls over caches of 4096 keys of 128, us by workgroups / by waves: 1024 rows and heads 65.0 / 64.3, 4096: 50.3 / 40.1, 16384: 156 / 115.
inline bool many_joins(int64_t slots, int64_t splits) { return slots >= 2048 && splits <= 64; }

} // namespace attn_rules

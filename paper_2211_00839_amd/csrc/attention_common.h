// What the kernels of attention share: their arguments, the tiles of rows in LDS, and the two kinds of product made of them.
//
// Everything is computed turned round: a 32 x 32 block of scores has the tile's rows (keys; in the gradients of k and v, queries) down a
// lane's 16 registers and the workgroup's own rows across the lanes, so that softmax's sums run inside a lane and what comes out of the
// exponential is, as it stands, an operand of the second product.
#pragma once
#include "encoder_lds.h"
#include "encoder_math.h"

namespace attn {

using namespace enc;

constexpr int THREADS = 256;
constexpr int MAX_BUCKETS = 128;        // of one direction
constexpr int MAX_REACH = 1024;         // largest distance at which the last bucket may begin

struct Heads {
    char *p;
    long long batch, row, head;         // bytes from sequence to sequence, row to row, head to head
};

struct Bias {
    const void *table;                  // null: none
    bool f32, both;                     // both: what follows the query has the table's second half
    int buckets, reach;                 // of one direction; the distance from which on the last one holds
    unsigned short border[MAX_BUCKETS]; // bucket c + 1 begins at distance border[c]
};

struct Args {
    Heads q, k, v, o;                   // o: out
    Heads dout, dq, dk, dv;
    float *saved;                       // per row of q and head: the scores' maximum in powers of two, log2 of the sum over it
    float *stats;                       // gradients, four planes [head][row of q]: both added, delta, each of the two
    long long plane;                    // floats of such a plane
    long long q_all;                    // rows of q in all sequences
    const int *q_offsets, *k_offsets, *k_lengths;
    int batch, heads, kv_heads, group;  // group: query heads that share a head of k and v
    int q_rows, k_rows;                 // of a sequence; with offsets: of all of them
    int D, pack;                        // pack: query heads whose rows lie side by side in a tile
    bool causal, clear, direct;         // clear: rows that belong to no sequence become zeros; direct: rows are read 16 bytes at a time
    float scale, scale2;                // scale2: times log2 e
    Bias bias;
    int tiles, splits;
    float *part_o, *part_ml;            // with splits: their sums, and per row maximum and sum
    float *part_bias;                   // the table's gradient, a part of each workgroup
};

// Sequence b's rows: the first one's place in q and in k (in the whole tensor where there are offsets, else in its own batch), and how many.
// Offsets and lengths that are out of range are held inside it.
struct Sequence {
    long long q0, k0;
    int q_len, k_len;
    long long q_first;                  // counted over all sequences
};
__device__ __forceinline__ Sequence sequence(const Args &a, int b)
{
    Sequence s;
    s.q0 = s.k0 = 0;
    s.q_len = a.q_rows;
    s.k_len = a.k_rows;
    s.q_first = (long long)b * a.q_rows;
    if (a.q_offsets) {
        const int from = min(max(a.q_offsets[b], 0), a.q_rows), to = min(max(a.q_offsets[b + 1], from), a.q_rows);
        s.q0 = s.q_first = from;
        s.q_len = to - from;
    }
    if (a.k_offsets) {
        const int from = min(max(a.k_offsets[b], 0), a.k_rows), to = min(max(a.k_offsets[b + 1], from), a.k_rows);
        s.k0 = from;
        s.k_len = to - from;
    } else if (a.k_lengths) {
        s.k_len = min(max(a.k_lengths[b], 0), a.k_rows);
    }
    return s;
}
__device__ __forceinline__ char *rows_of(const Heads &h, int b, bool offsets, long long row0, int head)
{
    return h.p + (offsets ? 0 : (long long)b * h.batch) + row0 * h.row + (long long)head * h.head;
}

// Workgroups go round the eight dies; each die takes a run of consecutive ones, whose keys its L2 then holds.
__device__ __forceinline__ int place_of(int id, int total)
{
    const int each = (total + 7) / 8;
    return (id & 7) * each + (id >> 3);
}

// ---- rows of up to DP elements ----------------------------------------------------------------------------------------------

template <typename T, int DP> struct Row {
    static constexpr int BYTES = DP * (int)sizeof(T), CHUNKS = BYTES / 16, EACH = 16 / (int)sizeof(T);
    static constexpr int STEPS = BYTES / 32;            // fragments: 16 bytes of each half of a wave
    static constexpr int BLOCKS = DP / 32;
    // The 16-byte chunk c of row r lies at chunk c ^ turn(r): 16 rows' chunks c lie in different banks, and so do the four rows of four
    // chunks that a transposing read touches.
    static __device__ __forceinline__ int turn(int r)
    {
        return CHUNKS == 8 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
    }
};

// Chunk `chunk` of a row of D elements at any alignment; what lies behind the row is zeros.
template <typename T> __device__ __forceinline__ uint4 chunk_of(const char *row, int chunk, int D)
{
    constexpr int EACH = 16 / (int)sizeof(T);
    const int count = D - chunk * EACH;
    if (count >= EACH) {
        const u32x4_any v = *reinterpret_cast<const u32x4_any *>(row + chunk * 16);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    unsigned w[4] = {0, 0, 0, 0};
    const T *p = reinterpret_cast<const T *>(row) + chunk * EACH;
#pragma unroll
    for (int e = 0; e < EACH - 1; ++e)
        if (e < count) {
            if constexpr (sizeof(T) == 4) w[e] = __builtin_bit_cast(unsigned, p[e]);
            else w[e / 2] |= (unsigned)__builtin_bit_cast(unsigned short, p[e]) << (16 * (e & 1));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// `count` consecutive elements (at most four) of a row of results.
template <typename T> __device__ __forceinline__ void store4(T *p, int count, float a, float b, float c, float d)
{
    if (count >= 4) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4_any *>(p) = f32x4{a, b, c, d};
        } else {
            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
            typedef __bf16 bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
            *reinterpret_cast<bf16x4_any *>(p) = bf16x4{(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
        }
        return;
    }
    const float v[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < count) p[i] = (T)v[i];
}

// Loads ROWS rows to `lds` (lds_addr: the same, as an address), LOADERS threads together; wave: which of theirs this one is.  `rows` of them
// exist; the others, and what lies behind D, become zeros, which no weight of zero turns into anything else.
template <typename T, int DP, int ROWS, int LOADERS>
__device__ __forceinline__ void load_rows(unsigned char *lds, unsigned lds_addr, const char *base, int pitch, int rows, int D, bool direct, int wave)
{
    using R = Row<T, DP>;
    constexpr int N = ROWS * R::CHUNKS / LOADERS;
    static_assert(N * LOADERS == ROWS * R::CHUNKS, "whole rounds");
    const int lane = threadIdx.x & 63;
    const bool whole = direct && rows >= ROWS && D == DP;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const int at = u * LOADERS + wave * 64;
        const int ci = at + lane, row = ci / R::CHUNKS, chunk = (ci % R::CHUNKS) ^ R::turn(row);
        if (whole) {
            tile::load16_to_lds(base, (unsigned)(row * pitch + chunk * 16), lds_addr + at * 16);
        } else {
            const bool there = row < rows && chunk * R::EACH < D;
            if (there && direct) tile::load16_to_lds(base, (unsigned)(row * pitch + chunk * 16), lds_addr + at * 16);
            else *reinterpret_cast<uint4 *>(lds + ci * 16) = there ? chunk_of<T>(base + (unsigned)(row * pitch), chunk, D) : make_uint4(0, 0, 0, 0);
        }
    }
}
template <typename T, int DP, int ROWS, int LOADERS> constexpr int loads_of() { return ROWS * Row<T, DP>::CHUNKS / LOADERS; }

// Where this lane reads: its row's chunks, and the transposed ones.
template <typename T, int DP> struct Reader {
    using R = Row<T, DP>;
    int row, swap;                      // byte of row lane & 31; its turn with this lane's half, times 16
    int up[R::BLOCKS], down[R::BLOCKS]; // bf16: 4 x 16 blocks of rows 4 half .. and 8 + 4 half ..
    __device__ __forceinline__ void init()
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31, i16 = lane & 15;
        row = r * R::BYTES;
        swap = (half ^ R::turn(r)) << 4;
        if constexpr (sizeof(T) == 2) {
            const int line = 4 * half + (i16 >> 2);
#pragma unroll
            for (int b = 0; b < R::BLOCKS; ++b) {
                const int chunk = 4 * b + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
                up[b] = line * R::BYTES + ((chunk ^ R::turn(line)) << 4) + (i16 & 1) * 8;
                down[b] = (line + 8) * R::BYTES + ((chunk ^ R::turn(line + 8)) << 4) + (i16 & 1) * 8;
            }
        }
    }
    // Fragment s of row 32 block + (lane & 31).
    __device__ __forceinline__ uint4 along(const unsigned char *tile, int block, int s) const
    {
        return *reinterpret_cast<const uint4 *>(tile + block * 32 * R::BYTES + row + ((s << 5) ^ swap));
    }
};

// The tile's row that register i of a block belongs to.
__device__ __forceinline__ int row_of(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

// acc += (32 rows of a tile) (32 rows held in registers)^T, one fragment of their length
template <typename T> __device__ __forceinline__ f32x16 scores(const uint4 &rows, const uint4 &mine, f32x16 acc)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, rows), __builtin_bit_cast(bf16x8, mine), acc, 0, 0, 0);
    } else {
        const f32x4 a = __builtin_bit_cast(f32x4, rows), b = __builtin_bit_cast(f32x4, mine);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], acc, 0, 0, 0);
        return acc;
    }
}

// acc[.][block] += (32 rows of a tile)^T p: block's 32 elements of the rows, weighted.  p as scores() leaves it; bf16: rounded to bf16 on
// its way into the product, to half a step of 2^-8 each, as the rows themselves were.
template <typename T, int DP, int N>
__device__ __forceinline__ void weigh(const Reader<T, DP> &at, const unsigned char *tile, int block, const f32x16 (&p)[N], f32x16 (&acc)[N][DP / 32])
{
    using R = Row<T, DP>;
    if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) tile::s16x4 *lds_ptr;
        unsigned char *from = const_cast<unsigned char *>(tile) + block * 32 * R::BYTES;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 w[N];
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int e = 0; e < 8; ++e) w[n][e] = (__bf16)p[n][8 * s + e];
#pragma unroll
            for (int b = 0; b < R::BLOCKS; ++b) {
                const tile::s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(from + at.up[b] + s * 16 * R::BYTES));
                const tile::s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(from + at.down[b] + s * 16 * R::BYTES));
                const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int n = 0; n < N; ++n) acc[n][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w[n], acc[n][b], 0, 0, 0);
            }
        }
    } else {
        const int lane = threadIdx.x & 63, half = lane >> 5, l = lane & 31;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = row_of(i, half);
#pragma unroll
            for (int b = 0; b < R::BLOCKS; ++b) {
                const int chunk = 8 * b + (l >> 2);
                const float v = *reinterpret_cast<const float *>(tile + (block * 32 + r) * R::BYTES + ((chunk ^ R::turn(r)) << 4) + (l & 3) * 4);
#pragma unroll
                for (int n = 0; n < N; ++n) acc[n][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[n][i], acc[n][b], 0, 0, 0);
            }
        }
    }
}

// Is there an infinity or a NaN in 32 rows of a tile?
template <typename T, int DP> __device__ __forceinline__ bool any_not_finite(const unsigned char *tile, int block)
{
    using R = Row<T, DP>;
    const int lane = threadIdx.x & 63;
    bool bad = false;
#pragma unroll
    for (int u = 0; u < 32 * R::CHUNKS / 64; ++u) {
        const uint4 v = *reinterpret_cast<const uint4 *>(tile + block * 32 * R::BYTES + (u * 64 + lane) * 16);
        const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bad |= (w[i] & 0x7f800000u) == 0x7f800000u;
            if constexpr (sizeof(T) == 2) bad |= (w[i] & 0x7f80u) == 0x7f80u;
        }
    }
    return __any(bad);
}

// weigh() for a block on the border of what may be seen: `seen` has a bit for each register.  A row that is not seen has no part in a sum at
// all, also where it is not finite and its weight of zero would make a NaN of it; such rows are rare, and then each row is added by itself.
template <typename T, int DP, int N>
__device__ __forceinline__ void weigh_seen(const Reader<T, DP> &at, const unsigned char *tile, int block, const f32x16 (&p)[N], const unsigned (&seen)[N],
                                           f32x16 (&acc)[N][DP / 32])
{
    using R = Row<T, DP>;
    if (!any_not_finite<T, DP>(tile, block)) {
        weigh<T, DP, N>(at, tile, block, p, acc);
        return;
    }
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll 1
    for (int r = 0; r < 32; ++r) {
        const int reg = ((r >> 3) << 2) | (r & 3), owner = (r >> 2) & 1;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float w = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) w = i == reg ? p[n][i] : w;
            int there = (seen[n] >> reg) & 1;
            const float other = __shfl_xor(w, 32);
            const int there_too = __shfl_xor(there, 32);
            if (owner != half) {
                w = other;
                there = there_too;
            }
#pragma unroll
            for (int b = 0; b < R::BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int d = 32 * b + row_of(i, half);
                    const T v = *reinterpret_cast<const T *>(tile + (block * 32 + r) * R::BYTES + (((d / R::EACH) ^ R::turn(r)) << 4) +
                                                             (d % R::EACH) * (int)sizeof(T));
                    if (there) acc[n][b][i] = fmaf(w, to_f32(v), acc[n][b][i]);
                }
        }
    }
}

// Both halves' values.
__device__ __forceinline__ void halves(float x, float *low, float *high)
{
    const unsigned bits = __builtin_bit_cast(unsigned, x);
    unsigned copy = bits;
    asm("" : "+v"(copy));           // (the instruction exchanges halves of two registers: they may not be one)
    const auto r = __builtin_amdgcn_permlane32_swap(bits, copy, false, false);
    const unsigned a = r[0], b = r[1];
    *low = __builtin_bit_cast(float, a);
    *high = __builtin_bit_cast(float, b);
}
__device__ __forceinline__ float add_halves(float x)
{
    float a, b;
    halves(x, &a, &b);
    return a + b;
}
__device__ __forceinline__ float max_halves(float x)
{
    float a, b;
    halves(x, &a, &b);
    return fmaxf(a, b);
}

// ---- bias -----------------------------------------------------------------------------------------------------------------

// The bias by offset, key's position - query's, in powers of two: entry `reach + offset` of a head's, offsets -reach .. reach (causal: .. 0).
__device__ __forceinline__ int bias_entries(const Args &a) { return a.causal ? a.bias.reach + 1 : 2 * a.bias.reach + 1; }

__device__ __forceinline__ int bucket_of(const Bias &b, int offset)
{
    const int size = abs(offset);
    int c = 0;
    for (int i = 0; i < b.buckets - 1; ++i) c += size >= (int)b.border[i] ? 1 : 0;
    return c + (b.both && offset > 0 ? b.buckets : 0);
}
__device__ __forceinline__ void fill_bias(const Args &a, int head, float *to)
{
    const int n = bias_entries(a);
    for (int e = threadIdx.x; e < n; e += THREADS) {
        const int at = bucket_of(a.bias, e - a.bias.reach) * a.heads + head;
        const float v = a.bias.f32 ? ((const float *)a.bias.table)[at] : (float)((const __bf16 *)a.bias.table)[at];
        // (the type's lowest value, as a mask, stays a number: a row of nothing else is a row of equal scores)
        to[e] = fabsf(v) <= 3.402823466e38f ? __builtin_amdgcn_fmed3f(v * 1.44269504f, -3.4e38f, 3.4e38f) : v;
    }
}
// Entry of an offset.
__device__ __forceinline__ int bias_entry(const Args &a, int offset)
{
    return min(max(offset, -a.bias.reach), a.causal ? 0 : a.bias.reach) + a.bias.reach;
}

// Adds the bias to a block of scaled scores: register i's offset is first + row_of(i, half).  lo .. hi: the block's offsets over the wave.
__device__ __forceinline__ void add_bias(const Args &a, const float *table, int first, int lo, int hi, float scale2, f32x16 &s)
{
    const int half = (threadIdx.x & 63) >> 5;
    if (hi <= -a.bias.reach || (lo >= a.bias.reach && !a.causal)) {
        const float b = table[hi <= -a.bias.reach ? 0 : 2 * a.bias.reach];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale2, b);
    } else if (lo >= -a.bias.reach && hi <= (a.causal ? 0 : a.bias.reach)) {
        const float *at = table + first + 4 * half + a.bias.reach;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale2, at[8 * (i >> 2) + (i & 3)]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale2, table[bias_entry(a, first + row_of(i, half))]);
    }
}

// The same where the registers hold queries and the lanes keys: register i's offset is first - row_of(i, half).
__device__ __forceinline__ void add_bias_down(const Args &a, const float *table, int first, int lo, int hi, float scale2, f32x16 &s)
{
    const int half = (threadIdx.x & 63) >> 5;
    if (hi <= -a.bias.reach || (lo >= a.bias.reach && !a.causal)) {
        const float b = table[hi <= -a.bias.reach ? 0 : 2 * a.bias.reach];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale2, b);
    } else if (lo >= -a.bias.reach && hi <= (a.causal ? 0 : a.bias.reach)) {
        const float *at = table + first - 4 * half + a.bias.reach;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale2, at[-(8 * (i >> 2) + (i & 3))]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale2, table[bias_entry(a, first - row_of(i, half))]);
    }
}

// Rows in front of the first sequence and behind the last one become zeros; part: which of `parts` workgroups this is.
template <typename T> __device__ __forceinline__ void clear_rows(const Heads &h, const int *offsets, int batch, int rows, int head, int D, int part, int parts)
{
    const int from = min(max(offsets[0], 0), rows), to = min(max(offsets[batch], from), rows);
    const long long count = (long long)(rows - (to - from)) * D;
    for (long long e = (long long)part * THREADS + threadIdx.x; e < count; e += (long long)parts * THREADS) {
        const int r = (int)(e / D), d = (int)(e % D);
        const long long row = r < from ? r : (long long)r + (to - from);
        reinterpret_cast<T *>(h.p + row * h.row + (long long)head * h.head)[d] = (T)0.f;
    }
}

} // namespace attn

// What the kernels of attention share: their arguments, the tiles of rows in LDS, and the two kinds of product made of them.
//
// Everything is computed turned round: a 32 x 32 block of scores has the tile's rows (keys; in the gradients of k and v, queries) down a
// lane's 16 registers and the workgroup's own rows across the lanes, so that softmax's sums run inside a lane and what comes out of the
// exponential is, as it stands, an operand of the second product.
#pragma once
#include "encoder_lds.h"
#include "encoder_math.h"

#include <type_traits>

namespace attn {

using namespace enc;

constexpr int THREADS = 256;
constexpr int MAX_BUCKETS = 128;        // of one direction
constexpr int MAX_REACH = 1024;         // largest distance at which the last bucket may begin

struct Heads {
    char *p;
    long long batch, row, head;         // bytes from sequence to sequence, row to row, head to head
};

// A divisor and what makes its quotients cheap: x times floor(2^32 / d) over 2^32 is x / d or one less.
struct Divisor {
    unsigned d, m;
    Divisor() = default;
    explicit Divisor(long long v) : d((unsigned)v), m(v == 1 ? 0xffffffffu : (unsigned)((1ull << 32) / (unsigned long long)v)) {}
};
__device__ __forceinline__ int divide(int x, const Divisor &by, int *rest = nullptr)
{
    unsigned q = (unsigned)(((unsigned long long)(unsigned)x * by.m) >> 32), r = (unsigned)x - q * by.d;
    if (r >= by.d) {
        ++q;
        r -= by.d;
    }
    if (rest) *rest = (int)r;
    return (int)q;
}

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
    long long q_all, k_all;             // rows of q and of k in all sequences
    const int *q_offsets, *k_offsets, *k_lengths;
    int batch, heads, kv_heads, group;  // group: query heads that share a head of k and v
    int q_rows, k_rows;                 // of a sequence; with offsets: of all of them
    int D, pack;                        // pack: query heads whose rows lie side by side in a tile
    bool causal, clear;                 // clear: rows that belong to no sequence become zeros
    float scale, scale2;                // scale2: times log2 e
    Bias bias;
    int tiles, splits, least;           // least: tiles of a split
    int workgroups;                     // all there are
    int packed;                         // workgroups go to the tiles that there are, whatever sequence they lie in (see tile_of): 1 of rows, 2 parts of keys
    int slots;                          // packed: most tiles of all sequences together, for each head
    Divisor by_heads, by_round, by_each, by_tiles, by_packs, by_pack, by_kv_heads, by_splits, by_group;      // round: a die's units between a workgroup's and its next; each: workgroups of a unit; packs: of packed heads to a head of k and v
    float *part_o, *part_ml;            // with splits: their sums, and per row maximum and sum
    float *part_k, *part_v;             // gradients of k and v with splits: their sums
    float *part_bias;                   // the table's gradient, a part of each workgroup
};

// Sequence b's rows: the first one's place in q and in k (in the whole tensor where there are offsets, else in its own batch), and how many.
// Offsets and lengths that are out of range are held inside it.
struct Sequence {
    long long q0, k0;
    int q_len, k_len;
    long long q_first, k_first;         // counted over all sequences
};
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ Sequence sequence(const Args &a, int b)
{
    Sequence s;
    s.q0 = s.k0 = 0;
    s.q_len = a.q_rows;
    s.k_len = a.k_rows;
    s.q_first = (long long)b * a.q_rows;
    s.k_first = (long long)b * a.k_rows;
    if (a.q_offsets) {
        const int from = uniform(min(max(a.q_offsets[b], 0), a.q_rows)), to = uniform(min(max(a.q_offsets[b + 1], from), a.q_rows));
        s.q0 = s.q_first = from;
        s.q_len = to - from;
    }
    if (a.k_offsets) {
        const int from = uniform(min(max(a.k_offsets[b], 0), a.k_rows)), to = uniform(min(max(a.k_offsets[b + 1], from), a.k_rows));
        s.k0 = s.k_first = from;
        s.k_len = to - from;
    } else if (a.k_lengths) {
        s.k_len = uniform(min(max(a.k_lengths[b], 0), a.k_rows));
    }
    return s;
}
__device__ __forceinline__ char *rows_of(const Heads &h, int b, bool offsets, long long row0, int head)
{
    return h.p + (offsets ? 0 : (long long)b * h.batch) + row0 * h.row + (long long)head * h.head;
}

// What a workgroup is for.  Workgroups go round the eight dies; all those of a sequence and a head of k and v (a unit) go to one of them, whose L2
// then holds that head's rows, and the next head's to the next, so that a long sequence is everyone's.  Few units that do not go round evenly are
// cut instead: each die gets an eighth of all there is, in order.  each: workgroups of a unit.
struct Unit {
    int sequence, kv_head, in;          // in: which of the unit's
};
inline __host__ __device__ bool goes_round(long long units) { return (units + 7) / 8 * 8 * 5 <= units * 6; }
// Workgroups that go on from one to the next have every so many units' the same `in`: a unit's order is shifted by how many such rounds lie before
// it, so that nobody has only the first parts of theirs.
__device__ __forceinline__ bool unit_of(const Args &a, int id, int sequences, Unit *u)
{
    const int units = sequences * a.kv_heads, each = (int)a.by_each.d, turn = id >> 3, die = id & 7;
    int unit;
    if (goes_round(units)) {
        const int mine = divide(turn, a.by_each, &u->in);
        unit = mine * 8 + die;
        if (unit >= units) return false;
        divide(u->in + divide(mine, a.by_round), a.by_each, &u->in);
    } else {
        const int all = units * each, some = (all + 7) >> 3, place = die * some + turn;
        if (place >= all || turn >= some) return false;
        unit = divide(place, a.by_each, &u->in);
    }
    u->sequence = divide(unit, a.by_kv_heads, &u->kv_head);
    return true;
}
// The same where sequences lie end to end by offsets: the slot-th tile of `ROWS` rows (of `pack` heads side by side) of all of them, counted over the
// sequences, so that no workgroup is started for a tile that a shorter sequence does not have (one that starts for nothing costs as much as a small
// one's work: 256 samples of 1 to 512 tokens with a bias, 8 heads: forward 129 us, now 72).  Every thread of the workgroup has to come along; lds: 64 bytes.
// False: there are fewer tiles, `tile` is how many.
// count(b): tiles of sequence b.
template <int THREADS_, typename Count> __device__ __forceinline__ bool tile_of(int batch, int slot, void *lds, Count count, int *sequence, int *tile, int *tiles)
{
    constexpr int WAVES = THREADS_ / 64;
    int *const sums = (int *)lds, *const found = sums + 8;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int before = 0;
    if (tid == 0) found[0] = -1;
    for (int b0 = 0; b0 < batch; b0 += THREADS_) {
        const int b = b0 + tid;
        const int mine = b < batch ? count(b) : 0;
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(sum, o);
            sum += lane >= o ? x : 0;
        }
        if (lane == 63) sums[wave] = sum;
        tile::wait_lds();
        tile::meet();
        int all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const int x = sums[w];
            sum += w < wave ? x : 0;
            all += x;
        }
        const int first = before + sum - mine;
        if (slot >= first && slot < first + mine) {
            found[0] = b;
            found[1] = slot - first;
            found[2] = mine;
        }
        before += all;
        tile::wait_lds();
        tile::meet();
        if (slot < before) break;
    }
    if (batch == 0) {
        tile::wait_lds();
        tile::meet();
    }
    const int b = uniform(found[0]);
    *tile = b < 0 ? uniform(before) : uniform(found[1]);
    *tiles = uniform(found[2]);
    *sequence = b;
    tile::wait_lds();
    tile::meet();
    return b >= 0;
}
// Tiles of `size` rows of sequence b, `pack` heads of a row side by side.
__device__ __forceinline__ int tiles_between(const int *offsets, int rows, int b, int pack, int size)
{
    const int from = min(max(offsets[b], 0), rows), to = min(max(offsets[b + 1], from), rows);
    return ((to - from) * pack + size - 1) / size;
}
// Tiles of keys in one part of them, of a sequence of `tiles`; and how many parts that makes.
__device__ __forceinline__ int tiles_of_part(const Args &a, int tiles) { return max(divide(tiles + a.splits - 1, a.by_splits), min(tiles, a.least)); }
__device__ __forceinline__ int parts_of(const Args &a, int tiles)
{
    const int per = tiles_of_part(a, tiles);
    return tiles == 0 ? 1 : (tiles + per - 1) / per;
}
__device__ __forceinline__ int keys_of(const Args &a, int b) { return a.k_lengths ? min(max(a.k_lengths[b], 0), a.k_rows) : a.k_rows; }
inline long long workgroups_of(long long sequences, long long kv_heads, long long each)
{
    const long long units = sequences * kv_heads;
    return goes_round(units) ? (units + 7) / 8 * 8 * each : (units * each + 7) / 8 * 8;
}

// A value of which the compiler knows nothing: what is made of it is made where it is used, not kept in registers through the loops before.
__device__ __forceinline__ int opaque(int x)
{
    asm volatile("" : "+v"(x));
    return x;
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

// Chunk `chunk` of a row of D elements at any alignment; what lies behind the row is zeros.  WHOLE: D is a multiple of a chunk's elements.
template <typename T, bool WHOLE> __device__ __forceinline__ uint4 chunk_of(const char *row, int chunk, int D)
{
    constexpr int EACH = 16 / (int)sizeof(T);
    const int count = D - chunk * EACH;
    if constexpr (WHOLE) {
        if (count <= 0) return make_uint4(0, 0, 0, 0);
        const u32x4_any v = *reinterpret_cast<const u32x4_any *>(row + chunk * 16);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
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

// Waits for loaded values here, not at their first use, which may lie in a loop and would wait for that loop's own loads too, each time round.
template <int N> __device__ __forceinline__ void arrive(uint4 (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i].x), "+v"(v[i].y), "+v"(v[i].z), "+v"(v[i].w));
}

// `count` consecutive elements (at most four; WHOLE: four) of a row of results.
template <typename T, bool WHOLE> __device__ __forceinline__ void store4(T *p, int count, float a, float b, float c, float d)
{
    if (WHOLE || count >= 4) {
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

// An address that is the same in all lanes, for loads that take it from scalar registers.
__device__ __forceinline__ const void *uniform(const void *p)
{
    const unsigned long long x = (unsigned long long)p;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)x), hi = __builtin_amdgcn_readfirstlane((unsigned)(x >> 32));
    return (const void *)(((unsigned long long)hi << 32) | lo);
}

// Brings ROWS rows of a matrix to LDS, LOADERS threads together, each always the same places of a tile.  DIRECT: straight from memory (all rows
// 16-byte aligned, D a multiple of 16 bytes; what lies behind D then holds other elements of the row, which meet zeros on the other side or lead
// to results that are not stored), else through the registers with zeros behind D.  Of a last tile's rows that do not exist the last one stands in
// until clear() puts zeros there, which no weight of zero turns into anything else.
template <typename T, int DP, int ROWS, int LOADERS, bool DIRECT> struct Loader {
    using R = Row<T, DP>;
    static constexpr int N = ROWS * R::CHUNKS / LOADERS, STEP = LOADERS / R::CHUNKS;       // rounds; rows from round to round
    static constexpr int KINDS = STEP >= 16 ? 1 : 16 / STEP < N ? 16 / STEP : N;          // (rows 16 apart are turned alike)
    static_assert(N * LOADERS == ROWS * R::CHUNKS && STEP >= 1, "whole rounds");
    int row, pitch;
    unsigned off[KINDS];
    int chunk[DIRECT ? 1 : KINDS];
    __device__ __forceinline__ void init(long long pitch_, int D, int t)
    {
        row = t / R::CHUNKS;
        pitch = (int)pitch_;
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const int c = (t % R::CHUNKS) ^ R::turn(row + i * STEP);
            if constexpr (DIRECT) {
                off[i] = (unsigned)(row * pitch + min(c, D / R::EACH - 1) * 16);
            } else {
                chunk[i] = c;
            }
        }
    }
    // wave: which of the loaders' waves this is
    __device__ __forceinline__ void issue(unsigned char *lds, unsigned lds_addr, const char *base, int rows, int D, int wave) const
    {
        if constexpr (DIRECT) {
            base = (const char *)uniform(base);
            if (rows >= ROWS) {
#pragma unroll
                for (int u = 0; u < N; ++u) tile::load16_to_lds(base, off[u % KINDS] + (unsigned)(u * STEP * pitch), lds_addr + (u * LOADERS + wave * 64) * 16);
            } else {
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    const int back = min(rows - 1 - row - u * STEP, 0);         // (to the last row there is)
                    tile::load16_to_lds(base, off[u % KINDS] + (unsigned)((u * STEP + back) * pitch), lds_addr + (u * LOADERS + wave * 64) * 16);
                }
            }
        } else {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int r = row + u * STEP;
                const bool there = r < rows && chunk[u % KINDS] * R::EACH < D;
                *reinterpret_cast<uint4 *>(lds + (u * LOADERS + wave * 64 + lane) * 16) =
                    there ? chunk_of<T, false>(base + (unsigned)(r * pitch), chunk[u % KINDS], D) : make_uint4(0, 0, 0, 0);
            }
        }
    }
    // Once the loads are in.
    __device__ __forceinline__ void clear(unsigned char *lds, int rows, int wave) const
    {
        if constexpr (DIRECT) {
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int u = 0; u < N; ++u)
                if (row + u * STEP >= rows) *reinterpret_cast<uint4 *>(lds + (u * LOADERS + wave * 64 + lane) * 16) = make_uint4(0, 0, 0, 0);
        }
    }
};

// Where this lane reads: its row's chunks, and the transposed ones.  One address of each, from which the others differ in single bits; they are
// made anew for each block, for there are better uses for sixteen registers.
template <typename T, int DP> struct Reader {
    using R = Row<T, DP>;
    int here;                           // chunk `half` of row lane & 31
    int across;                         // bf16: the 4 x 16 block of rows 4 half .. and elements 0 ..
    __device__ __forceinline__ void init()
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31, i16 = lane & 15;
        here = r * R::BYTES + ((half ^ R::turn(r)) << 4);
        const int line = 4 * half + (i16 >> 2), chunk = 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
        across = line * R::BYTES + ((chunk ^ R::turn(line)) << 4) + (i16 & 1) * 8;
    }
    // Fragment s of row 32 block + (lane & 31), from `here`.
    static __device__ __forceinline__ uint4 along(const unsigned char *tile, int here, int block, int s)
    {
        return *reinterpret_cast<const uint4 *>(tile + block * 32 * R::BYTES + (here ^ (s << 5)));
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

// Fragments are asked for this many products before they are used (left to itself the compiler asks for one and waits for it, every time: the
// latency of LDS four times the length of a product).  Rows of 64 leave registers for three waves to a SIMD, which need less of it.
template <int DP> constexpr int AHEAD = DP == 64 ? 2 : 4;

// `count` products, product(i, fragment) of the fragment that read(i) asks for.
template <int COUNT, int CLOSE, typename Read, typename Product> __device__ __forceinline__ void in_turn(Read read, Product product)
{
    decltype(read(0)) f[COUNT];
#pragma unroll
    for (int i = 0; i < (CLOSE < COUNT ? CLOSE : COUNT); ++i) f[i] = read(i);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        if (i + CLOSE < COUNT) f[i + CLOSE] = read(i + CLOSE);
        tile::pin();
        product(i, f[i]);
        tile::pin();
    }
}

template <int N> __device__ __forceinline__ void set_zero(f32x16 (&x)[N])
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[n][i] = 0.f;
}

// All blocks of 32 rows of a tile against 32 rows in registers, their whole length; the blocks take turns, each a chain of its own.
template <typename T, int DP, int N>
__device__ __forceinline__ void scores(const Reader<T, DP> &at, const unsigned char *tile, const uint4 (&mine)[Row<T, DP>::STEPS], f32x16 (&to)[N])
{
    const int here = opaque(at.here);
    set_zero(to);
    in_turn<N * Row<T, DP>::STEPS, AHEAD<DP>>([&](int i) { return at.along(tile, here, i % N, i / N); },
                                   [&](int i, const uint4 &rows) { to[i % N] = scores<T>(rows, mine[i / N], to[i % N]); });
}
// A block of each of two tiles against rows of their own.
template <typename T, int DP>
__device__ __forceinline__ void scores(const Reader<T, DP> &at, const unsigned char *tile0, const unsigned char *tile1, int block,
                                       const uint4 (&mine0)[Row<T, DP>::STEPS], const uint4 (&mine1)[Row<T, DP>::STEPS], f32x16 (&to)[2])
{
    const int here = opaque(at.here);
    set_zero(to);
    in_turn<2 * Row<T, DP>::STEPS, AHEAD<DP>>([&](int i) { return at.along(i & 1 ? tile1 : tile0, here, block, i >> 1); },
                                   [&](int i, const uint4 &rows) { to[i & 1] = scores<T>(rows, i & 1 ? mine1[i >> 1] : mine0[i >> 1], to[i & 1]); });
}

// acc[b] += (rows of N blocks of a tile, from `block` on)^T p: block b's 32 elements of the rows, weighted.  p as scores() leaves it; bf16: rounded
// to bf16 on its way into the product, to half a step of 2^-8 each, as the rows themselves were.
template <typename T, int DP, int N>
__device__ __forceinline__ void weigh(const Reader<T, DP> &at, const unsigned char *tile, int block, const f32x16 (&p)[N], f32x16 (&acc)[DP / 32])
{
    using R = Row<T, DP>;
    if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) tile::s16x4 *lds_ptr;
        unsigned char *from = const_cast<unsigned char *>(tile) + block * 32 * R::BYTES;
        const int across = opaque(at.across);
        bf16x8 w;
        in_turn<N * 2 * R::BLOCKS, AHEAD<DP>>(
            [&](int i) {
                const int b = i % R::BLOCKS, first = i / R::BLOCKS * 16;
                const tile::s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(from + (across ^ (b << 6)) + first * R::BYTES));
                const tile::s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(from + (across ^ (b << 6) ^ 32) + (first + 8) * R::BYTES));
                return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            },
            [&](int i, const bf16x8 &v) {
                const int b = i % R::BLOCKS, s = i / R::BLOCKS;
                if (b == 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = (__bf16)p[s >> 1][8 * (s & 1) + e];
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w, acc[b], 0, 0, 0);
            });
    } else {
        const int lane = threadIdx.x & 63, half = lane >> 5, l = lane & 31;
        in_turn<N * 16 * R::BLOCKS, 4>(
            [&](int i) {
                const int b = i % R::BLOCKS, r = row_of(i / R::BLOCKS % 16, half), chunk = 8 * b + (l >> 2);
                return *reinterpret_cast<const float *>(tile + ((block + i / R::BLOCKS / 16) * 32 + r) * R::BYTES + ((chunk ^ R::turn(r)) << 4) + (l & 3) * 4);
            },
            [&](int i, float v) {
                const int b = i % R::BLOCKS, j = i / R::BLOCKS;
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[j / 16][j % 16], acc[b], 0, 0, 0);
            });
    }
}

// ---- infinities and NaN at the border of what may be seen -----------------------------------------------------------------
//
// A row that is not seen has no part in a sum at all, where a weight of zero would make a NaN of an infinity.  Only blocks on the causal
// border are weighed for lanes that do not see all of their rows; a tile there that holds something that is not finite is left out, and added row by row
// once everything else is done.  Rare: what it takes is code behind the loops, not time or registers in them.

// The largest size among a chunk's elements, as bits; and whether it is a number's.
template <typename T> __device__ __forceinline__ unsigned largest(const uint4 &v, unsigned m)
{
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            m = max(m, w[i] & 0x7fffffffu);
        } else {
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            m = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu)));
        }
    }
    return m;
}
template <typename T> __device__ __forceinline__ bool any_not_finite(unsigned m)
{
    return __any(sizeof(T) == 4 ? m >= 0x7f800000u : m >= 0x7f800000u || (m & 0xffffu) >= 0x7f80u);
}
// Of a tile's rows.
template <typename T, int DP, int ROWS> __device__ __forceinline__ bool any_not_finite(const unsigned char *tile)
{
    const int lane = threadIdx.x & 63;
    unsigned m = 0;
#pragma unroll 4
    for (int u = 0; u < ROWS * Row<T, DP>::CHUNKS / 64; ++u) m = largest<T>(*reinterpret_cast<const uint4 *>(tile + (u * 64 + lane) * 16), m);
    return any_not_finite<T>(m);
}
// The same of `count` rows in memory.
template <typename T> __device__ __forceinline__ bool any_not_finite(const char *rows, long long pitch, int count, int D)
{
    const int lane = threadIdx.x & 63;
    unsigned m = 0;
#pragma unroll 1
    for (int r = lane & 31; r < count; r += 32)
#pragma unroll 1
        for (int c = lane >> 5; c * (16 / (int)sizeof(T)) < D; c += 2) m = largest<T>(chunk_of<T, false>(rows + r * pitch, c, D), m);
    return any_not_finite<T>(m);
}
template <typename T> __device__ __forceinline__ float dot(const char *a, const char *b, int D)
{
    float sum = 0.f;
#pragma unroll 1
    for (int d = 0; d < D; ++d) sum = fmaf(to_f32(reinterpret_cast<const T *>(a)[d]), to_f32(reinterpret_cast<const T *>(b)[d]), sum);
    return sum;
}
// Adds rows by themselves: visit(add) calls add(weight, row) for each.  The sums lie in LDS meanwhile (4 KB of the wave's own), block by block.
template <typename T, int DP, typename Visit> __device__ __forceinline__ void add_rows(unsigned char *lds, int D, f32x16 (&acc)[DP / 32], Visit visit)
{
    const int lane = threadIdx.x & 63;
    float *const sums = reinterpret_cast<float *>(lds) + lane;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[i * 64] = acc[b][i];
        visit([&](float weight, const char *row) {
#pragma unroll 1
            for (int i = 0; i < 16; ++i) {
                const int d = min(32 * b + row_of(i, lane >> 5), D - 1);        // (what lies behind D is not stored)
                sums[i * 64] = fmaf(weight, to_f32(reinterpret_cast<const T *>(row)[d]), sums[i * 64]);
            }
        });
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[b][i] = sums[i * 64];
        __builtin_amdgcn_sched_barrier(0);
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

// The bias by offset, key's position - query's, in powers of two: entry MARGIN + reach + offset of a head's, offsets -reach .. reach (causal: .. 0)
// and the last bucket's value as far beyond them as a tile on their border goes, so that no offset of such a tile needs a limit.
constexpr int MARGIN = 96;
inline __host__ __device__ int bias_width(int reach, bool causal) { return (causal ? reach + 1 : 2 * reach + 1) + 2 * MARGIN; }
// Of the gradient's sums by offset, without the margin.
inline __host__ __device__ int bias_entries(int reach, bool causal) { return causal ? reach + 1 : 2 * reach + 1; }

// The distances of bucket c of one direction: from .. to - 1.
__device__ __forceinline__ void distances(const Bias &b, int c, int *from, int *to)
{
    *from = c == 0 ? 0 : (int)b.border[c - 1];
    *to = c == b.buckets - 1 ? b.reach + MARGIN + 1 : (int)b.border[c];
}
// A thread for each bucket, or several where there are few.  (What is behind the query is masked where causal.)
__device__ __forceinline__ void fill_bias(const Args &a, int head, int count, float *to)
{
    const int all = a.bias.both ? 2 * a.bias.buckets : a.bias.buckets, parts = all <= 32 ? 8 : all <= 64 ? 4 : all <= 128 ? 2 : 1;
    const int c = threadIdx.x / parts, width = bias_width(a.bias.reach, !a.bias.both);
    if (c >= all) return;
    const bool behind = c >= a.bias.buckets;
    int from, until;
    distances(a.bias, behind ? c - a.bias.buckets : c, &from, &until);
    for (int g0 = 0; g0 < count; g0 += 4) {
        float v[4];                     // (four heads' values on their way at once)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = c * a.heads + head + min(g0 + g, count - 1);
            v[g] = a.bias.f32 ? ((const float *)a.bias.table)[at] : (float)((const __bf16 *)a.bias.table)[at];
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (g0 + g >= count) break;
            // (the type's lowest value, as a mask, stays a number: a row of nothing else is a row of equal scores)
            const float x = fabsf(v[g]) <= 3.402823466e38f ? __builtin_amdgcn_fmed3f(v[g] * 1.44269504f, -3.4e38f, 3.4e38f) : v[g];
            float *const zero = to + (g0 + g) * width + MARGIN + a.bias.reach;
            for (int r = from + (int)threadIdx.x % parts; r < until; r += parts)
                if (!behind) zero[-r] = x;
                else if (r > 0) zero[r] = x;
        }
    }
}
// The table's value at an offset, in powers of two.
__device__ __forceinline__ float bias_at(const Args &a, int head, int offset)
{
    int c = 0;
    for (int i = 0; i < a.bias.buckets - 1; ++i) c += abs(offset) >= (int)a.bias.border[i] ? 1 : 0;
    const int at = (c + (a.bias.both && offset > 0 ? a.bias.buckets : 0)) * a.heads + head;
    const float v = a.bias.f32 ? ((const float *)a.bias.table)[at] : (float)((const __bf16 *)a.bias.table)[at];
    return fabsf(v) <= 3.402823466e38f ? __builtin_amdgcn_fmed3f(v * 1.44269504f, -3.4e38f, 3.4e38f) : v;
}

// Is every offset lo .. hi in the last bucket of one direction?
__device__ __forceinline__ bool is_far(const Args &a, int lo, int hi) { return hi <= -a.bias.reach || (lo >= a.bias.reach && !a.causal); }
// That bucket's value.
__device__ __forceinline__ float far_bias(const Args &a, const float *table, int hi)
{
    return table[MARGIN + (hi <= -a.bias.reach ? 0 : 2 * a.bias.reach)];
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

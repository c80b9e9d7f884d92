// Attention forward: out = softmax(scale Q K^T + bias) V, one pass over the keys with the running maximum and sum of the softmax.
#pragma once
#include "attention_common.h"

namespace attn {

// KEYS false: a workgroup's four waves hold 32 N rows of q each and share tiles of TILE keys, the next one on its way while one is used.
// KEYS true: few rows of q (one block of 32), and each wave goes through blocks of 32 keys of its own, every fourth one, without meeting
// the others; their sums are joined at the end.  Either may leave its keys to several workgroups (splits), joined by k_attention_join.
template <typename T, int DP, bool KEYS> struct Forward {
    using R = Row<T, DP>;
    static constexpr int TILE = KEYS || R::BYTES == 512 ? 32 : 64;
    static constexpr int LOADERS = KEYS ? 64 : THREADS;
    static constexpr int STAGES = KEYS && R::BYTES == 512 ? 1 : 2;
    static constexpr int HALF = TILE * R::BYTES, STAGE = 2 * HALF;              // of keys, of keys and values
    static constexpr int TILES_BYTES = STAGES * STAGE * (KEYS ? 4 : 1);
    static constexpr int LOADS = 2 * TILE * R::CHUNKS / LOADERS;                // of a lane, to a stage
};

template <typename T, int DP, int N, bool KEYS, bool BIAS, bool DIRECT>
__global__ __launch_bounds__(THREADS, N == 1 && sizeof(T) == 2 && !KEYS ? 2 : 1) void k_attention(Args a)
{
    using F = Forward<T, DP, KEYS>;
    using R = Row<T, DP>;
    constexpr int MINE = 32 * N, ROWS = KEYS ? 32 : 4 * MINE, BLOCKS = F::TILE / 32;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups = a.heads / a.pack;
    const int total = a.tiles * groups * (a.batch + (a.clear ? 1 : 0)) * a.splits;
    int at = place_of(blockIdx.x, total);
    if (at >= total) return;
    const int split = at % a.splits;
    at /= a.splits;
    const int first_tile = a.tiles - 1 - at % a.tiles;          // (causal: the longest first)
    at /= a.tiles;
    const int group = at % groups, b = at / groups;
    if (b == a.batch) {
        if (split == 0)
            for (int g = 0; g < a.pack; ++g) clear_rows<T>(a.o, a.q_offsets, a.batch, a.q_rows, group * a.pack + g, a.D, first_tile, a.tiles);
        return;
    }
    const Sequence seq = sequence(a, b);
    const int head0 = group * a.pack, kv_head = head0 / a.group, shift = seq.k_len - seq.q_len;
    const char *const keys = rows_of(a.k, b, a.k_offsets != nullptr, seq.k0, kv_head), *const values = rows_of(a.v, b, a.k_offsets != nullptr, seq.k0, kv_head);
    float *const table = reinterpret_cast<float *>(lds + F::TILES_BYTES);
    const int entries = BIAS ? bias_entries(a) : 0;
    if constexpr (BIAS)
        for (int g = 0; g < a.pack; ++g) fill_bias(a, head0 + g, table + g * entries);
    unsigned char *const stages = lds + (KEYS ? wave * F::STAGES * F::STAGE : 0);
    const unsigned stages_addr = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds + (KEYS ? wave * F::STAGES * F::STAGE : 0);
    Reader<T, DP> reader;
    reader.init();
    Loader<T, DP, F::TILE, F::LOADERS, DIRECT> load_k, load_v;
    load_k.init(a.k.row, a.D, KEYS ? lane : tid);
    load_v.init(a.v.row, a.D, KEYS ? lane : tid);
    const int columns = seq.q_len * a.pack;
    for (int tile0 = first_tile * ROWS; tile0 < columns; tile0 += a.tiles * ROWS) {
        // ---- this wave's rows of q
        const int mine0 = tile0 + (KEYS ? 0 : wave * MINE);
        uint4 q[N][R::STEPS];
        int pos[N], head[N], row[N];
        bool there[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = mine0 + 32 * n + (lane & 31), in = min(c, columns - 1);
            there[n] = c < columns;
            row[n] = in / a.pack;
            head[n] = in - row[n] * a.pack;
            pos[n] = shift + row[n];
            const char *p = rows_of(a.q, b, a.q_offsets != nullptr, seq.q0 + row[n], head0 + head[n]);
#pragma unroll
            for (int s = 0; s < R::STEPS; ++s) q[n][s] = chunk_of<T, DIRECT>(p, 2 * s + half, a.D);
        }
        // ---- the keys that any of them sees, and this workgroup's and this wave's tiles of them
        const int last = shift + (min(tile0 + ROWS, columns) - 1) / a.pack;                     // the last row's position
        const int end = a.causal ? max(0, min(seq.k_len, last + 1)) : seq.k_len;
        const int lowest = shift + min(mine0, columns - 1) / a.pack, highest = shift + (min(mine0 + MINE, columns) - 1) / a.pack;
        const int tiles = (end + F::TILE - 1) / F::TILE, per = max((tiles + a.splits - 1) / a.splits, min(tiles, a.least));
        const int t0 = split * per + (KEYS ? wave : 0), t1 = min(tiles, (split + 1) * per), step = KEYS ? 4 : 1;
        auto load = [&](int t, int buf) {
            const int k0 = t * F::TILE;
            unsigned char *const to = stages + buf * F::STAGE;
            const unsigned to_addr = stages_addr + buf * F::STAGE;
            load_k.issue(to, to_addr, keys + (long long)k0 * a.k.row, end - k0, a.D, KEYS ? 0 : wave);
            load_v.issue(to + F::HALF, to_addr + F::HALF, values + (long long)k0 * a.v.row, end - k0, a.D, KEYS ? 0 : wave);
        };
        // A tile that has come; of the keys behind the last one the scores are masked, of the values there have to be zeros.
        auto clear = [&](int t, int buf) {
            const int rows = end - t * F::TILE;
            if (rows < F::TILE) load_v.clear(stages + buf * F::STAGE + F::HALF, rows, KEYS ? 0 : wave);
        };
        // top: the maximum that the exponents are taken from (it follows the scores' maximum when that is 2^8 above it); sum: of this lane's keys
        float top[N], sum[N];
        f32x16 acc[N][R::BLOCKS];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            top[n] = -__builtin_inff();
            sum[n] = 0.f;
#pragma unroll
            for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[n][d][i] = 0.f;
        }
        bool left_out = false;
        if (F::STAGES == 2 && t0 < t1) load(t0, 0);
        if constexpr (KEYS && BIAS) __syncthreads();
        int buf = 0;
        for (int t = t0; t < t1; t += step, buf ^= F::STAGES - 1) {
            if constexpr (KEYS) {
                tile::wait_lds();
                if (F::STAGES == 1) {
                    load(t, 0);
                    tile::wait_loads<0>();
                } else if (t + step < t1) {
                    load(t + step, buf ^ 1);
                    if (DIRECT) tile::wait_loads<F::LOADS>();
                } else {
                    tile::wait_loads<0>();
                }
                clear(t, buf);
                tile::wait_lds();
            } else {
                tile::wait_loads<0>();
                clear(t, buf);
                tile::wait_lds();
                tile::meet();
                if (t + 1 < t1) load(t + 1, buf ^ 1);
            }
            const int k0 = t * F::TILE;
            if (!KEYS && a.causal && k0 > highest) continue;
            const unsigned char *const ktile = stages + buf * F::STAGE, *const vtile = ktile + F::HALF;
            const bool border = a.causal && k0 + F::TILE - 1 > lowest, edge = border || k0 + F::TILE > end;
            f32x16 p[BLOCKS][N];
#pragma unroll
            for (int kb = 0; kb < BLOCKS; ++kb) {
#pragma unroll
                for (int n = 0; n < N; ++n)
#pragma unroll
                    for (int i = 0; i < 16; ++i) p[kb][n][i] = 0.f;
#pragma unroll
                for (int s = 0; s < R::STEPS; ++s) {
                    const uint4 k = reader.along(ktile, kb, s);
#pragma unroll
                    for (int n = 0; n < N; ++n) p[kb][n] = scores<T>(k, q[n][s], p[kb][n]);
                }
            }
            if constexpr (BIAS) {
#pragma unroll
                for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        const int j0 = k0 + 32 * kb;
                        add_bias(a, table + head[n] * entries, j0 - pos[n], j0 - highest, j0 + 31 - lowest, a.scale2, p[kb][n]);
                    }
            }
            if (edge) {
#pragma unroll
                for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        const int most = min(a.causal ? pos[n] : end - 1, end - 1) - k0 - 32 * kb;
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[kb][n][i] = row_of(i, half) <= most ? p[kb][n][i] : -__builtin_inff();
                    }
            }
            const float by = BIAS ? 1.f : a.scale2;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float m = p[0][n][0];
#pragma unroll
                for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) m = fmaxf(m, p[kb][n][i]);
                m = max_halves(m) * by;
                if (__any(m > top[n] + 8.f)) {
                    const float next = fmaxf(m, top[n]);
                    const float back = top[n] == next ? 1.f : __builtin_amdgcn_exp2f(top[n] - next);
                    top[n] = next;
                    sum[n] *= back;
#pragma unroll
                    for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[n][d][i] *= back;
                }
                const float from = top[n] == -__builtin_inff() ? 0.f : top[n];
                float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float e = __builtin_amdgcn_exp2f(BIAS ? p[kb][n][i] - from : fmaf(p[kb][n][i], a.scale2, -from));
                        p[kb][n][i] = e;
                        part[i & 3] += e;
                    }
                sum[n] += (part[0] + part[1]) + (part[2] + part[3]);
            }
#pragma unroll
            for (int kb = 0; kb < BLOCKS; ++kb) {
                if (border && any_not_finite<T, DP>(vtile, kb)) left_out = true;
                else weigh<T, DP, N>(reader, vtile, kb, p[kb], acc);
            }
        }
        if (left_out) {
            // the blocks on the border that hold something that is not finite
#pragma unroll 1
            for (int t = t0; t < t1; t += step)
#pragma unroll 1
                for (int j0 = t * F::TILE; j0 < min(end, (t + 1) * F::TILE); j0 += 32) {
                    const char *const rows = values + (long long)j0 * a.v.row;
                    if (t * F::TILE + F::TILE - 1 <= lowest || t * F::TILE > highest || !any_not_finite<T>(rows, a.v.row, end - j0, a.D)) continue;
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        const char *const mine = rows_of(a.q, b, a.q_offsets != nullptr, seq.q0 + row[n], head0 + head[n]);
#pragma unroll 1
                        for (int j = j0; j < min(end, j0 + 32); ++j) {
                            if (j > pos[n]) continue;
                            const float s = dot<T>(mine, keys + (long long)j * a.k.row, a.D);
                            const float x = BIAS ? fmaf(s, a.scale2, table[head[n] * entries + bias_entry(a, j - pos[n])]) : s * a.scale2;
                            add_row<T, DP>(values + (long long)j * a.v.row, a.D, __builtin_amdgcn_exp2f(x - (top[n] == -__builtin_inff() ? 0.f : top[n])), acc[n]);
                        }
                    }
                }
        }
        // ---- what leaves
#pragma unroll
        for (int n = 0; n < N; ++n) sum[n] = add_halves(sum[n]);
        int d0 = 0, d1 = 4 * R::BLOCKS;                         // groups of four elements that this wave stores
        if constexpr (KEYS) {
            // the waves' sums over one maximum, a quarter of the elements in each wave
            tile::wait_lds();
            __syncthreads();
            float *const sums = reinterpret_cast<float *>(lds), *const ml = sums + 4 * DP * 32;
            static_assert(4 * DP * 32 * 4 + 4 * 64 * 4 <= F::TILES_BYTES, "they fit where the tiles were");
#pragma unroll
            for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[((wave * R::BLOCKS + d) * 16 + i) * 64 + lane] = acc[0][d][i];
            if (half == 0) {
                ml[wave * 64 + lane] = top[0];
                ml[wave * 64 + 32 + lane] = sum[0];
            }
            __syncthreads();
            float m = -__builtin_inff(), weight[4], total_sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w * 64 + (lane & 31)]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float its = ml[w * 64 + (lane & 31)], l = ml[w * 64 + 32 + (lane & 31)];
                weight[w] = its == m ? 1.f : __builtin_amdgcn_exp2f(its - m);
                // (a wave without keys has no part in it; one whose scores are all NaN has)
                if (l == 0.f) weight[w] = 0.f;
                total_sum = l == 0.f ? total_sum : fmaf(weight[w], l, total_sum);
            }
            top[0] = m;
            sum[0] = total_sum;
            d0 = wave * R::BLOCKS;
            d1 = d0 + R::BLOCKS;
#pragma unroll
            for (int g = 0; g < R::BLOCKS; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float part = sums[((w * R::BLOCKS * 4 + d0 + g) * 4 + e) * 64 + lane];
                        v = weight[w] == 0.f ? v : fmaf(weight[w], part, v);
                    }
                    acc[0][g >> 2][4 * (g & 3) + e] = v;
                }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (!there[n]) continue;
            const int h = head0 + head[n];
            const long long slot = (seq.q_first + row[n]) * a.heads + h;
            const int D = opaque(a.D), first = opaque(8 * d0 + 4 * half);
            if (a.splits > 1) {
                const long long in = (long long)split * (a.q_all * a.heads) + slot;
                if (half == 0 && (!KEYS || wave == 0)) *reinterpret_cast<float2 *>(a.part_ml + 2 * in) = make_float2(top[n], sum[n]);
#pragma unroll
                for (int g = 0; g < (KEYS ? R::BLOCKS : 4 * R::BLOCKS); ++g) {
                    const int d = first + 8 * g;
                    if (d < D)
                        store4<float, DIRECT>(a.part_o + in * a.D + d, D - d, acc[n][g >> 2][4 * (g & 3)], acc[n][g >> 2][4 * (g & 3) + 1], acc[n][g >> 2][4 * (g & 3) + 2],
                               acc[n][g >> 2][4 * (g & 3) + 3]);
                }
                continue;
            }
            const float scale = sum[n] == 0.f ? 0.f : 1.f / sum[n];
            T *const out = reinterpret_cast<T *>(rows_of(a.o, b, a.q_offsets != nullptr, seq.q0 + row[n], h));
#pragma unroll
            for (int g = 0; g < (KEYS ? R::BLOCKS : 4 * R::BLOCKS); ++g) {
                const int d = first + 8 * g;
                if (d < D)
                    store4<T, DIRECT>(out + d, D - d, acc[n][g >> 2][4 * (g & 3)] * scale, acc[n][g >> 2][4 * (g & 3) + 1] * scale,
                           acc[n][g >> 2][4 * (g & 3) + 2] * scale, acc[n][g >> 2][4 * (g & 3) + 3] * scale);
            }
            if (a.saved && half == 0 && (!KEYS || wave == 0)) {
                // a row that sees no key: a maximum that leaves every weight at zero
                const bool none = sum[n] == 0.f;
                const float m = top[n] == -__builtin_inff() ? 0.f : top[n];
                *reinterpret_cast<float2 *>(a.saved + 2 * slot) = make_float2(none ? __builtin_inff() : m, none ? 0.f : __builtin_amdgcn_logf(sum[n]));
            }
        }
        // (another round of rows uses the tiles again)
        tile::wait_loads<0>();
        tile::wait_lds();
        __syncthreads();
    }
}

// Joins the splits' sums: a workgroup of eight waves for each row and head, each with every eighth split.
constexpr int JOIN_THREADS = 512, MOST_SPLITS = 512;
template <typename T> __global__ __launch_bounds__(JOIN_THREADS) void k_attention_join(Args a)
{
    __shared__ float weight[MOST_SPLITS], most[8], sums[8][128], totals[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long slots = a.q_all * a.heads, slot = blockIdx.x;
    const long long row = slot / a.heads;
    const int h = (int)(slot % a.heads);
    if (a.q_offsets && (row < min(max(a.q_offsets[0], 0), a.q_rows) || row >= min(max(a.q_offsets[a.batch], 0), a.q_rows))) return;
    float2 ml = make_float2(-__builtin_inff(), 0.f);
    if (tid < a.splits) ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (tid * slots + slot));
    float m = ml.x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    if (lane == 0) most[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = fmaxf(m, most[w]);
    // (a split without keys has no part in it; one whose scores are all NaN has)
    const float w = ml.y == 0.f ? 0.f : ml.x == m ? 1.f : __builtin_amdgcn_exp2f(ml.x - m);
    float total = ml.y == 0.f ? 0.f : w * ml.y;
    weight[tid] = w;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o);
    if (lane == 0) totals[wave] = total;
    __syncthreads();
    float v0 = 0.f, v1 = 0.f;
    const float *p = a.part_o + slot * a.D + lane;
#pragma unroll 4
    for (int s = wave; s < a.splits; s += 8) {
        const float x = weight[s];
        const float *const from = p + s * slots * a.D;
        const float y0 = lane < a.D ? from[0] : 0.f, y1 = lane + 64 < a.D ? from[64] : 0.f;
        v0 = x == 0.f ? v0 : fmaf(x, y0, v0);
        v1 = x == 0.f ? v1 : fmaf(x, y1, v1);
    }
    sums[wave][lane] = v0;
    sums[wave][64 + lane] = v1;
    __syncthreads();
    total = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) total += totals[i];
    const long long in = a.q_offsets ? row : row % a.q_rows;
    T *const out = reinterpret_cast<T *>(a.o.p + (a.q_offsets ? 0 : row / a.q_rows * a.o.batch) + in * a.o.row + (long long)h * a.o.head);
    if (tid < a.D) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sums[i][tid];
        out[tid] = (T)(total == 0.f ? 0.f : v / total);
    }
    if (a.saved && tid == 0) {
        const bool none = total == 0.f;
        const float t = m == -__builtin_inff() ? 0.f : m;
        *reinterpret_cast<float2 *>(a.saved + 2 * slot) = make_float2(none ? __builtin_inff() : t, none ? 0.f : __builtin_amdgcn_logf(total));
    }
}

} // namespace attn

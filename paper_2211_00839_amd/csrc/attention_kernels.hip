// Attention forward: out = softmax(scale Q K^T + bias) V, one pass over the keys with the running maximum and sum of the softmax.
//
// Bounds: long sequences by the matrix cores (4 d multiplies and adds a pair) beside one exponential a pair, few rows by reading k and v once, a single
// short one by latency.  Measured, bf16: 2 x 8192 tokens, 16 heads of 128: 1.07 ms, 1030 TFLOP/s (64 rows to a wave spilled: 381; three waves to a SIMD
// with tiles of 32 keys were slower); heads of 64, 4 x 2048 x 16 with a bias: 118 us, 580 TFLOP/s; one token over 100 003 keys, 16 heads on 2 of
// 128: 25 us, 4.1 TB/s, and 6 for the join; one token over 300 keys: 9.6 us.
#pragma once
#include "attention_common.h"

namespace attn {

// SHARED false: a workgroup's four waves hold 32 rows of q each and share tiles of TILE keys, the next one on its way while one is used.
// SHARED true: few rows of q.  Eight waves (four where tiles are large) hold the same 32, and each goes through tiles of 32 keys of its own, every
// eighth one, without meeting the others; their sums are joined at the end.
// Either may leave its keys to several workgroups (splits), joined by k_attention_join.
template <typename T, int DP, bool SHARED> struct Forward {
    using R = Row<T, DP>;
    static constexpr int TILE = SHARED || R::BYTES == 512 ? 32 : 64;
    static constexpr int WAVES = SHARED && R::BYTES < 512 ? 8 : 4, GROUP = 64 * WAVES;
    static constexpr int LOADERS = SHARED ? 64 : GROUP;
    static constexpr int STAGES = SHARED && R::BYTES >= 256 ? 1 : 2;
    static constexpr int HALF = TILE * R::BYTES, STAGE = 2 * HALF;              // of keys, of keys and values
    static constexpr int TILES_BYTES = STAGES * STAGE * (SHARED ? WAVES : 1);
    static constexpr int STATS_BYTES = SHARED ? WAVES * 64 * 4 : 0;             // a maximum and a sum for each of the 32 rows
    static constexpr int LOADS = 2 * TILE * R::CHUNKS / LOADERS;                // of a lane, to a stage
};

template <typename T, int DP, bool SHARED, bool BIAS, bool DIRECT>
__global__ __launch_bounds__(SHARED && sizeof(T) * DP < 512 ? 512 : 256, SHARED ? (sizeof(T) * DP < 512 ? 2 : 1) : sizeof(T) == 4 ? 1 : DP == 64 ? 3 : 2)
    void k_attention(Args a)
{
    using F = Forward<T, DP, SHARED>;
    using R = Row<T, DP>;
    constexpr int ROWS = SHARED ? 32 : 128, BLOCKS = F::TILE / 32, WAVES = F::WAVES;
    constexpr int GROUPS = SHARED ? 4 * R::BLOCKS / WAVES : 4 * R::BLOCKS;      // of four elements, that a wave stores of its rows
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int sequences = a.batch + (a.clear ? 1 : 0);
    int id = blockIdx.x;
    do {
        int b, kv_head, pack, first_tile, split = 0, tiles_here = a.tiles;
        if (SHARED && a.packed == 2) {
            int in, of;
            const int slot = divide(id, a.by_heads, &in);
            if (!tile_of<F::GROUP>(
                    a.batch, slot, lds, [&](int b) { return parts_of(a, (keys_of(a, b) + F::TILE - 1) / F::TILE); }, &b, &split, &of))
                break;                                          // (nor are there any behind it)
            kv_head = divide(divide(in, a.by_tiles, &first_tile), a.by_packs, &pack);
        } else if (a.packed) {
            int head;
            const int slot = divide(id, a.by_heads, &head);
            kv_head = divide(head, a.by_packs, &pack);
            int of;
            if (!tile_of<F::GROUP>(
                    a.batch, slot, lds, [&](int b) { return tiles_between(a.q_offsets, a.q_rows, b, a.pack, ROWS); }, &b, &first_tile, &of)) {
                // those left over clear the rows that belong to no sequence
                if (a.clear)
                    for (int g = 0; g < a.pack; ++g)
                        clear_rows<T>(a.o, a.q_offsets, a.batch, a.q_rows, (kv_head * (int)a.by_packs.d + pack) * a.pack + g, a.D, slot - first_tile,
                                      a.slots + 1 - first_tile);
                continue;
            }
            first_tile = of - 1 - first_tile;                   // (causal: the longest first)
            tiles_here = of;
        } else {
            Unit unit;
            if (!unit_of(a, id, sequences, &unit)) continue;
            int in_turn;
            b = unit.sequence;
            kv_head = unit.kv_head;
            split = divide(divide(unit.in, a.by_tiles, &in_turn), a.by_packs, &pack);
            first_tile = a.tiles - 1 - in_turn;
        }
        const int head0 = (kv_head * (int)a.by_packs.d + pack) * a.pack;
        if (b == a.batch) {
            if (split == 0)
                for (int g = 0; g < a.pack; ++g) clear_rows<T>(a.o, a.q_offsets, a.batch, a.q_rows, head0 + g, a.D, first_tile, a.tiles);
            continue;
        }
        const Sequence seq = sequence(a, b);
        const int columns = seq.q_len * a.pack, shift = seq.k_len - seq.q_len;
        if (first_tile * ROWS >= columns) continue;
        const char *const keys = rows_of(a.k, b, a.k_offsets != nullptr, seq.k0, kv_head), *const values = rows_of(a.v, b, a.k_offsets != nullptr, seq.k0, kv_head);
        float *const table = reinterpret_cast<float *>(lds + F::TILES_BYTES + F::STATS_BYTES);
        const int width = BIAS ? bias_width(a.bias.reach, a.causal) : 0;
        bool filled = false;
        unsigned char *const stages = lds + (SHARED ? wave * F::STAGES * F::STAGE : 0);
        const unsigned stages_addr = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds + (SHARED ? wave * F::STAGES * F::STAGE : 0);
        Reader<T, DP> reader;
        reader.init();
        Loader<T, DP, F::TILE, F::LOADERS, DIRECT> load_k, load_v;
        load_k.init(a.k.row, a.D, SHARED ? lane : tid);
        load_v.init(a.v.row, a.D, SHARED ? lane : tid);
        for (int tile0 = first_tile * ROWS; tile0 < columns; tile0 += tiles_here * ROWS) {
            // ---- the keys that any of this workgroup's rows sees, and its and this wave's tiles of them
            const int mine0 = tile0 + (SHARED ? 0 : wave * 32);
            const int last = shift + divide(min(tile0 + ROWS, columns) - 1, a.by_pack);                     // the last row's position
            const int end = a.causal ? max(0, min(seq.k_len, last + 1)) : seq.k_len;
            const int lowest = shift + divide(min(mine0, columns - 1), a.by_pack), highest = shift + divide(min(mine0 + 32, columns) - 1, a.by_pack);
            // (counted parts are those of all the keys: fewer tiles may make more parts)
            const int tiles = (end + F::TILE - 1) / F::TILE, per = tiles_of_part(a, a.packed == 2 ? (seq.k_len + F::TILE - 1) / F::TILE : tiles);
            const int from = split * per, t0 = from + (SHARED ? wave : 0), t1 = min(tiles, from + per), step = SHARED ? WAVES : 1;
            // ---- this wave's rows of q
            const int column = mine0 + (lane & 31), in = min(column, columns - 1);
            const bool there = column < columns;
            int in_pack;
            const int row = divide(in, a.by_pack, &in_pack), head = head0 + in_pack, pos = shift + row;
            const long long slot = (seq.q_first + row) * a.heads + head;
            if (a.splits > 1 && from >= t1 && split > 0) {
                if (there && half == 0 && (!SHARED || wave == 0))
                    *reinterpret_cast<float2 *>(a.part_ml + 2 * ((long long)split * (a.q_all * a.heads) + slot)) = make_float2(-__builtin_inff(), 0.f);
                continue;
            }
            auto load_keys = [&](int t, int buf) {
                const int k0 = t * F::TILE;
                load_k.issue(stages + buf * F::STAGE, stages_addr + buf * F::STAGE, keys + (long long)k0 * a.k.row, end - k0, a.D, SHARED ? 0 : wave);
            };
            auto load_values = [&](int t, int buf) {
                const int k0 = t * F::TILE;
                load_v.issue(stages + buf * F::STAGE + F::HALF, stages_addr + buf * F::STAGE + F::HALF, values + (long long)k0 * a.v.row, end - k0, a.D,
                             SHARED ? 0 : wave);
            };
            auto load = [&](int t, int buf) {
                load_keys(t, buf);
                load_values(t, buf);
            };
            // A tile that has come; of the keys behind the last one the scores are masked, of the values there have to be zeros.
            auto clear = [&](int t, int buf) {
                const int rows = end - t * F::TILE;
                if (rows < F::TILE) load_v.clear(stages + buf * F::STAGE + F::HALF, rows, SHARED ? 0 : wave);
            };
            if (t0 < t1) load(t0, 0);
            uint4 q[R::STEPS];
            {
                const char *p = rows_of(a.q, b, a.q_offsets != nullptr, seq.q0 + row, head);
#pragma unroll
                for (int s = 0; s < R::STEPS; ++s) q[s] = chunk_of<T, DIRECT>(p, 2 * s + half, a.D);
                arrive(q);
            }
            const float *const my_table = table + (head - head0) * width;
            if constexpr (BIAS)
                if (!filled) {
                    fill_bias(a, head0, a.pack, table);
                    filled = true;
                    if constexpr (SHARED) {
                        tile::wait_lds();
                        tile::meet();
                    }
                }
            // top: the maximum that the exponents are taken from (it follows the scores' maximum when that is 2^8 above it); sum: of this lane's keys
            float top = -__builtin_inff(), sum = 0.f;
            f32x16 acc[R::BLOCKS];
#pragma unroll
            for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
            bool left_out = false;
            // One tile.  edge: some of it is masked; near: its offsets are not all in the bias's last bucket.  (One body for all of them: several would each
            // want the sums in registers of their own.)
            auto compute = [&](bool edge, bool near, int k0, const unsigned char *ktile, auto keys_read, auto values_wanted) {
                const unsigned char *const vtile = ktile + F::HALF;
                f32x16 p[BLOCKS];
                scores<T, DP, BLOCKS>(reader, ktile, q, p);
                keys_read();
                float by = a.scale2, plus = 0.f;        // what is still to be done to the scores
                if (BIAS && near) {
                    const float *const bias = my_table + (k0 - pos) + 4 * half + a.bias.reach + MARGIN;
#pragma unroll
                    for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[kb][i] = fmaf(p[kb][i], a.scale2, bias[32 * kb + row_of(i, 0)]);
                    by = 1.f;
                } else if (BIAS) {
                    plus = far_bias(a, my_table, k0 + F::TILE - 1 - lowest);
                    if (__any(!(fabsf(plus) < 4096.f))) {
                        // (where the bias swallows the scores, as the type's lowest value does, it has to do so in every tile)
#pragma unroll
                        for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                            for (int i = 0; i < 16; ++i) p[kb][i] = fmaf(p[kb][i], a.scale2, plus);
                        by = 1.f;
                        plus = 0.f;
                    }
                }
                if (edge) {
                    const int most = min(a.causal ? pos : end - 1, end - 1) - k0;
#pragma unroll
                    for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) p[kb][i] = 32 * kb + row_of(i, half) <= most ? p[kb][i] : -__builtin_inff();
                }
                float m = p[0][0];
#pragma unroll
                for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) m = fmaxf(m, p[kb][i]);
                m = max_halves(m);
                m = fmaf(m, by, plus);
                if (__any(m > top + 8.f)) {
                    const float next = fmaxf(m, top);
                    const float back = top == next ? 1.f : __builtin_amdgcn_exp2f(top - next);
                    top = next;
                    sum *= back;
#pragma unroll
                    for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[d][i] *= back;
                }
                const float from = (top == -__builtin_inff() ? 0.f : top) - plus;
                float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kb = 0; kb < BLOCKS; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(p[kb][i], by, -from));
                        p[kb][i] = e;
                        part[i & 3] += e;
                    }
                sum += (part[0] + part[1]) + (part[2] + part[3]);
                values_wanted();
                if (a.causal && min(k0 + F::TILE, end) - 1 > lowest && any_not_finite<T, DP, F::TILE>(vtile)) {
                    left_out = true;
                    return;
                }
                weigh<T, DP, BLOCKS>(reader, vtile, 0, p, acc);
            };
            int buf = 0;
            for (int t = t0; t < t1; t += step, buf ^= F::STAGES - 1) {
                const int k0 = t * F::TILE;
                const unsigned char *const ktile = stages + buf * F::STAGE;
                const bool edge = k0 + F::TILE > end || (a.causal && k0 + F::TILE - 1 > lowest);
                const bool near = BIAS && !is_far(a, k0 - highest, k0 + F::TILE - 1 - lowest);
                if constexpr (SHARED && F::STAGES == 1) {
                    // one stage: the next keys are asked for once these are read, the next values once these are
                    if (DIRECT) tile::wait_loads<F::LOADS / 2>();
                    tile::wait_lds();
                    compute(edge, near, k0, ktile,
                            [&] {
                                tile::wait_lds();
                                if (t + step < t1) load_keys(t + step, 0);
                            },
                            [&] {
                                if (DIRECT && t + step < t1) tile::wait_loads<F::LOADS / 2>();
                                else tile::wait_loads<0>();
                                clear(t, 0);
                                tile::wait_lds();
                            });
                    tile::wait_lds();
                    if (t + step < t1) load_values(t + step, 0);
                    continue;
                }
                if constexpr (SHARED) {
                    tile::wait_lds();
                    if (t + step < t1) {
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
                    if ((a.causal && k0 > highest) || mine0 >= columns) continue;
                }
                compute(edge, near, k0, ktile, [] {}, [] {});
            }
            if (!SHARED && a.causal) tile::meet();
            if (left_out) {
                // the tiles on the border that hold something that is not finite
                const char *const mine = rows_of(a.q, b, a.q_offsets != nullptr, seq.q0 + row, head);
                add_rows<T, DP>(SHARED ? stages : lds + wave * 4096, a.D, acc, [&](auto add) {
#pragma unroll 1
                    for (int t = t0; t < t1; t += step) {
                        const int j0 = t * F::TILE, count = min(F::TILE, end - j0);
                        if (j0 + count - 1 <= lowest || j0 > highest) continue;
                        if (!any_not_finite<T>(values + (long long)j0 * a.v.row, a.v.row, count, a.D)) continue;
#pragma unroll 1
                        for (int j = j0; j < j0 + count; ++j) {
                            if (j > pos) continue;
                            float x = dot<T>(mine, keys + (long long)j * a.k.row, a.D) * a.scale2;
                            if constexpr (BIAS) x += bias_at(a, head, j - pos);
                            add(__builtin_amdgcn_exp2f(x - (top == -__builtin_inff() ? 0.f : top)), values + (long long)j * a.v.row);
                        }
                    }
                });
            }
            // ---- what leaves
            sum = add_halves(sum);
            int d0 = 0;                             // groups of four elements that this wave stores
            if constexpr (SHARED) {
                // the waves' sums over one maximum, as many of the elements in each wave
                tile::wait_lds();
                tile::meet();
                float *const sums = reinterpret_cast<float *>(lds), *const ml = reinterpret_cast<float *>(lds + F::TILES_BYTES);
                static_assert(WAVES * DP * 32 * 4 <= F::TILES_BYTES, "they fit where the tiles were");
                const int had = max(1, min(WAVES, t1 - from));       // waves that had keys
                if (wave < had)
#pragma unroll
                for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sums[((wave * R::BLOCKS + d) * 16 + i) * 64 + lane] = acc[d][i];
                if (half == 0) {
                    ml[wave * 64 + lane] = top;
                    ml[wave * 64 + 32 + lane] = sum;
                }
                tile::wait_lds();
                tile::meet();
                float m = -__builtin_inff(), weight[WAVES], total_sum = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml[w * 64 + (lane & 31)]);
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float its = ml[w * 64 + (lane & 31)], l = ml[w * 64 + 32 + (lane & 31)];
                    weight[w] = its == m ? 1.f : __builtin_amdgcn_exp2f(its - m);
                    // (a wave without keys has no part in it; one whose scores are all NaN has)
                    if (l == 0.f) weight[w] = 0.f;
                    total_sum = l == 0.f ? total_sum : fmaf(weight[w], l, total_sum);
                }
                top = m;
                sum = total_sum;
                d0 = wave * GROUPS;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = 0.f;
#pragma unroll
                        for (int w = 0; w < WAVES; ++w) {
                            if (w >= had) break;
                            const float part = sums[((w * R::BLOCKS * 4 + d0 + g) * 4 + e) * 64 + lane];
                            v = weight[w] == 0.f ? v : fmaf(weight[w], part, v);
                        }
                        acc[0][4 * g + e] = v;
                    }
            }
            if (there) {
                const bool none = sum == 0.f, one = half == 0 && (!SHARED || wave == 0);
                const int D = opaque(a.D), first = opaque(8 * d0 + 4 * half);
                if (a.splits > 1) {
                    const long long part = (long long)split * (a.q_all * a.heads) + slot;
                    if (one) *reinterpret_cast<float2 *>(a.part_ml + 2 * part) = make_float2(top, sum);
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        const int d = first + 8 * g, x = g >> 2, y = 4 * (g & 3);
                        if (d < D) store4<float, DIRECT>(a.part_o + part * a.D + d, D - d, acc[x][y], acc[x][y + 1], acc[x][y + 2], acc[x][y + 3]);
                    }
                } else {
                    const float scale = none ? 0.f : 1.f / sum;
                    T *const out = reinterpret_cast<T *>(rows_of(a.o, b, a.q_offsets != nullptr, seq.q0 + row, head));
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        const int d = first + 8 * g, x = g >> 2, y = 4 * (g & 3);
                        if (d < D)
                            store4<T, DIRECT>(out + d, D - d, acc[x][y] * scale, acc[x][y + 1] * scale, acc[x][y + 2] * scale, acc[x][y + 3] * scale);
                    }
                    // (a row that sees no key: a maximum that leaves every weight at zero)
                    if (a.saved && one)
                        *reinterpret_cast<float2 *>(a.saved + 2 * slot) =
                            make_float2(none ? __builtin_inff() : top == -__builtin_inff() ? 0.f : top, none ? 0.f : __builtin_amdgcn_logf(sum));
                }
            }
            // (another round of rows uses the tiles again)
            tile::wait_loads<0>();
            tile::wait_lds();
            tile::meet();
        }
    } while (SHARED && (id += (int)gridDim.x) < a.workgroups);
}

// What the joins share: a row and head's place, and how many parts it has; false: it belongs to no sequence.
struct Joined {
    long long row;
    int head, splits;
};
__device__ __forceinline__ bool joined(const Args &a, long long slot, Joined *j)
{
    j->row = slot / a.heads;
    j->head = (int)(slot % a.heads);
    if (a.q_offsets && (j->row < min(max(a.q_offsets[0], 0), a.q_rows) || j->row >= min(max(a.q_offsets[a.batch], 0), a.q_rows))) return false;
    // (parts behind a sequence's keys were not computed)
    const int b = a.q_offsets ? 0 : (int)(j->row / a.q_rows);
    j->splits = a.packed == 2 ? min(a.splits, parts_of(a, (keys_of(a, b) + 31) / 32)) : a.splits;
    return true;
}
template <typename T> __device__ __forceinline__ T *joined_row(const Args &a, const Joined &j)
{
    const long long in = a.q_offsets ? j.row : j.row % a.q_rows;
    return reinterpret_cast<T *>(a.o.p + (a.q_offsets ? 0 : j.row / a.q_rows * a.o.batch) + in * a.o.row + (long long)j.head * a.o.head);
}
__device__ __forceinline__ void save_joined(const Args &a, long long slot, float most, float total)
{
    const bool none = total == 0.f;
    const float t = most == -__builtin_inff() ? 0.f : most;
    *reinterpret_cast<float2 *>(a.saved + 2 * slot) = make_float2(none ? __builtin_inff() : t, none ? 0.f : __builtin_amdgcn_logf(total));
}

// Joins the splits' sums: a workgroup of eight waves for each row and head, each with every eighth split.
constexpr int JOIN_THREADS = 512, MOST_SPLITS = 512;
template <typename T> __global__ __launch_bounds__(JOIN_THREADS) void k_attention_join(Args a)
{
    __shared__ float weight[MOST_SPLITS], most[8], sums[8][128], totals[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long slots = a.q_all * a.heads, slot = blockIdx.x;
    Joined j;
    if (!joined(a, slot, &j)) return;
    const int splits = j.splits;
    float2 ml = make_float2(-__builtin_inff(), 0.f);
    if (tid < splits) ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (tid * slots + slot));
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
    for (int s = wave; s < splits; s += 8) {
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
    T *const out = joined_row<T>(a, j);
    if (tid < a.D) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sums[i][tid];
        out[tid] = (T)(total == 0.f ? 0.f : v / total);
    }
    if (a.saved && tid == 0) save_joined(a, slot, m, total);
}

// The same with many rows and up to 64 splits: a wave for each row and head.  Bound by reading the parts.
template <typename T> __global__ __launch_bounds__(JOIN_THREADS) void k_attention_join_many(Args a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long slots = a.q_all * a.heads, slot = (long long)blockIdx.x * (JOIN_THREADS / 64) + wave;
    Joined j;
    if (slot >= slots || !joined(a, slot, &j)) return;
    float2 ml = make_float2(-__builtin_inff(), 0.f);
    if (lane < j.splits) ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (lane * slots + slot));
    float m = ml.x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
    // (a split without keys has no part in it; one whose scores are all NaN has)
    const float w = ml.y == 0.f ? 0.f : ml.x == m ? 1.f : __builtin_amdgcn_exp2f(ml.x - m);
    float total = ml.y == 0.f ? 0.f : w * ml.y;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += __shfl_xor(total, o);
    float v0 = 0.f, v1 = 0.f;
    const float *p = a.part_o + slot * a.D + lane;
#pragma unroll 4
    for (int s = 0; s < j.splits; ++s) {
        const float x = __shfl(w, s);
        const float *const from = p + s * slots * a.D;
        const float y0 = lane < a.D ? from[0] : 0.f, y1 = lane + 64 < a.D ? from[64] : 0.f;
        v0 = x == 0.f ? v0 : fmaf(x, y0, v0);
        v1 = x == 0.f ? v1 : fmaf(x, y1, v1);
    }
    T *const out = joined_row<T>(a, j);
    if (lane < a.D) out[lane] = (T)(total == 0.f ? 0.f : v0 / total);
    if (lane + 64 < a.D) out[lane + 64] = (T)(total == 0.f ? 0.f : v1 / total);
    if (a.saved && lane == 0) save_joined(a, slot, m, total);
}

} // namespace attn

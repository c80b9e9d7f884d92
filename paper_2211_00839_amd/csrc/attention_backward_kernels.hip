// Attention's gradients, which compute the probabilities again from the scores and what the forward call saved of each row:
//
//   p = exp(s - max) / sum,   dp = dout v,   delta = dout out,   ds = p (dp - delta)
//   dq = scale ds K,   dk = scale ds^T Q,   dv = p^T dout,   d bias[c] = the sum of ds over the pairs of bucket c
//
// Two kernels, one that goes along the keys of its rows of q (dq, the bias) and one that goes along the queries of its rows of k (dk, dv; all
// the query heads that share the key head, one after the other): each sum stays in one wave's registers and has one order.
// Seven products where the formulas have five; the two that are made twice cost less than a sum of dq over the workgroups through memory
// (T / 128 times dq in fp32, written and read), and atomics would give them no fixed order.
//
// Bound by the matrix cores beside one exponential a pair in each kernel.  Measured, bf16, 2 x 8192 tokens, 16 heads of 128: k_attention_dq 1.48 ms (three products,
// 1110 TFLOP/s), k_attention_dkv 2.13 ms (four, 1030); 4 x 2048 x 16 heads of 64 with a bias 200 and 219 us (510 and 630).
#pragma once
#include "attention_common.h"

namespace attn {

// SHARED false: a workgroup's four waves have 32 rows each and share the tiles they go along; true, where that would make few workgroups: they
// have the same 32 rows, go along every fourth tile of 32 each by itself, and add up at the end.
template <typename T, int DP, bool SHARED, bool BIAS> struct Backward {
    using R = Row<T, DP>;
    static constexpr int ROWS = SHARED ? 32 : 128, LOADERS = SHARED ? 64 : THREADS;
    static constexpr int TILE = SHARED || R::BYTES == 512 || (BIAS && R::BYTES == 256) ? 32 : 64;       // rows in LDS at once
    static constexpr int STAGES = SHARED && (R::BYTES == 512 || (BIAS && R::BYTES == 256)) ? 1 : 2;
    static constexpr int HALF = TILE * R::BYTES, STAGE = 2 * HALF, TILES_BYTES = STAGES * STAGE * (SHARED ? 4 : 1);
    static constexpr int LOADS = 2 * TILE * R::CHUNKS / LOADERS;
    // the bias's gradient: a wave's block of ds on its way to the sums along its diagonals
    static constexpr int TURN_PITCH = 40, TURN_BYTES = 32 * TURN_PITCH * 4;
    static_assert(!SHARED || 4 * DP * 32 * 4 <= TILES_BYTES, "the waves' sums fit where the tiles were");
    // gradients of k and v.  Of wide bf16 rows two waves to a SIMD have no registers for their rows of v, which lie in LDS, and tiles of 32
    // leave room for them (T 8192, 32 heads of 128: 2.40 ms; one wave to a SIMD with all of it in registers 3.0, with the two products of
    // a block side by side and spilled registers 2.9).
    static constexpr bool TIGHT = !SHARED && sizeof(T) == 2 && DP == 128;
    static constexpr int KV_TILE = TIGHT ? 32 : TILE, KV_HALF = KV_TILE * R::BYTES, KV_STAGE = 2 * KV_HALF, KV_TILES_BYTES = STAGES * KV_STAGE * (SHARED ? 4 : 1),
                         KV_LOADS = 2 * KV_TILE * R::CHUNKS / LOADERS, V_BYTES = TIGHT ? 128 * R::BYTES : 0;
    // what is known of each query of a tile
    static constexpr int FACTS = BIAS ? 3 : 2, FACTS_STAGE = FACTS * KV_TILE, FACTS_BYTES = STAGES * FACTS_STAGE * 4 * (SHARED ? 4 : 1);
};

// The four waves' sums, a quarter of the elements in each wave: groups of four elements from 8 wave BLOCKS on.  Every wave has to come along.
template <int BLOCKS> __device__ __forceinline__ void add_waves(unsigned char *lds, f32x16 (&acc)[BLOCKS])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float *const sums = reinterpret_cast<float *>(lds);
    tile::wait_lds();
    tile::meet();
#pragma unroll
    for (int d = 0; d < BLOCKS; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[((wave * BLOCKS + d) * 16 + i) * 64 + lane] = acc[d][i];
    tile::wait_lds();
    tile::meet();
#pragma unroll
    for (int g = 0; g < BLOCKS; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v += sums[((w * BLOCKS * 4 + wave * BLOCKS + g) * 4 + e) * 64 + lane];
            acc[g >> 2][4 * (g & 3) + e] = v;
        }
}
// Rows of results: groups of four elements from element `first` on, as many as there are in `acc` (shared: of this wave's quarter).
template <typename T, int BLOCKS, int GROUPS, bool WHOLE>
__device__ __forceinline__ void store_row(T *to, int first, int D_, float scale, bool there, const f32x16 (&acc)[BLOCKS])
{
    const int D = opaque(D_), e0 = opaque(first);
    // (a row behind its sequence: zeros, whatever the weights of its zeros came to)
    auto of = [&](float x) { return there ? x * scale : 0.f; };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int e = e0 + 8 * g, x = g >> 2, y = 4 * (g & 3);
        if (e < D) store4<T, WHOLE>(to + e, D - e, of(acc[x][y]), of(acc[x][y + 1]), of(acc[x][y + 2]), of(acc[x][y + 3]));
    }
}

template <typename T, int DP, bool SHARED, bool BIAS, bool DIRECT>
__global__ __launch_bounds__(THREADS, sizeof(T) == 2 && !SHARED ? 2 : 1) void k_attention_dq(Args a)
{
    using W = Backward<T, DP, SHARED, BIAS>;
    using R = Row<T, DP>;
    constexpr int BLOCKS = W::TILE / 32;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int id = blockIdx.x;
    do {
        int b, head, first_tile, tiles_here = a.tiles;
        long long part_at;                                      // this workgroup's part of the bias's gradient, of its head's
        bool nothing = false;
        if (a.packed) {
            const int slot = divide(id, a.by_heads, &head);
            part_at = (long long)head * a.slots + slot;
            int of;
            if (tile_of<THREADS>(
                    a.batch, slot, lds, [&](int b) { return tiles_between(a.q_offsets, a.q_rows, b, 1, W::ROWS); }, &b, &first_tile, &of)) {
                first_tile = of - 1 - first_tile;               // (causal: the longest first)
                tiles_here = of;
            } else {
                // those left over clear the rows that belong to no sequence
                if (a.clear) clear_rows<T>(a.dq, a.q_offsets, a.batch, a.q_rows, head, a.D, slot - first_tile, a.slots + 1 - first_tile);
                nothing = true;
            }
            if (slot >= a.slots) continue;                      // (the one behind them has no part)
        } else {
            Unit unit;
            if (!unit_of(a, id, a.batch + (a.clear && a.q_offsets ? 1 : 0), &unit)) continue;
            int in_turn;
            b = unit.sequence;
            head = unit.kv_head * a.group + divide(unit.in, a.by_tiles, &in_turn);
            first_tile = a.tiles - 1 - in_turn;
            part_at = ((long long)head * a.batch + b) * a.tiles + first_tile;
            if (b == a.batch) {
                clear_rows<T>(a.dq, a.q_offsets, a.batch, a.q_rows, head, a.D, first_tile, a.tiles);
                continue;
            }
        }
        const int kv_head = divide(head, a.by_group);
        const int buckets = a.bias.buckets, all = a.bias.both ? 2 * buckets : buckets;
        float *const part = BIAS && a.part_bias ? a.part_bias + part_at * all : nullptr;
        if (nothing) {
            if (part)
                for (int c = tid; c < all; c += THREADS) part[c] = 0.f;
            continue;
        }
        const Sequence seq = sequence(a, b);
        if (first_tile * W::ROWS >= seq.q_len) {
            if (part)
                for (int c = tid; c < all; c += THREADS) part[c] = 0.f;
            continue;
        }
        const int shift = seq.k_len - seq.q_len;
        const bool q_ragged = a.q_offsets != nullptr, k_ragged = a.k_offsets != nullptr;
        const char *const keys = rows_of(a.k, b, k_ragged, seq.k0, kv_head), *const values = rows_of(a.v, b, k_ragged, seq.k0, kv_head);
        const int reach = a.bias.reach, width = BIAS ? bias_width(reach, a.causal) : 0, entries = BIAS ? bias_entries(reach, a.causal) : 0;
        float *const table = reinterpret_cast<float *>(lds + W::TILES_BYTES);
        float *const turn = reinterpret_cast<float *>(lds + W::TILES_BYTES + wave * W::TURN_BYTES) + width;
        float *const nears = reinterpret_cast<float *>(lds + W::TILES_BYTES + 4 * W::TURN_BYTES) + width;         // [wave][entries]
        float *const mine_near = nears + wave * entries;
        float far_before = 0.f, far_behind = 0.f;
        if constexpr (BIAS) {
            fill_bias(a, head, 1, table);
            for (int e = lane; e < entries; e += 64) mine_near[e] = 0.f;
            tile::wait_lds();
            tile::meet();
        }
        unsigned char *const stages = lds + (SHARED ? wave * W::STAGES * W::STAGE : 0);
        const unsigned stages_addr = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds + (SHARED ? wave * W::STAGES * W::STAGE : 0);
        const int loader = SHARED ? 0 : wave;
        Reader<T, DP> reader;
        reader.init();
        Loader<T, DP, W::TILE, W::LOADERS, DIRECT> load_k, load_v;
        load_k.init(a.k.row, a.D, SHARED ? lane : tid);
        load_v.init(a.v.row, a.D, SHARED ? lane : tid);
        for (int tile0 = first_tile * W::ROWS; tile0 < seq.q_len; tile0 += tiles_here * W::ROWS) {
            const int mine0 = tile0 + (SHARED ? 0 : wave * 32), row = mine0 + (lane & 31), h_row = min(row, seq.q_len - 1), pos = shift + h_row;
            const bool there = row < seq.q_len;
            const long long place = seq.q_first + h_row;
            const int last = shift + min(tile0 + W::ROWS, seq.q_len) - 1, end = a.causal ? max(0, min(seq.k_len, last + 1)) : seq.k_len;
            const int lowest = shift + mine0, highest = shift + min(mine0 + 32, seq.q_len) - 1;
            const int tiles = (end + W::TILE - 1) / W::TILE, t0 = SHARED ? wave : 0, step = SHARED ? 4 : 1;
            auto load = [&](int t, int buf) {
                const int k0 = t * W::TILE;
                unsigned char *const to = stages + buf * W::STAGE;
                const unsigned to_addr = stages_addr + buf * W::STAGE;
                load_k.issue(to, to_addr, keys + (long long)k0 * a.k.row, end - k0, a.D, loader);
                load_v.issue(to + W::HALF, to_addr + W::HALF, values + (long long)k0 * a.v.row, end - k0, a.D, loader);
            };
            if (W::STAGES == 2 && t0 < tiles) load(t0, 0);
            uint4 q[R::STEPS], g[R::STEPS];
            float delta = 0.f;
            {
                const char *pq = rows_of(a.q, b, q_ragged, seq.q0 + h_row, head), *pg = rows_of(a.dout, b, q_ragged, seq.q0 + h_row, head),
                           *po = rows_of(a.o, b, q_ragged, seq.q0 + h_row, head);
                uint4 o[R::STEPS];
#pragma unroll
                for (int s = 0; s < R::STEPS; ++s) {
                    q[s] = chunk_of<T, DIRECT>(pq, 2 * s + half, a.D);
                    g[s] = chunk_of<T, DIRECT>(pg, 2 * s + half, a.D);
                    o[s] = chunk_of<T, DIRECT>(po, 2 * s + half, a.D);
                }
#pragma unroll
                for (int s = 0; s < R::STEPS; ++s) {
                    if (!there) q[s] = g[s] = o[s] = make_uint4(0, 0, 0, 0);
                    const unsigned x[4] = {g[s].x, g[s].y, g[s].z, g[s].w}, y[4] = {o[s].x, o[s].y, o[s].z, o[s].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (sizeof(T) == 4) {
                            delta = fmaf(__builtin_bit_cast(float, x[e]), __builtin_bit_cast(float, y[e]), delta);
                        } else {
                            delta = fmaf(__builtin_bit_cast(float, x[e] << 16), __builtin_bit_cast(float, y[e] << 16), delta);
                            delta = fmaf(__builtin_bit_cast(float, x[e] & 0xffff0000u), __builtin_bit_cast(float, y[e] & 0xffff0000u), delta);
                        }
                    }
                }
            }
            delta = add_halves(delta);
            float top = __builtin_inff(), log_sum = 0.f;
            if (there) {
                const float2 v = *reinterpret_cast<const float2 *>(a.saved + 2 * (place * a.heads + head));
                top = v.x;
                log_sum = v.y;
            }
            arrive(q);
            arrive(g);
            const float both = top + log_sum;
            if (there && half == 0 && (!SHARED || wave == 0)) {
                float *const to = a.stats + (long long)head * a.q_all + place;
                to[0] = both;
                to[a.plane] = delta;
                to[2 * a.plane] = top;
                to[3 * a.plane] = log_sum;
            }
            f32x16 acc[1][R::BLOCKS];
#pragma unroll
            for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[0][d][i] = 0.f;
            bool left_out = false;
            // One tile.  edge: some of it is masked; near: its offsets are not all in the bias's last bucket.
            auto compute = [&](bool edge, bool near, int k0, const unsigned char *ktile) {
                const unsigned char *const vtile = ktile + W::HALF;
                const bool skip = a.causal && min(k0 + W::TILE, end) - 1 > lowest && any_not_finite<T, DP, W::TILE>(ktile);
                left_out |= skip;
#pragma unroll
                for (int kb = 0; kb < BLOCKS; ++kb) {
                    __builtin_amdgcn_sched_barrier(0);          // (a block's fragments at a time: there are no registers for more)
                    const int j0 = k0 + 32 * kb;
                    f32x16 of[2], ds[1];
                    scores<T, DP>(reader, ktile, vtile, kb, q, g, of);
                    f32x16 &s = of[0];
                    const f32x16 &dp = of[1];
                    if constexpr (BIAS) {
                        if (near) {
                            const float *const bias = table + (j0 - pos) + 4 * half + reach + MARGIN;
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], a.scale2, bias[row_of(i, 0)]);
                        } else {
                            const float bias = far_bias(a, table, k0 + W::TILE - 1 - lowest);
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], a.scale2, bias);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        ds[0][i] = __builtin_amdgcn_exp2f(BIAS ? (s[i] - top) - log_sum : fmaf(s[i], a.scale2, -both)) * (dp[i] - delta);
                    if (edge) {
                        // (a row that sees one key alone has p = 1 and dp = delta: nothing, where the two roundings of one number would leave a residue;
                        // such a row's key is the first, which lies in a tile of this kind)
                        const int seen = min(a.causal ? pos : end - 1, end - 1), most = (seen == 0 ? -1 : seen) - j0;
#pragma unroll
                        for (int i = 0; i < 16; ++i) ds[0][i] = row_of(i, half) <= most ? ds[0][i] : 0.f;
                    }
                    if (BIAS && !near) {
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum += ds[0][i];
                        if (k0 + W::TILE - 1 - lowest <= -reach) far_before += sum;
                        else far_behind += sum;
                    }
                    if (BIAS && near) {
                        // lane l sums the diagonal of offset j0 - (lowest + 31) + l, each in its order
#pragma unroll
                        for (int i = 0; i < 16; ++i) turn[row_of(i, half) * W::TURN_PITCH + (lane & 31)] = ds[0][i];
                        asm volatile("" ::: "memory");
                        float sum = 0.f;
#pragma unroll
                        for (int r = 0; r < 32; ++r) {
                            const int c = r + 31 - lane;
                            const float x = turn[r * W::TURN_PITCH + (c & 31)];
                            sum += c >= 0 && c < 32 ? x : 0.f;
                        }
                        asm volatile("" ::: "memory");
                        const int offset = j0 - (lowest + 31) + lane;
                        if (lane < 63) {
                            if (offset <= -reach) far_before += sum;
                            else if (a.causal ? offset > 0 : offset >= reach) far_behind += sum;       // (causal: zeros)
                            else mine_near[offset + reach] += sum;
                        }
                    }
                    if (!skip) weigh<T, DP, 1>(reader, ktile, kb, ds, acc[0]);
                }
            };
            int buf = 0;
            for (int t = t0; t < tiles; t += step, buf ^= W::STAGES - 1) {
                if constexpr (SHARED) {
                    tile::wait_lds();
                    if (W::STAGES == 1) {
                        load(t, 0);
                        tile::wait_loads<0>();
                    } else if (t + step < tiles) {
                        load(t + step, buf ^ 1);
                        if (DIRECT) tile::wait_loads<W::LOADS>();
                    } else {
                        tile::wait_loads<0>();
                    }
                } else {
                    tile::wait_loads<0>();
                }
                if (end - t * W::TILE < W::TILE) load_k.clear(stages + buf * W::STAGE, end - t * W::TILE, loader);
                tile::wait_lds();
                if constexpr (!SHARED) {
                    tile::meet();
                    if (t + 1 < tiles) load(t + 1, buf ^ 1);
                }
                const int k0 = t * W::TILE;
                if (!SHARED && ((a.causal && k0 > highest) || mine0 >= seq.q_len)) continue;
                const unsigned char *const ktile = stages + buf * W::STAGE;
                const bool edge = k0 + W::TILE > end || (a.causal && k0 + W::TILE - 1 > lowest);
                compute(edge, BIAS && !is_far(a, k0 - (lowest + 31), k0 + W::TILE - 1 - lowest), k0, ktile);
            }
            if (!SHARED && a.causal) tile::meet();
            if (left_out) {
                // the tiles on the border that hold something that is not finite
                const char *const mine = rows_of(a.q, b, q_ragged, seq.q0 + h_row, head), *const my_grad = rows_of(a.dout, b, q_ragged, seq.q0 + h_row, head);
                add_rows<T, DP>(SHARED ? stages : lds + wave * 4096, a.D, acc[0], [&](auto add) {
#pragma unroll 1
                    for (int t = t0; t < tiles; t += step) {
                        const int j0 = t * W::TILE, count = min(W::TILE, end - j0);
                        if (j0 + count - 1 <= lowest || j0 > highest) continue;
                        if (!any_not_finite<T>(keys + (long long)j0 * a.k.row, a.k.row, count, a.D)) continue;
#pragma unroll 1
                        for (int j = j0; j < j0 + count; ++j) {
                            if (j > pos || pos == 0 || !there) continue;       // (pos 0: one key alone)
                            const char *const key = keys + (long long)j * a.k.row;
                            float x = dot<T>(mine, key, a.D) * a.scale2;
                            if constexpr (BIAS) x += bias_at(a, head, j - pos);
                            const float p = __builtin_amdgcn_exp2f((x - top) - log_sum);
                            add(p * (dot<T>(my_grad, values + (long long)j * a.v.row, a.D) - delta), key);
                        }
                    }
                });
            }
            T *const to = reinterpret_cast<T *>(rows_of(a.dq, b, q_ragged, seq.q0 + h_row, head));
            if constexpr (SHARED) {
                add_waves<R::BLOCKS>(lds, acc[0]);
                if (there) store_row<T, R::BLOCKS, R::BLOCKS, DIRECT>(to, 8 * wave * R::BLOCKS + 4 * half, a.D, a.scale, true, acc[0]);
            } else {
                if (there) store_row<T, R::BLOCKS, 4 * R::BLOCKS, DIRECT>(to, 4 * half, a.D, a.scale, true, acc[0]);
            }
            tile::wait_loads<0>();
            tile::wait_lds();
            tile::meet();
        }
        if constexpr (BIAS) {
            if (!part) continue;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                far_before += __shfl_xor(far_before, o);
                far_behind += __shfl_xor(far_behind, o);
            }
            float *const far = table;           // (the bias itself is not needed any more)
            if (lane == 0) {
                far[2 * wave] = far_before;
                far[2 * wave + 1] = far_behind;
            }
            tile::wait_lds();
            tile::meet();
            // Several threads to a bucket where there are few: a wide one has a hundred numbers to add, which short sequences wait for (100 samples of 1
            // to 512 tokens, 8 heads of 64, a training step: 184 us; with one thread to a bucket 197).
            // (The thread's number is looked at anew: kept from fill_bias() on, it would be a register that the compiler has to put somewhere all the while.)
            const int parts = all <= 32 ? 8 : all <= 64 ? 4 : all <= 128 ? 2 : 1, me = opaque(tid), c = me / parts, k = me % parts;
            float sum = 0.f;
            if (c < all) {
                const int in = c < buckets ? c : c - buckets, sign = c < buckets ? -1 : 1;
                if (in == buckets - 1) {
                    for (int w = k; w < 4; w += parts) sum += far[2 * w + (sign > 0 ? 1 : 0)];
                } else {
                    int from, to;
                    distances(a.bias, in, &from, &to);
                    for (int r = max(from, sign > 0 ? 1 : 0) + k; r < to; r += parts) {
                        const float *const at = nears + sign * r + reach;
                        sum += (at[0] + at[entries]) + (at[2 * entries] + at[3 * entries]);
                    }
                }
            }
            for (int o = 1; o < parts; o <<= 1) sum += __shfl_xor(sum, o);
            if (c < all && k == 0) part[c] = sum;
            tile::wait_lds();
            tile::meet();
        }
    } while (SHARED && (id += (int)gridDim.x) < a.workgroups);
}

// Adds up the table's gradient over the workgroups that computed parts of it: a workgroup for each bucket and head.
template <typename T> __global__ __launch_bounds__(THREADS) void k_bias_gradient(const float *parts, long long count, int all, int heads, T *to)
{
    __shared__ float sums[4];
    const int c = blockIdx.x % all, head = blockIdx.x / all;
    float sum = 0.f;
    for (long long p = threadIdx.x; p < count; p += THREADS) sum += parts[((long long)head * count + p) * all + c];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) to[c * heads + head] = (T)((sums[0] + sums[1]) + (sums[2] + sums[3]));
}

template <typename T, int DP, bool SHARED, bool BIAS, bool DIRECT> __global__ __launch_bounds__(THREADS, sizeof(T) == 2 && !SHARED ? 2 : 1) void k_attention_dkv(Args a)
{
    using W = Backward<T, DP, SHARED, BIAS>;
    using R = Row<T, DP>;
    constexpr int BLOCKS = W::KV_TILE / 32;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int id = blockIdx.x;
    do {
        int b, kv_head, split, first_tile, tiles_here = a.tiles;
        if (a.packed) {
            int in;
            const int slot = divide(id, a.by_heads, &in);
            kv_head = divide(in, a.by_splits, &split);
            int of;
            if (!tile_of<THREADS>(
                    a.batch, slot, lds, [&](int b) { return tiles_between(a.k_offsets, a.k_rows, b, 1, W::ROWS); }, &b, &first_tile, &of)) {
                if (a.clear && split == 0) {
                    clear_rows<T>(a.dk, a.k_offsets, a.batch, a.k_rows, kv_head, a.D, slot - first_tile, a.slots + 1 - first_tile);
                    clear_rows<T>(a.dv, a.k_offsets, a.batch, a.k_rows, kv_head, a.D, slot - first_tile, a.slots + 1 - first_tile);
                }
                continue;
            }
            tiles_here = of;
        } else {
            Unit unit;
            if (!unit_of(a, id, a.batch + (a.clear && a.k_offsets ? 1 : 0), &unit)) continue;
            b = unit.sequence;
            kv_head = unit.kv_head;
            first_tile = divide(unit.in, a.by_splits, &split);          // (causal: the first keys have the most queries)
            if (b == a.batch) {
                if (split > 0) continue;
                clear_rows<T>(a.dk, a.k_offsets, a.batch, a.k_rows, kv_head, a.D, first_tile, a.tiles);
                clear_rows<T>(a.dv, a.k_offsets, a.batch, a.k_rows, kv_head, a.D, first_tile, a.tiles);
                continue;
            }
        }
        const Sequence seq = sequence(a, b);
        const int shift = seq.k_len - seq.q_len;
        const bool q_ragged = a.q_offsets != nullptr, k_ragged = a.k_offsets != nullptr;
        unsigned char *const my_values = lds + W::KV_TILES_BYTES + wave * 32 * R::BYTES;       // (TIGHT)
        float *const all_facts = reinterpret_cast<float *>(lds + W::KV_TILES_BYTES + W::V_BYTES), *const table = all_facts + W::FACTS_BYTES / 4;
        float *const facts = all_facts + (SHARED ? wave * W::STAGES * W::FACTS_STAGE : 0);
        unsigned char *const stages = lds + (SHARED ? wave * W::STAGES * W::KV_STAGE : 0);
        const unsigned lds_addr = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;
        const unsigned stages_addr = lds_addr + (SHARED ? wave * W::STAGES * W::KV_STAGE : 0);
        const unsigned facts_addr = lds_addr + W::KV_TILES_BYTES + W::V_BYTES + (SHARED ? wave * W::STAGES * W::FACTS_STAGE * 4 : 0);
        const int loader = SHARED ? 0 : wave;
        int table_of = -1;                                          // the query head whose bias is there
        Reader<T, DP> reader;
        reader.init();
        Loader<T, DP, W::KV_TILE, W::LOADERS, DIRECT> load_q, load_g;
        load_q.init(a.q.row, a.D, SHARED ? lane : tid);
        load_g.init(a.dout.row, a.D, SHARED ? lane : tid);
        const int rows = a.clear && !k_ragged ? a.k_rows : seq.k_len;       // rows behind the sequence get zeros
        for (int tile0 = first_tile * W::ROWS; tile0 < rows; tile0 += tiles_here * W::ROWS) {
            const int mine0 = tile0 + (SHARED ? 0 : wave * 32), key = mine0 + (lane & 31), h_key = min(key, seq.k_len - 1);
            const bool there = key < seq.k_len;
            const int q_tiles = (seq.q_len + W::KV_TILE - 1) / W::KV_TILE, q_from = a.causal ? min(max(0, tile0 - shift) / W::KV_TILE, q_tiles) : 0;
            const int per = tile0 < seq.k_len ? q_tiles - q_from : 0;
            // this workgroup's tiles, of all the heads' end to end: c0 .. c1 - 1
            const int count = per * a.group, c0 = (int)((long long)count * split / a.splits), c1 = (int)((long long)count * (split + 1) / a.splits);
            const int c_mine = c0 + (SHARED ? wave : 0), c_first = SHARED && BIAS && c1 > c0 ? min(c1, (c0 / per + 1) * per) : c1;      // (its first head's end)
            auto load = [&](int g, int t, int buf) {
                const int i0 = (q_from + t) * W::KV_TILE, head = kv_head * a.group + g;
                const char *pq = rows_of(a.q, b, q_ragged, seq.q0 + i0, head), *pg = rows_of(a.dout, b, q_ragged, seq.q0 + i0, head);
                unsigned char *const to = stages + buf * W::KV_STAGE;
                const unsigned to_addr = stages_addr + buf * W::KV_STAGE;
                load_q.issue(to, to_addr, pq, seq.q_len - i0, a.D, loader);
                load_g.issue(to + W::KV_HALF, to_addr + W::KV_HALF, pg, seq.q_len - i0, a.D, loader);
                // what the exponents are taken from, delta, and with a bias the sum's logarithm by itself: a plane of each
#pragma unroll
                for (int f = 0; f < W::FACTS; ++f) {
                    if (!SHARED && wave != f) continue;
                    const int plane = !BIAS ? f : f == 0 ? 2 : f == 1 ? 1 : 3;
                    const float *from = a.stats + plane * a.plane + (long long)head * a.q_all + seq.q_first + i0;
                    if (lane < W::KV_TILE) tile::load4_to_lds(uniform(from), min(lane, seq.q_len - 1 - i0) * 4, facts_addr + (buf * W::FACTS_STAGE + f * W::KV_TILE) * 4);
                }
            };
            // A tile that has come; rows that are not there become zeros with weights of zero.
            auto clear = [&](int i0, int buf) {
                const int rows = seq.q_len - i0;
                if (rows >= W::KV_TILE) return;
                load_q.clear(stages + buf * W::KV_STAGE, rows, loader);
                load_g.clear(stages + buf * W::KV_STAGE + W::KV_HALF, rows, loader);
#pragma unroll
                for (int f = 0; f < W::FACTS; ++f) {
                    if (!SHARED && wave != f) continue;
                    if (lane < W::KV_TILE && lane >= rows) facts[buf * W::FACTS_STAGE + f * W::KV_TILE + lane] = f == 0 ? __builtin_inff() : 0.f;
                }
            };
            // a tile is the t-th of head g; steps go through them without dividing each time
            int g = per > 0 ? c_mine / per : 0, t = c_mine - g * per;
            if (W::STAGES == 2 && c_mine < c_first) load(g, t, 0);
            uint4 k[R::STEPS], v[W::TIGHT ? 1 : R::STEPS];
            {
                const char *pk = rows_of(a.k, b, k_ragged, seq.k0 + max(h_key, 0), kv_head), *pv = rows_of(a.v, b, k_ragged, seq.k0 + max(h_key, 0), kv_head);
#pragma unroll
                for (int s = 0; s < R::STEPS; ++s) {
                    uint4 x = make_uint4(0, 0, 0, 0), y = x;
                    if (c1 > c0) {
                        x = chunk_of<T, DIRECT>(pk, 2 * s + half, a.D);
                        y = chunk_of<T, DIRECT>(pv, 2 * s + half, a.D);
                    }
                    k[s] = x;
                    if constexpr (W::TIGHT) *reinterpret_cast<uint4 *>(my_values + (reader.here ^ (s << 5))) = y;
                    else v[s] = y;
                }
            }
            arrive(k);
            if constexpr (!W::TIGHT) arrive(v);
            f32x16 dk[1][R::BLOCKS], dv[1][R::BLOCKS];
#pragma unroll
            for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) dk[0][d][i] = dv[0][d][i] = 0.f;
            bool left_out = false;
            auto compute = [&](bool edge, bool near, int i_tile, int buf) {
                const unsigned char *const qtile = stages + buf * W::KV_STAGE, *const gtile = qtile + W::KV_HALF;
                const float *const fact = facts + buf * W::FACTS_STAGE;
                const bool skip = edge && (any_not_finite<T, DP, W::KV_TILE>(gtile) || any_not_finite<T, DP, W::KV_TILE>(qtile));
                left_out |= skip;
#pragma unroll
                for (int rb = 0; rb < BLOCKS; ++rb) {
                    const int p0 = shift + i_tile + 32 * rb;
                    f32x16 p[1], ds[1];
                    if constexpr (W::TIGHT) {
                        scores<T, DP, 1>(reader, qtile + 32 * rb * R::BYTES, k, p);
                    } else {
                        f32x16 of[2];
                        scores<T, DP>(reader, qtile, gtile, rb, k, v, of);
                        p[0] = of[0];
                        ds[0] = of[1];
                    }
                    if constexpr (BIAS) {
                        if (near) {
                            const float *const bias = table + (key - p0) - 4 * half + a.bias.reach + MARGIN;
#pragma unroll
                            for (int i = 0; i < 16; ++i) p[0][i] = fmaf(p[0][i], a.scale2, bias[-row_of(i, 0)]);
                        } else {
                            const float bias = far_bias(a, table, mine0 + 31 - (shift + i_tile));
#pragma unroll
                            for (int i = 0; i < 16; ++i) p[0][i] = fmaf(p[0][i], a.scale2, bias);
                        }
                    }
                    const float *const known = fact + 32 * rb + 4 * half;
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const f32x4 from = *reinterpret_cast<const f32x4 *>(known + 8 * f);
                        f32x4 log_sum = {0.f, 0.f, 0.f, 0.f};
                        if constexpr (BIAS) log_sum = *reinterpret_cast<const f32x4 *>(known + 2 * W::KV_TILE + 8 * f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = p[0][4 * f + e];
                            p[0][4 * f + e] = __builtin_amdgcn_exp2f(BIAS ? (x - from[e]) - log_sum[e] : fmaf(x, a.scale2, -from[e]));
                        }
                    }
                    // least: the first position whose query sees this lane's key
                    auto hide = [&](f32x16 &x, int least) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = least <= p0 + row_of(i, half) ? x[i] : 0.f;
                    };
                    if constexpr (W::TIGHT) {
                        if (edge) hide(p[0], key);
                        if (!skip) weigh<T, DP, 1>(reader, gtile, rb, p, dv[0]);
                        __builtin_amdgcn_sched_barrier(0);
                        struct Pair {
                            uint4 theirs, mine;
                        };
                        const int here = opaque(reader.here);
                        set_zero(ds);
                        in_turn<R::STEPS, 2>([&](int i) { return Pair{reader.along(gtile, here, rb, i), reader.along(my_values, here, 0, i)}; },
                                             [&](int i, const Pair &x) { ds[0] = scores<T>(x.theirs, x.mine, ds[0]); });
                    }
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const f32x4 delta = *reinterpret_cast<const f32x4 *>(known + W::KV_TILE + 8 * f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) ds[0][4 * f + e] = p[0][4 * f + e] * (ds[0][4 * f + e] - delta[e]);
                    }
                    if (edge) {
                        if (!W::TIGHT) hide(p[0], key);
                        hide(ds[0], max(key, 1));           // (position 0 sees one key alone: its ds is nothing, as in k_attention_dq)
                    }
                    if (!skip) {
                        if (!W::TIGHT) weigh<T, DP, 1>(reader, gtile, rb, p, dv[0]);
                        weigh<T, DP, 1>(reader, qtile, rb, ds, dk[0]);
                    }
                    __builtin_amdgcn_sched_barrier(0);          // (a block's fragments at a time: there are no registers for more)
                }
            };
            auto choose = [&](int i_tile, int buf) {
                const int p0 = shift + i_tile, p1 = p0 + W::KV_TILE - 1;       // the tile's positions
                if (mine0 >= seq.k_len || (a.causal && p1 < mine0)) return;
                compute(a.causal && p0 < mine0 + 31, BIAS && !is_far(a, mine0 - p1, mine0 + 31 - p0), i_tile, buf);
            };
            // Brings the bias of a query head; every wave has to come along.
            auto bias_of = [&](int g) {
                fill_bias(a, kv_head * a.group + g, 1, table);
                table_of = g;
                tile::wait_lds();
                tile::meet();
            };
            int buf = 0;
            auto next = [&](int step) {
                t += step;
                while (t >= per) {
                    t -= per;
                    ++g;
                }
            };
            if constexpr (SHARED) {
                // with a bias head by head, since it is a head's: end is where this head's tiles end
                int from = c0;
                do {
                    const int head = per > 0 ? from / per : 0, end = BIAS ? min(c1, (head + 1) * per) : c1;
                    if constexpr (BIAS)
                        if (from < c1 && head != table_of) {
                            tile::wait_lds();
                            tile::meet();
                            bias_of(head);
                        }
                    if (from + wave < end) {
                        g = (from + wave) / per;
                        t = from + wave - g * per;
                    }
                    for (int c = from + wave; c < end; c += 4, buf ^= W::STAGES - 1) {
                        const int i_tile = (q_from + t) * W::KV_TILE;
                        tile::wait_lds();
                        if (W::STAGES == 1) {
                            load(g, t, 0);
                            next(4);
                            tile::wait_loads<0>();
                        } else {
                            if (c == from + wave && from > c0) load(g, t, buf);
                            next(4);
                            if (c + 4 < end) {
                                load(g, t, buf ^ 1);
                                if (DIRECT) tile::wait_loads<W::KV_LOADS + W::FACTS>();
                                else tile::wait_loads<0>();
                            } else {
                                tile::wait_loads<0>();
                            }
                        }
                        clear(i_tile, buf);
                        tile::wait_lds();
                        choose(i_tile, buf);
                    }
                    from = end;
                } while (from < c1);
            } else {
                for (int c = c0; c < c1; ++c, buf ^= 1) {
                    const int g_now = g, i_tile = (q_from + t) * W::KV_TILE;
                    tile::wait_loads<0>();
                    clear(i_tile, buf);
                    tile::wait_lds();
                    tile::meet();
                    if constexpr (BIAS)
                        if (g_now != table_of) bias_of(g_now);
                    next(1);
                    if (c + 1 < c1) load(g, t, buf ^ 1);
                    choose(i_tile, buf);
                }
            }
            if (!SHARED && a.causal) tile::meet();
            if (left_out) {
                // the tiles on the border that hold something that is not finite
                const char *const mine = rows_of(a.k, b, k_ragged, seq.k0 + h_key, kv_head), *const my_value = rows_of(a.v, b, k_ragged, seq.k0 + h_key, kv_head);
                auto visit = [&](bool of_v, auto add) {
#pragma unroll 1
                        for (int c = c0; c < c1; ++c) {
                            if (SHARED && (c - (BIAS ? max(c0, c / per * per) : c0)) % 4 != wave) continue;
                            const int h = kv_head * a.group + c / per, i0 = (q_from + c % per) * W::KV_TILE, n = min(W::KV_TILE, seq.q_len - i0);
                            const char *const pq = rows_of(a.q, b, q_ragged, seq.q0 + i0, h), *const pg = rows_of(a.dout, b, q_ragged, seq.q0 + i0, h);
                            if (shift + i0 >= mine0 + 31 || shift + i0 + W::KV_TILE - 1 < mine0) continue;
                            if (!any_not_finite<T>(pg, a.dout.row, n, a.D) && !any_not_finite<T>(pq, a.q.row, n, a.D)) continue;
#pragma unroll 1
                            for (int i = 0; i < n; ++i) {
                                if (key > shift + i0 + i || !there) continue;
                                if (!of_v && shift + i0 + i == 0) continue;         // (one key alone)
                                const char *const row_q = pq + (long long)i * a.q.row, *const row_g = pg + (long long)i * a.dout.row;
                                const float *const fact = a.stats + (long long)h * a.q_all + seq.q_first + i0 + i;
                                float x = dot<T>(row_q, mine, a.D) * a.scale2;
                                if constexpr (BIAS) x += bias_at(a, h, key - shift - i0 - i);
                                const float p = __builtin_amdgcn_exp2f((x - fact[2 * a.plane]) - fact[3 * a.plane]);
                                if (of_v) add(p, row_g);
                                else add(p * (dot<T>(row_g, my_value, a.D) - fact[a.plane]), row_q);
                            }
                        }
                };
                add_rows<T, DP>(SHARED ? stages : lds + wave * 4096, a.D, dv[0], [&](auto add) { visit(true, add); });
                add_rows<T, DP>(SHARED ? stages : lds + wave * 4096, a.D, dk[0], [&](auto add) { visit(false, add); });
            }
            // What leaves: rows of dk and dv, or with splits their parts in fp32.
            const bool stored = a.splits > 1 ? there : key < rows;
            const long long place = ((split * a.k_all + seq.k_first + key) * a.kv_heads + kv_head) * a.D;
            constexpr int GROUPS = SHARED ? R::BLOCKS : 4 * R::BLOCKS;
            const int first = (SHARED ? 8 * wave * R::BLOCKS : 0) + 4 * half;
            auto store = [&](const Heads &to, float *parts, float scale, bool zeros, f32x16 (&acc)[R::BLOCKS]) {
                if constexpr (SHARED) add_waves<R::BLOCKS>(lds, acc);
                if (!stored) return;
                if (a.splits > 1) store_row<float, R::BLOCKS, GROUPS, DIRECT>(parts + place, first, a.D, 1.f, !zeros, acc);
                else store_row<T, R::BLOCKS, GROUPS, DIRECT>(reinterpret_cast<T *>(rows_of(to, b, k_ragged, seq.k0 + key, kv_head)), first, a.D, scale, there && !zeros, acc);
            };
            store(a.dk, a.part_k, a.scale, seq.k_len == 1, dk[0]);          // (a key that is alone: every weight of it is 1)
            store(a.dv, a.part_v, 1.f, false, dv[0]);
            tile::wait_loads<0>();
            tile::wait_lds();
            tile::meet();
        }
    } while (SHARED && (id += (int)gridDim.x) < a.workgroups);
}

// Adds up the splits' parts of dk and dv, four elements to a thread.
template <typename T> __global__ __launch_bounds__(THREADS) void k_attention_dkv_join(Args a)
{
    const int fours = (a.D + 3) / 4;
    const long long all = a.k_all * a.kv_heads * fours, each = a.k_all * a.kv_heads * a.D;
    for (long long at = (long long)blockIdx.x * THREADS + threadIdx.x; at < all; at += (long long)gridDim.x * THREADS) {
        const int d = (int)(at % fours) * 4, head = (int)(at / fours % a.kv_heads);
        const long long row = at / fours / a.kv_heads;
        int b = 0;
        long long in = row;
        bool there;
        if (a.k_offsets) {
            const int from = min(max(a.k_offsets[0], 0), a.k_rows), to = min(max(a.k_offsets[a.batch], from), a.k_rows);
            there = row >= from && row < to;
            if (!there) continue;               // (cleared, where they are to be, by the call's first kernel)
        } else {
            b = (int)(row / a.k_rows);
            in = row - (long long)b * a.k_rows;
            there = !a.k_lengths || in < min(max(a.k_lengths[b], 0), a.k_rows);
            if (!there && !a.clear) continue;
        }
        float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
        const long long first = (row * a.kv_heads + head) * a.D + d;
        const int count = min(4, a.D - d);
        if (there)
            for (int s = 0; s < a.splits; ++s) {
                const float *const pk = a.part_k + s * each + first, *const pv = a.part_v + s * each + first;
                if (count == 4) {
                    const f32x4 x = *reinterpret_cast<const f32x4_any *>(pk), y = *reinterpret_cast<const f32x4_any *>(pv);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        k[e] += x[e];
                        v[e] += y[e];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (e < count) {
                            k[e] += pk[e];
                            v[e] += pv[e];
                        }
                }
            }
        store4<T, false>(reinterpret_cast<T *>(rows_of(a.dk, b, a.k_offsets != nullptr, in, head)) + d, count, k[0] * a.scale, k[1] * a.scale, k[2] * a.scale, k[3] * a.scale);
        store4<T, false>(reinterpret_cast<T *>(rows_of(a.dv, b, a.k_offsets != nullptr, in, head)) + d, count, v[0], v[1], v[2], v[3]);
    }
}

} // namespace attn

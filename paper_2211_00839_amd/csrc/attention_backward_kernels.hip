// Attention's gradients, which compute the probabilities again from the scores and what the forward call saved of each row:
//
//   p = exp(s - max) / sum,   dp = dout v,   delta = dout out,   ds = p (dp - delta)
//   dq = scale ds K,   dk = scale ds^T Q,   dv = p^T dout,   d bias[c] = the sum of ds over the pairs of bucket c
//
// Two kernels, one that goes along the keys of its rows of q (dq, the bias) and one that goes along the queries of its rows of k (dk, dv; all
// the query heads that share the key head, one after the other): each sum stays in one wave's registers and has one order.
// Seven products where the formulas have five; the two that are made twice cost less than a sum of dq over the workgroups through memory
// (T / 128 times dq in fp32, written and read), and atomics would give them no fixed order.
#pragma once
#include "attention_common.h"

namespace attn {

template <typename T, int DP, bool BIAS> struct Backward {
    using R = Row<T, DP>;
    static constexpr int TILE = R::BYTES == 512 || (BIAS && R::BYTES == 256) ? 32 : 64;         // rows in LDS at once
    static constexpr int HALF = TILE * R::BYTES, STAGE = 2 * HALF, TILES_BYTES = 2 * STAGE;
    // gradients of k and v: what is known of each query of a tile
    static constexpr int FACTS = BIAS ? 3 : 2, FACTS_BYTES = 2 * FACTS * TILE * 4;
    // the bias's gradient: a wave's block of ds on its way to the sums along its diagonals
    static constexpr int TURN_PITCH = 40, TURN_BYTES = 32 * TURN_PITCH * 4;
};

template <typename T, int DP, bool BIAS, bool DIRECT>
__global__ __launch_bounds__(THREADS, sizeof(T) == 2 ? 2 : 1) void k_attention_dq(Args a)
{
    using W = Backward<T, DP, BIAS>;
    using R = Row<T, DP>;
    constexpr int ROWS = 128, BLOCKS = W::TILE / 32;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int total = a.tiles * a.heads * (a.batch + (a.clear && a.q_offsets ? 1 : 0));
    int at = place_of(blockIdx.x, total);
    if (at >= total) return;
    const int first_tile = a.tiles - 1 - at % a.tiles;
    at /= a.tiles;
    const int head = at % a.heads, b = at / a.heads;
    if (b == a.batch) {
        clear_rows<T>(a.dq, a.q_offsets, a.batch, a.q_rows, head, a.D, first_tile, a.tiles);
        return;
    }
    const Sequence seq = sequence(a, b);
    const int kv_head = head / a.group, shift = seq.k_len - seq.q_len;
    const bool q_ragged = a.q_offsets != nullptr, k_ragged = a.k_offsets != nullptr;
    const char *const keys = rows_of(a.k, b, k_ragged, seq.k0, kv_head), *const values = rows_of(a.v, b, k_ragged, seq.k0, kv_head);
    const int entries = BIAS ? bias_entries(a) : 0, reach = a.bias.reach;
    float *const table = reinterpret_cast<float *>(lds + W::TILES_BYTES);
    float *const turn = reinterpret_cast<float *>(lds + W::TILES_BYTES + wave * W::TURN_BYTES) + entries;
    float *const near = reinterpret_cast<float *>(lds + W::TILES_BYTES + 4 * W::TURN_BYTES) + entries;       // [wave][entries]
    float *const mine_near = near + wave * entries;
    float far_before = 0.f, far_behind = 0.f;
    if constexpr (BIAS) {
        fill_bias(a, head, table);
        for (int e = lane; e < entries; e += 64) mine_near[e] = 0.f;
    }
    const unsigned lds_addr = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;
    Reader<T, DP> reader;
    reader.init();
    Loader<T, DP, W::TILE, THREADS, DIRECT> load_k, load_v;
    load_k.init(a.k.row, a.D, tid);
    load_v.init(a.v.row, a.D, tid);
    for (int tile0 = first_tile * ROWS; tile0 < seq.q_len; tile0 += a.tiles * ROWS) {
        const int mine0 = tile0 + wave * 32, row = mine0 + (lane & 31), h_row = min(row, seq.q_len - 1), pos = shift + h_row;
        const bool there = row < seq.q_len;
        const long long place = seq.q_first + h_row;
        uint4 q[R::STEPS], g[R::STEPS];
        float delta = 0.f;
        {
            const char *pq = rows_of(a.q, b, q_ragged, seq.q0 + h_row, head), *pg = rows_of(a.dout, b, q_ragged, seq.q0 + h_row, head),
                       *po = rows_of(a.o, b, q_ragged, seq.q0 + h_row, head);
#pragma unroll
            for (int s = 0; s < R::STEPS; ++s) {
                q[s] = g[s] = make_uint4(0, 0, 0, 0);
                if (!there) continue;
                q[s] = chunk_of<T, DIRECT>(pq, 2 * s + half, a.D);
                g[s] = chunk_of<T, DIRECT>(pg, 2 * s + half, a.D);
                const uint4 o = chunk_of<T, DIRECT>(po, 2 * s + half, a.D);
                const unsigned x[4] = {g[s].x, g[s].y, g[s].z, g[s].w}, y[4] = {o.x, o.y, o.z, o.w};
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
        const float both = top + log_sum;
        if (there && half == 0) {
            float *const to = a.stats + (long long)head * a.q_all + place;
            to[0] = both;
            to[a.plane] = delta;
            to[2 * a.plane] = top;
            to[3 * a.plane] = log_sum;
        }
        const int last = shift + min(tile0 + ROWS, seq.q_len) - 1, end = a.causal ? max(0, min(seq.k_len, last + 1)) : seq.k_len;
        const int lowest = shift + mine0, highest = shift + min(mine0 + 32, seq.q_len) - 1;
        const int tiles = (end + W::TILE - 1) / W::TILE;
        auto load = [&](int t, int buf) {
            const int k0 = t * W::TILE;
            unsigned char *const to = lds + buf * W::STAGE;
            const unsigned to_addr = lds_addr + buf * W::STAGE;
            load_k.issue(to, to_addr, keys + (long long)k0 * a.k.row, end - k0, a.D, wave);
            load_v.issue(to + W::HALF, to_addr + W::HALF, values + (long long)k0 * a.v.row, end - k0, a.D, wave);
        };
        f32x16 acc[1][R::BLOCKS];
#pragma unroll
        for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[0][d][i] = 0.f;
        if (tiles > 0) load(0, 0);
        bool left_out = false;
        int buf = 0;
        for (int t = 0; t < tiles; ++t, buf ^= 1) {
            tile::wait_loads<0>();
            if (end - t * W::TILE < W::TILE) load_k.clear(lds + buf * W::STAGE, end - t * W::TILE, wave);
            tile::wait_lds();
            tile::meet();
            if (t + 1 < tiles) load(t + 1, buf ^ 1);
            const unsigned char *const ktile = lds + buf * W::STAGE, *const vtile = ktile + W::HALF;
#pragma unroll
            for (int kb = 0; kb < BLOCKS; ++kb) {
                const int j0 = t * W::TILE + 32 * kb;
                if (j0 >= end || (a.causal && j0 > highest) || mine0 >= seq.q_len) continue;
                const bool border = a.causal && j0 + 31 > lowest, edge = border || j0 + 32 > end;
                f32x16 s, dp;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
                for (int f = 0; f < R::STEPS; ++f) s = scores<T>(reader.along(ktile, kb, f), q[f], s);
#pragma unroll
                for (int f = 0; f < R::STEPS; ++f) dp = scores<T>(reader.along(vtile, kb, f), g[f], dp);
                if constexpr (BIAS) add_bias(a, table, j0 - pos, j0 - highest, j0 + 31 - lowest, a.scale2, s);
                f32x16 ds[1];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = __builtin_amdgcn_exp2f(BIAS ? (s[i] - top) - log_sum : fmaf(s[i], a.scale2, -both));
                    ds[0][i] = p * (dp[i] - delta);
                }
                if (edge) {
                    const int most = min(a.causal ? pos : end - 1, end - 1) - j0;
#pragma unroll
                    for (int i = 0; i < 16; ++i) ds[0][i] = row_of(i, half) <= most ? ds[0][i] : 0.f;
                }
                if constexpr (BIAS) {
                    const int lo = j0 - (lowest + 31), hi = j0 + 31 - lowest;       // offsets of the whole block
                    if (hi <= -reach || (!a.causal && lo >= reach)) {
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum += ds[0][i];
                        if (hi <= -reach) far_before += sum;
                        else far_behind += sum;
                    } else {
                        // lane l sums the diagonal of offset lo + l, each in its order
#pragma unroll
                        for (int i = 0; i < 16; ++i) turn[row_of(i, half) * W::TURN_PITCH + (lane & 31)] = ds[0][i];
                        asm volatile("" ::: "memory");
                        float sum = 0.f;
#pragma unroll
                        for (int r = 0; r < 32; ++r) {
                            const int c = r + 31 - lane;
                            if (c >= 0 && c < 32) sum += turn[r * W::TURN_PITCH + c];
                        }
                        asm volatile("" ::: "memory");
                        const int offset = lo + lane;
                        if (lane < 63) {
                            if (offset <= -reach) far_before += sum;
                            else if (a.causal ? offset > 0 : offset >= reach) far_behind += sum;       // (causal: zeros)
                            else mine_near[offset + reach] += sum;
                        }
                    }
                }
                if (border && any_not_finite<T, DP>(ktile, kb)) left_out = true;
                else weigh<T, DP, 1>(reader, ktile, kb, ds, acc);
            }
        }
        if (left_out) {
#pragma unroll 1
            for (int j0 = 0; j0 < end; j0 += 32) {
                if (j0 + 31 <= lowest || j0 > highest || !any_not_finite<T>(keys + (long long)j0 * a.k.row, a.k.row, end - j0, a.D)) continue;
                const char *const mine = rows_of(a.q, b, q_ragged, seq.q0 + h_row, head), *const my_grad = rows_of(a.dout, b, q_ragged, seq.q0 + h_row, head);
#pragma unroll 1
                for (int j = j0; j < min(end, j0 + 32); ++j) {
                    if (j > pos || !there) continue;
                    const char *const key = keys + (long long)j * a.k.row;
                    const float x = dot<T>(mine, key, a.D), dp = dot<T>(my_grad, values + (long long)j * a.v.row, a.D);
                    const float p = __builtin_amdgcn_exp2f(BIAS ? (fmaf(x, a.scale2, table[bias_entry(a, j - pos)]) - top) - log_sum : fmaf(x, a.scale2, -both));
                    add_row<T, DP>(key, a.D, p * (dp - delta), acc[0]);
                }
            }
        }
        if (there) {
            T *const to = reinterpret_cast<T *>(rows_of(a.dq, b, q_ragged, seq.q0 + row, head));
            const int D = opaque(a.D), first = opaque(4 * half);
#pragma unroll
            for (int d = 0; d < 4 * R::BLOCKS; ++d) {
                const int e = first + 8 * d;
                if (e < D)
                    store4<T, DIRECT>(to + e, D - e, acc[0][d >> 2][4 * (d & 3)] * a.scale, acc[0][d >> 2][4 * (d & 3) + 1] * a.scale,
                           acc[0][d >> 2][4 * (d & 3) + 2] * a.scale, acc[0][d >> 2][4 * (d & 3) + 3] * a.scale);
            }
        }
        tile::wait_loads<0>();
        tile::wait_lds();
        __syncthreads();
    }
    if constexpr (BIAS) {
        if (!a.part_bias) return;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            far_before += __shfl_xor(far_before, o);
            far_behind += __shfl_xor(far_behind, o);
        }
        float *const far = table;           // (the bias itself is not needed any more)
        __syncthreads();
        if (lane == 0) {
            far[2 * wave] = far_before;
            far[2 * wave + 1] = far_behind;
        }
        __syncthreads();
        const int buckets = a.bias.buckets, all = a.bias.both ? 2 * buckets : buckets;
        for (int c = tid; c < all; c += THREADS) {
            const int in = c < buckets ? c : c - buckets, sign = c < buckets ? -1 : 1;
            float sum = 0.f;
            if (in == buckets - 1) {
                for (int w = 0; w < 4; ++w) sum += far[2 * w + (sign > 0 ? 1 : 0)];
            } else {
                const int from = in == 0 ? (sign > 0 ? 1 : 0) : a.bias.border[in - 1], to = a.bias.border[in];
                for (int w = 0; w < 4; ++w)
                    for (int r = from; r < to; ++r) sum += near[w * entries + sign * r + reach];
            }
            a.part_bias[(((long long)head * a.batch + b) * a.tiles + first_tile) * all + c] = sum;
        }
    }
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

template <typename T, int DP, bool BIAS, bool DIRECT> __global__ __launch_bounds__(THREADS, 1) void k_attention_dkv(Args a)
{
    using W = Backward<T, DP, BIAS>;
    using R = Row<T, DP>;
    constexpr int ROWS = 128, BLOCKS = W::TILE / 32;
    extern __shared__ __align__(1024) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int total = a.tiles * a.kv_heads * (a.batch + (a.clear && a.k_offsets ? 1 : 0));
    int at = place_of(blockIdx.x, total);
    if (at >= total) return;
    const int first_tile = at % a.tiles;                        // (causal: the first keys have the most queries)
    at /= a.tiles;
    const int kv_head = at % a.kv_heads, b = at / a.kv_heads;
    if (b == a.batch) {
        clear_rows<T>(a.dk, a.k_offsets, a.batch, a.k_rows, kv_head, a.D, first_tile, a.tiles);
        clear_rows<T>(a.dv, a.k_offsets, a.batch, a.k_rows, kv_head, a.D, first_tile, a.tiles);
        return;
    }
    const Sequence seq = sequence(a, b);
    const int shift = seq.k_len - seq.q_len;
    const bool q_ragged = a.q_offsets != nullptr, k_ragged = a.k_offsets != nullptr;
    float *const facts = reinterpret_cast<float *>(lds + W::TILES_BYTES), *const table = facts + W::FACTS_BYTES / 4;
    int table_of = -1;                                          // the query head whose bias is there
    const unsigned lds_addr = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;
    Reader<T, DP> reader;
    reader.init();
    Loader<T, DP, W::TILE, THREADS, DIRECT> load_q, load_g;
    load_q.init(a.q.row, a.D, tid);
    load_g.init(a.dout.row, a.D, tid);
    const int rows = a.clear && !k_ragged ? a.k_rows : seq.k_len;       // rows behind the sequence get zeros
    for (int tile0 = first_tile * ROWS; tile0 < rows; tile0 += a.tiles * ROWS) {
        const int mine0 = tile0 + wave * 32, key = mine0 + (lane & 31);
        const bool there = key < seq.k_len;
        uint4 k[R::STEPS], v[R::STEPS];
        {
            const char *pk = rows_of(a.k, b, k_ragged, seq.k0 + key, kv_head), *pv = rows_of(a.v, b, k_ragged, seq.k0 + key, kv_head);
#pragma unroll
            for (int s = 0; s < R::STEPS; ++s) {
                k[s] = there ? chunk_of<T, DIRECT>(pk, 2 * s + half, a.D) : make_uint4(0, 0, 0, 0);
                v[s] = there ? chunk_of<T, DIRECT>(pv, 2 * s + half, a.D) : make_uint4(0, 0, 0, 0);
            }
        }
        const int q_tiles = (seq.q_len + W::TILE - 1) / W::TILE, q_from = a.causal ? min(max(0, tile0 - shift) / W::TILE, q_tiles) : 0;
        const int per = tile0 < seq.k_len ? q_tiles - q_from : 0, count = per * a.group;
        auto load = [&](int g, int t, int buf) {
            const int head = kv_head * a.group + g, i0 = t * W::TILE;
            const char *pq = rows_of(a.q, b, q_ragged, seq.q0 + i0, head), *pg = rows_of(a.dout, b, q_ragged, seq.q0 + i0, head);
            unsigned char *const to_tile = lds + buf * W::STAGE;
            const unsigned to_addr = lds_addr + buf * W::STAGE;
            load_q.issue(to_tile, to_addr, pq, seq.q_len - i0, a.D, wave);
            load_g.issue(to_tile + W::HALF, to_addr + W::HALF, pg, seq.q_len - i0, a.D, wave);
            // a plane of facts by each wave: delta behind what the exponents are taken from
            if (wave < W::FACTS && lane < W::TILE) {
                const int plane = BIAS ? (wave == 0 ? 2 : wave == 1 ? 1 : 3) : wave;
                const float *from = a.stats + plane * a.plane + (long long)head * a.q_all + seq.q_first + i0;
                const int to = (buf * W::FACTS + wave) * W::TILE;
                if (i0 + lane < seq.q_len) bring4(uniform(from), lane * 4, lds_addr + W::TILES_BYTES + to * 4);
                else facts[to + lane] = wave == 0 ? __builtin_inff() : 0.f;
            }
        };
        f32x16 dk[1][R::BLOCKS], dv[1][R::BLOCKS];
#pragma unroll
        for (int d = 0; d < R::BLOCKS; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) dk[0][d][i] = dv[0][d][i] = 0.f;
        bool left_out = false;
        int g = 0, t = q_from, buf = 0;
        if (count > 0) load(0, q_from, 0);
        for (int c = 0; c < count; ++c, buf ^= 1) {
            const int g_now = g, i_tile = t * W::TILE;
            tile::wait_loads<0>();
            if (seq.q_len - i_tile < W::TILE) {
                load_q.clear(lds + buf * W::STAGE, seq.q_len - i_tile, wave);
                load_g.clear(lds + buf * W::STAGE + W::HALF, seq.q_len - i_tile, wave);
            }
            tile::wait_lds();
            tile::meet();
            if (++t == q_tiles) {
                t = q_from;
                ++g;
            }
            if constexpr (BIAS)
                if (g_now != table_of) {
                    fill_bias(a, kv_head * a.group + g_now, table);
                    table_of = g_now;
                    tile::wait_lds();
                    tile::meet();
                }
            if (c + 1 < count) load(g, t, buf ^ 1);
            const unsigned char *const qtile = lds + buf * W::STAGE, *const gtile = qtile + W::HALF;
            const float *const fact = facts + buf * W::FACTS * W::TILE;
#pragma unroll
            for (int rb = 0; rb < BLOCKS; ++rb) {
                const int i0 = i_tile + 32 * rb, p0 = shift + i0;
                if (i0 >= seq.q_len || mine0 >= seq.k_len || (a.causal && p0 + 31 < mine0)) continue;
                const bool border = a.causal && p0 < mine0 + 31;
                f32x16 s, dp;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = dp[i] = 0.f;
#pragma unroll
                for (int f = 0; f < R::STEPS; ++f) s = scores<T>(reader.along(qtile, rb, f), k[f], s);
#pragma unroll
                for (int f = 0; f < R::STEPS; ++f) dp = scores<T>(reader.along(gtile, rb, f), v[f], dp);
                if constexpr (BIAS) add_bias_down(a, table, key - p0, mine0 - (p0 + 31), mine0 + 31 - p0, a.scale2, s);
                f32x16 p[1], ds[1];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    const int r = 32 * rb + 8 * f + 4 * half;
                    const f32x4 from = *reinterpret_cast<const f32x4 *>(fact + r), delta = *reinterpret_cast<const f32x4 *>(fact + W::TILE + r);
                    f32x4 log_sum = {0.f, 0.f, 0.f, 0.f};
                    if constexpr (BIAS) log_sum = *reinterpret_cast<const f32x4 *>(fact + 2 * W::TILE + r);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 4 * f + e;
                        p[0][i] = __builtin_amdgcn_exp2f(BIAS ? (s[i] - from[e]) - log_sum[e] : fmaf(s[i], a.scale2, -from[e]));
                        ds[0][i] = p[0][i] * (dp[i] - delta[e]);
                    }
                }
                if (border) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const bool in = key <= p0 + row_of(i, half);
                        p[0][i] = in ? p[0][i] : 0.f;
                        ds[0][i] = in ? ds[0][i] : 0.f;
                    }
                }
                if (border && (any_not_finite<T, DP>(gtile, rb) || any_not_finite<T, DP>(qtile, rb))) {
                    left_out = true;
                } else {
                    weigh<T, DP, 1>(reader, gtile, rb, p, dv);
                    weigh<T, DP, 1>(reader, qtile, rb, ds, dk);
                }
            }
        }
        if (left_out) {
            const char *const mine = rows_of(a.k, b, k_ragged, seq.k0 + min(key, seq.k_len - 1), kv_head),
                             *const my_value = rows_of(a.v, b, k_ragged, seq.k0 + min(key, seq.k_len - 1), kv_head);
#pragma unroll 1
            for (int h = kv_head * a.group; h < (kv_head + 1) * a.group; ++h) {
#pragma unroll 1
                for (int i0 = q_from * W::TILE; i0 < seq.q_len && shift + i0 < mine0 + 31; i0 += 32) {
                    const char *const pq = rows_of(a.q, b, q_ragged, seq.q0 + i0, h), *const pg = rows_of(a.dout, b, q_ragged, seq.q0 + i0, h);
                    if (shift + i0 + 31 < mine0 || (!any_not_finite<T>(pg, a.dout.row, seq.q_len - i0, a.D) && !any_not_finite<T>(pq, a.q.row, seq.q_len - i0, a.D)))
                        continue;
#pragma unroll 1
                    for (int i = i0; i < min(seq.q_len, i0 + 32); ++i) {
                        if (key > shift + i || !there) continue;
                        const char *const row_q = pq + (long long)(i - i0) * a.q.row, *const row_g = pg + (long long)(i - i0) * a.dout.row;
                        const float *const fact = a.stats + (long long)h * a.q_all + seq.q_first + i;
                        float x = dot<T>(row_q, mine, a.D) * a.scale2;
                        if constexpr (BIAS) {
                            const int at = bucket_of(a.bias, key - shift - i) * a.heads + h;
                            x += (a.bias.f32 ? ((const float *)a.bias.table)[at] : (float)((const __bf16 *)a.bias.table)[at]) * 1.44269504f;
                        }
                        const float p = __builtin_amdgcn_exp2f((x - fact[2 * a.plane]) - fact[3 * a.plane]);
                        const float ds = p * (dot<T>(row_g, my_value, a.D) - fact[a.plane]);
                        add_row<T, DP>(row_g, a.D, p, dv[0]);
                        add_row<T, DP>(row_q, a.D, ds, dk[0]);
                    }
                }
            }
        }
        if (key < rows) {
            T *const to_k = reinterpret_cast<T *>(rows_of(a.dk, b, k_ragged, seq.k0 + key, kv_head)),
                    *const to_v = reinterpret_cast<T *>(rows_of(a.dv, b, k_ragged, seq.k0 + key, kv_head));
            // (a row behind the sequence: zeros, whatever the weights of its zeros came to)
            auto of = [&](float x) { return there ? x : 0.f; };
            const int D = opaque(a.D), first = opaque(4 * half);
#pragma unroll
            for (int d = 0; d < 4 * R::BLOCKS; ++d) {
                const int e = first + 8 * d, x = d >> 2, y = 4 * (d & 3);
                if (e >= D) continue;
                store4<T, DIRECT>(to_k + e, D - e, of(dk[0][x][y] * a.scale), of(dk[0][x][y + 1] * a.scale), of(dk[0][x][y + 2] * a.scale), of(dk[0][x][y + 3] * a.scale));
                store4<T, DIRECT>(to_v + e, D - e, of(dv[0][x][y]), of(dv[0][x][y + 1]), of(dv[0][x][y + 2]), of(dv[0][x][y + 3]));
            }
        }
        tile::wait_loads<0>();
        tile::wait_lds();
        __syncthreads();
    }
}

} // namespace attn

// Attention's forward call.
#include "attention_host.h"
#include "attention_kernels.hip"

namespace {

attn_rules::Cut forward_cut(const rcd_attention_shape &s)
{
    return attn_rules::cut_of(s.batch, s.heads, s.heads / s.kv_heads, attn_rules::longest_of(s.longest_q, s.q_rows, s.batch, s.q_offsets_dev != nullptr),
                              attn_rules::longest_of(s.longest_k, s.k_rows, s.batch, s.k_offsets_dev != nullptr), s.q_rows, s.dt == RCD_F32, width_of(s), s.k_lengths_dev != nullptr,
                              s.q_offsets_dev != nullptr);
}

SetUp g_set_up;

int set_up()
{
    return g_set_up([](auto t, auto dp, auto bias, auto direct) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool BIAS = decltype(bias)::value, DIRECT = decltype(direct)::value;
        const hipError_t e = raise_lds(&k_attention<T, DP, false, BIAS, DIRECT>);
        return e != hipSuccess ? e : raise_lds(&k_attention<T, DP, true, BIAS, DIRECT>);
    });
}

size_t forward_bytes(const rcd_attention_shape &s, const attn_rules::Cut &c, void *base, Args *a)
{
    if (c.splits == 1) return 0;
    Pieces room(base);
    const size_t slots = (size_t)all_rows(s.q_offsets_dev, s.q_rows, s.batch) * s.heads * c.splits;
    float *const o = room.take(slots * s.d), *const ml = room.take(slots * 2);
    if (a) {
        a->part_o = o;
        a->part_ml = ml;
    }
    return room.used;
}

} // namespace

int rcd_set_up_attention() { return set_up(); }

extern "C" {

size_t rcd_attention_workspace_bytes(const rcd_attention_shape *s)
{
    if (check_shape(s) != RCD_OK || s->batch == 0 || s->q_rows == 0) return 0;
    return forward_bytes(*s, forward_cut(*s), nullptr, nullptr);
}

int rcd_attention(const rcd_attention_shape *s, const rcd_heads *q, const rcd_heads *k, const rcd_heads *v, const rcd_heads *out, float *saved_dev,
                  int clear, void *workspace_dev, size_t workspace_bytes, void *stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    ENC_TRY(check_shape(s));
    ENC_TRY(check_heads(q, s->q_rows, s->batch, s->dt));
    ENC_TRY(check_heads(k, s->k_rows, s->batch, s->dt));
    ENC_TRY(check_heads(v, s->k_rows, s->batch, s->dt));
    ENC_TRY(check_result(out, s->q_rows, s->batch, s->dt, clear != 0, s->q_offsets_dev));
    if (!works_on(s->q_rows, s->batch, clear != 0, s->q_offsets_dev)) return RCD_OK;
    const attn_rules::Cut c = forward_cut(*s);
    Args a = args_of(*s);
    ENC_TRY(check_workspace(workspace_dev, workspace_bytes, forward_bytes(*s, c, workspace_dev, &a)));
    ENC_TRY(set_up());
    a.q = heads_of(q, s->dt);
    a.k = heads_of(k, s->dt);
    a.v = heads_of(v, s->dt);
    a.o = heads_of(out, s->dt);
    a.saved = saved_dev;
    a.clear = clear && s->q_offsets_dev;
    a.pack = c.pack;
    a.tiles = (int)c.tiles;
    a.splits = (int)c.splits;
    a.least = (int)c.least;
    const int bias_bytes = width_of(*s) * c.pack * 4;
    const int64_t rows = c.shared ? 32 : 128;
    Grid grid{s->batch + (a.clear ? 1 : 0), c.tiles * (a.group / c.pack) * c.splits, 0, s->heads / c.pack, 0};
    if (s->q_offsets_dev && c.splits == 1) {
        grid.packed_tiles = s->q_rows * c.pack / rows + s->batch;
    } else if (c.shared && c.splits > 1 && !s->q_offsets_dev && s->k_lengths_dev) {
        grid.packed_tiles = s->batch * c.splits;
        grid.heads *= c.tiles;
        grid.of_keys = true;
    }
    const bool direct = aligned(a.k, s->d, s->dt) && aligned(a.v, s->d, s->dt);
    ENC_TRY(with_variant(s->dt, s->d, s->bias_dev != nullptr, direct, [&](auto t, auto dp, auto bias, auto way) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool BIAS = decltype(bias)::value, DIRECT = decltype(way)::value;
        using S = Forward<T, DP, true>;
        using F = Forward<T, DP, false>;
        if (!c.shared) return launch(&k_attention<T, DP, false, BIAS, DIRECT>, grid, F::GROUP, F::TILES_BYTES + bias_bytes, a, stream);
        grid.most = 256;            // (a compute unit has room for one)
        return launch(&k_attention<T, DP, true, BIAS, DIRECT>, grid, S::GROUP, S::TILES_BYTES + S::STATS_BYTES + bias_bytes, a, stream);
    }));
    if (c.splits > 1) {
        const int64_t slots = a.q_all * s->heads;
        const bool many = attn_rules::many_joins(slots, c.splits);
        const dim3 joins((unsigned)(many ? attn_rules::ceil_div(slots, JOIN_THREADS / 64) : slots));
        if (s->dt == RCD_F32) {
            if (many) hipLaunchKernelGGL((k_attention_join_many<float>), joins, dim3(JOIN_THREADS), 0, stream, a);
            else hipLaunchKernelGGL((k_attention_join<float>), joins, dim3(JOIN_THREADS), 0, stream, a);
        } else {
            if (many) hipLaunchKernelGGL((k_attention_join_many<__bf16>), joins, dim3(JOIN_THREADS), 0, stream, a);
            else hipLaunchKernelGGL((k_attention_join<__bf16>), joins, dim3(JOIN_THREADS), 0, stream, a);
        }
        ENC_HIP_TRY(hipGetLastError());
    }
    return RCD_OK;
}

} // extern "C"

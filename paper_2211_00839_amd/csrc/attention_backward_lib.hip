// Attention's backward call.
#include "attention_host.h"
#include "attention_backward_kernels.hip"

namespace {

SetUp g_set_up;

int set_up()
{
    return g_set_up([](auto t, auto dp, auto bias, auto direct) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool BIAS = decltype(bias)::value, DIRECT = decltype(direct)::value;
        hipError_t e = raise_lds(&k_attention_dq<T, DP, false, BIAS, DIRECT>);
        if (e == hipSuccess) e = raise_lds(&k_attention_dq<T, DP, true, BIAS, DIRECT>);
        if (e == hipSuccess) e = raise_lds(&k_attention_dkv<T, DP, false, BIAS, DIRECT>);
        return e != hipSuccess ? e : raise_lds(&k_attention_dkv<T, DP, true, BIAS, DIRECT>);
    });
}

template <typename W> int dq_lds(bool bias, int reach, bool causal)
{
    return W::TILES_BYTES + (bias ? (bias_width(reach, causal) + 4 * bias_entries(reach, causal)) * 4 + 4 * W::TURN_BYTES : 0);
}
template <typename W> int dkv_lds(bool bias, int reach, bool causal) { return W::KV_TILES_BYTES + W::V_BYTES + W::FACTS_BYTES + (bias ? bias_width(reach, causal) * 4 : 0); }

// The gradient of q: whether the waves share their rows (where there is room for it), the workgroups for each sequence and head, and where sequences
// lie end to end the most tiles that all of them have.
struct Way {
    bool shared;
    int64_t tiles, packed_tiles;
    int64_t parts(int64_t batch) const { return std::max(packed_tiles, batch * tiles); }      // (of the bias's gradient, for each head)
};
Way dq_way(const rcd_attention_shape &s)
{
    const int64_t longest = attn_rules::longest_of(s.longest_q, s.q_rows, s.batch, s.q_offsets_dev != nullptr);
    Way w;
    w.shared = attn_rules::shared_rows(s.batch * s.heads, longest, attn_rules::FEW_WORKGROUPS);
    if (w.shared)
        w.shared = with_variant(s.dt, s.d, s.bias_dev != nullptr, true, [&](auto t, auto dp, auto bias, auto) {
                       using W = Backward<decltype(t), decltype(dp)::value, true, decltype(bias)::value>;
                       return dq_lds<W>(s.bias_dev != nullptr, reach_of(s), s.causal != 0);
                   }) <= MOST_LDS;
    w.tiles = attn_rules::tiles_of(attn_rules::units_of(s.batch, s.kv_heads) * (s.heads / s.kv_heads), longest, w.shared);
    w.packed_tiles = s.q_offsets_dev ? s.q_rows / (w.shared ? 32 : 128) + s.batch : 0;
    return w;
}

// The gradients of k and v: and into how many parts the queries are cut.
struct KvWay {
    bool shared;
    int64_t tiles, parts;
};
KvWay dkv_way(const rcd_attention_shape &s)
{
    const int64_t longest = attn_rules::longest_of(s.longest_k, s.k_rows, s.batch, s.k_offsets_dev != nullptr);
    const int64_t longest_q = attn_rules::longest_of(s.longest_q, s.q_rows, s.batch, s.q_offsets_dev != nullptr);
    KvWay w;
    w.shared = attn_rules::shared_rows(s.batch * s.kv_heads, longest, attn_rules::FEW_WORKGROUPS);
    w.tiles = attn_rules::tiles_of(attn_rules::units_of(s.batch, s.kv_heads), longest, w.shared);
    const bool uneven = s.causal || s.q_offsets_dev || s.k_offsets_dev || s.k_lengths_dev;
    w.parts = attn_rules::parts_of(w.tiles * s.kv_heads * s.batch, uneven, longest_q, s.heads / s.kv_heads);
    return w;
}

size_t backward_bytes(const rcd_attention_shape &s, void *base, Args *a)
{
    Pieces room(base);
    const size_t plane = up256((size_t)all_rows(s.q_offsets_dev, s.q_rows, s.batch) * s.heads * 4) / 4;
    float *const stats = room.take(4 * plane);
    float *const parts = s.bias_dev ? room.take((size_t)s.heads * dq_way(s).parts(s.batch) * s.buckets) : nullptr;
    const int64_t splits = dkv_way(s).parts;
    const size_t sums = splits > 1 ? (size_t)splits * all_rows(s.k_offsets_dev, s.k_rows, s.batch) * s.kv_heads * s.d : 0;
    float *const part_k = splits > 1 ? room.take(sums) : nullptr, *const part_v = splits > 1 ? room.take(sums) : nullptr;
    if (a) {
        a->part_k = part_k;
        a->part_v = part_v;
        a->stats = stats;
        a->plane = (long long)plane;
        a->part_bias = parts;
    }
    return room.used;
}

} // namespace

int rcd_set_up_attention_backward() { return set_up(); }

extern "C" {

size_t rcd_attention_backward_workspace_bytes(const rcd_attention_shape *s)
{
    if (check_shape(s) != RCD_OK) return 0;
    return backward_bytes(*s, nullptr, nullptr);
}

int rcd_attention_backward(const rcd_attention_shape *s, const rcd_heads *dout, const rcd_heads *q, const rcd_heads *k, const rcd_heads *v,
                           const rcd_heads *out, const float *saved_dev, const rcd_heads *dq, const rcd_heads *dk, const rcd_heads *dv, void *dbias_dev,
                           int clear, void *workspace_dev, size_t workspace_bytes, void *stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    ENC_TRY(check_shape(s));
    for (const rcd_heads *h : {dout, q, out}) ENC_TRY(check_heads(h, s->q_rows, s->batch, s->dt));
    for (const rcd_heads *h : {k, v}) ENC_TRY(check_heads(h, s->k_rows, s->batch, s->dt));
    ENC_TRY(check_result(dq, s->q_rows, s->batch, s->dt, clear != 0, s->q_offsets_dev));
    for (const rcd_heads *h : {dk, dv}) ENC_TRY(check_result(h, s->k_rows, s->batch, s->dt, clear != 0, s->k_offsets_dev));
    if (!saved_dev && s->q_rows > 0 && s->batch > 0) return RCD_ERR_INVALID_ARG;
    if (dbias_dev && !s->bias_dev) return RCD_ERR_INVALID_ARG;
    Args a = args_of(*s);
    ENC_TRY(check_workspace(workspace_dev, workspace_bytes, backward_bytes(*s, workspace_dev, &a)));
    ENC_TRY(set_up());
    a.q = heads_of(q, s->dt);
    a.k = heads_of(k, s->dt);
    a.v = heads_of(v, s->dt);
    a.o = heads_of(out, s->dt);
    a.dout = heads_of(dout, s->dt);
    a.dq = heads_of(dq, s->dt);
    a.dk = heads_of(dk, s->dt);
    a.dv = heads_of(dv, s->dt);
    a.saved = const_cast<float *>(saved_dev);
    a.clear = clear != 0;
    const int reach = reach_of(*s);
    const bool causal = s->causal != 0;
    const Way way = dq_way(*s);
    bool packed = false;            // the gradient of q's workgroups were counted over all sequences' tiles
    if (works_on(s->q_rows, s->batch, a.clear, s->q_offsets_dev)) {
        Args x = a;
        x.tiles = (int)way.tiles;
        if (!dbias_dev) x.part_bias = nullptr;
        Grid grid{s->batch + (a.clear && a.q_offsets ? 1 : 0), way.tiles * a.group, way.packed_tiles, s->heads, 0};
        const bool direct = aligned(a.k, s->d, s->dt) && aligned(a.v, s->d, s->dt);
        ENC_TRY(with_variant(s->dt, s->d, s->bias_dev != nullptr, direct, [&](auto t, auto dp, auto bias, auto how) {
            using T = decltype(t);
            constexpr int DP = decltype(dp)::value;
            constexpr bool BIAS = decltype(bias)::value, DIRECT = decltype(how)::value;
            if (!way.shared) return launch(&k_attention_dq<T, DP, false, BIAS, DIRECT>, grid, THREADS, dq_lds<Backward<T, DP, false, BIAS>>(BIAS, reach, causal), x, stream);
            grid.most = 512;
            return launch(&k_attention_dq<T, DP, true, BIAS, DIRECT>, grid, THREADS, dq_lds<Backward<T, DP, true, BIAS>>(BIAS, reach, causal), x, stream);
        }));
        packed = x.packed;
    }
    if (dbias_dev) {
        const long long count = s->q_rows > 0 ? packed ? way.packed_tiles : s->batch * way.tiles : 0;
        const dim3 grid((unsigned)(s->buckets * s->heads));
        if (s->bias_dt == RCD_F32)
            hipLaunchKernelGGL((k_bias_gradient<float>), grid, dim3(THREADS), 0, stream, a.part_bias, count, (int)s->buckets, (int)s->heads, (float *)dbias_dev);
        else
            hipLaunchKernelGGL((k_bias_gradient<__bf16>), grid, dim3(THREADS), 0, stream, a.part_bias, count, (int)s->buckets, (int)s->heads, (__bf16 *)dbias_dev);
        ENC_HIP_TRY(hipGetLastError());
    }
    if (works_on(s->k_rows, s->batch, a.clear, s->k_offsets_dev)) {
        const KvWay kv = dkv_way(*s);
        a.tiles = (int)kv.tiles;
        a.splits = (int)kv.parts;
        Grid grid{s->batch + (a.clear && a.k_offsets ? 1 : 0), kv.tiles * kv.parts, 0, s->kv_heads * kv.parts, 0};
        if (s->k_offsets_dev) grid.packed_tiles = s->k_rows / (kv.shared ? 32 : 128) + s->batch;
        const bool direct = aligned(a.q, s->d, s->dt) && aligned(a.dout, s->d, s->dt);
        ENC_TRY(with_variant(s->dt, s->d, s->bias_dev != nullptr, direct, [&](auto t, auto dp, auto bias, auto how) {
            using T = decltype(t);
            constexpr int DP = decltype(dp)::value;
            constexpr bool BIAS = decltype(bias)::value, DIRECT = decltype(how)::value;
            if (!kv.shared) return launch(&k_attention_dkv<T, DP, false, BIAS, DIRECT>, grid, THREADS, dkv_lds<Backward<T, DP, false, BIAS>>(BIAS, reach, causal), a, stream);
            grid.most = 512;
            return launch(&k_attention_dkv<T, DP, true, BIAS, DIRECT>, grid, THREADS, dkv_lds<Backward<T, DP, true, BIAS>>(BIAS, reach, causal), a, stream);
        }));
        if (kv.parts > 1) {
            const int64_t fours = a.k_all * s->kv_heads * attn_rules::ceil_div(s->d, 4);
            const dim3 grid((unsigned)std::min<int64_t>(attn_rules::ceil_div(fours, THREADS), 8192));
            if (s->dt == RCD_F32) hipLaunchKernelGGL((k_attention_dkv_join<float>), grid, dim3(THREADS), 0, stream, a);
            else hipLaunchKernelGGL((k_attention_dkv_join<__bf16>), grid, dim3(THREADS), 0, stream, a);
            ENC_HIP_TRY(hipGetLastError());
        }
    }
    return RCD_OK;
}

} // extern "C"

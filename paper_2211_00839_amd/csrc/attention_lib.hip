// Host side of attention: argument checks, workspace layout, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <mutex>
#include <type_traits>

#include "host_error.h"
#include "attention_rules.h"
#include "attention_kernels.hip"
#include "attention_backward_kernels.hip"

namespace {

using namespace attn;

constexpr int64_t MOST_ROWS = (int64_t)1 << 29;           // (a row's number and a launch's stride over rows add up in 32 bits)
constexpr int64_t MOST_HEADS = (int64_t)1 << 15;
constexpr int64_t MOST_PITCH = (int64_t)1 << 24;       // bytes from row to row: 64 rows stay within 32-bit offsets
constexpr int64_t MOST_D = 128;
constexpr int MOST_LDS = 160 * 1024;

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int64_t size_of(int dt) { return dt == RCD_F32 ? 4 : 2; }

struct Pieces {
    char *base;
    size_t used = 0;
    explicit Pieces(void *p) : base((char *)p) {}
    float *take(size_t count)
    {
        float *p = base ? reinterpret_cast<float *>(base + used) : nullptr;
        used += up256(count * sizeof(float));
        return p;
    }
};

int check_workspace(const void *ws, size_t bytes, size_t need)
{
    if (need == 0) return RCD_OK;
    return !ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || bytes < need ? RCD_ERR_WORKSPACE : RCD_OK;
}

inline int64_t all_rows(const int32_t *offsets, int64_t rows, int64_t batch) { return offsets ? rows : rows * batch; }

int check_shape(const rcd_attention_shape *s)
{
    if (!s) return RCD_ERR_INVALID_ARG;
    if (s->dt != RCD_F32 && s->dt != RCD_BF16) return RCD_ERR_UNSUPPORTED;
    if (s->batch < 0 || s->heads < 1 || s->kv_heads < 1 || s->heads % s->kv_heads != 0 || s->d < 1 || s->q_rows < 0 || s->k_rows < 0 ||
        s->longest_q < 0 || s->longest_k < 0)
        return RCD_ERR_INVALID_ARG;
    if (s->k_offsets_dev && s->k_lengths_dev) return RCD_ERR_INVALID_ARG;
    const float scale2 = s->scale * 1.44269504f;
    if (!(s->scale > 0.f) || !std::isnormal(s->scale) || !std::isnormal(scale2)) return RCD_ERR_INVALID_ARG;
    if (s->d > MOST_D || s->heads > MOST_HEADS || s->q_rows > MOST_ROWS || s->k_rows > MOST_ROWS || s->batch > MOST_ROWS ||
        s->batch * s->heads > attn_rules::MOST_WORKGROUPS - s->heads)
        return RCD_ERR_UNSUPPORTED;
    if (s->bias_dev) {
        if (s->bias_dt != RCD_F32 && s->bias_dt != RCD_BF16) return RCD_ERR_UNSUPPORTED;
        if (!s->borders_host) return RCD_ERR_INVALID_ARG;
        const int64_t each = s->causal ? s->buckets : s->buckets / 2;
        if (each < 2 || (!s->causal && s->buckets % 2 != 0)) return RCD_ERR_INVALID_ARG;
        if (each > MAX_BUCKETS) return RCD_ERR_UNSUPPORTED;
        for (int64_t i = 0; i + 1 < each; ++i)
            if (s->borders_host[i] < (i ? s->borders_host[i - 1] : 1)) return RCD_ERR_INVALID_ARG;
        if (s->borders_host[each - 2] > MAX_REACH) return RCD_ERR_UNSUPPORTED;
    }
    return RCD_OK;
}

int64_t entries_of(const rcd_attention_shape &s)
{
    if (!s.bias_dev) return 0;
    const int64_t reach = s.borders_host[(s.causal ? s.buckets : s.buckets / 2) - 2];
    return s.causal ? reach + 1 : 2 * reach + 1;
}

int check_heads(const rcd_heads *h, int64_t rows, int64_t batch, int dt)
{
    if (!h) return RCD_ERR_INVALID_ARG;
    if (h->batch < 0 || h->row < 0 || h->head < 0) return RCD_ERR_INVALID_ARG;
    if (rows > 0 && batch > 0 && !h->p) return RCD_ERR_INVALID_ARG;
    if (h->row * size_of(dt) >= MOST_PITCH) return RCD_ERR_UNSUPPORTED;
    return RCD_OK;
}

Heads heads_of(const rcd_heads *h, int dt)
{
    const long long e = size_of(dt);
    return {(char *)h->p, h->batch * e, h->row * e, h->head * e};
}
// Rows that may be read 16 bytes at a time, to LDS without passing the registers.
bool aligned(const Heads &h, int64_t d, int dt)
{
    return (reinterpret_cast<uintptr_t>(h.p) & 15) == 0 && ((h.batch | h.row | h.head) & 15) == 0 && (d * size_of(dt)) % 16 == 0;
}

Args args_of(const rcd_attention_shape &s)
{
    Args a{};
    a.q_offsets = s.q_offsets_dev;
    a.k_offsets = s.k_offsets_dev;
    a.k_lengths = s.k_lengths_dev;
    a.batch = (int)s.batch;
    a.heads = (int)s.heads;
    a.kv_heads = (int)s.kv_heads;
    a.group = (int)(s.heads / s.kv_heads);
    a.q_rows = (int)s.q_rows;
    a.k_rows = (int)s.k_rows;
    a.q_all = all_rows(s.q_offsets_dev, s.q_rows, s.batch);
    a.D = (int)s.d;
    a.pack = a.splits = 1;
    a.causal = s.causal != 0;
    a.scale = s.scale;
    a.scale2 = s.scale * 1.44269504f;
    if (s.bias_dev) {
        a.bias.table = s.bias_dev;
        a.bias.f32 = s.bias_dt == RCD_F32;
        a.bias.both = !s.causal;
        a.bias.buckets = (int)(s.causal ? s.buckets : s.buckets / 2);
        for (int i = 0; i + 1 < a.bias.buckets; ++i) a.bias.border[i] = (unsigned short)s.borders_host[i];
        a.bias.reach = a.bias.border[a.bias.buckets - 2];
    }
    return a;
}

attn_rules::Cut forward_cut(const rcd_attention_shape &s)
{
    return attn_rules::cut_of(s.batch, s.heads, s.heads / s.kv_heads, attn_rules::longest_of(s.longest_q, s.q_rows, s.batch, s.q_offsets_dev != nullptr),
                              attn_rules::longest_of(s.longest_k, s.k_rows, s.batch, s.k_offsets_dev != nullptr), s.q_rows, s.dt == RCD_F32, entries_of(s));
}

// Calls go(type, DP, bias or not) with the variant.
template <typename Go> int with_variant(int dt, int64_t d, bool bias, Go go)
{
    using std::integral_constant;
    auto by_bias = [&](auto t, auto dp) { return bias ? go(t, dp, std::true_type{}) : go(t, dp, std::false_type{}); };
    auto by_d = [&](auto t) { return d <= 64 ? by_bias(t, integral_constant<int, 64>{}) : by_bias(t, integral_constant<int, 128>{}); };
    return dt == RCD_F32 ? by_d(float{}) : by_d(__bf16{});
}

// What is set up once per device and variant: the kernels use more LDS than a kernel may by default.
constexpr int MAX_DEVICES = 64;
std::mutex g_mutex;
bool g_ready[MAX_DEVICES] = {};

template <typename K> hipError_t raise_lds(K kernel)
{
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, MOST_LDS);
}

int set_up()
{
    int dev = 0;
    ENC_HIP_TRY(hipGetDevice(&dev));
    if (dev < 0 || dev >= MAX_DEVICES) return RCD_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_mutex);
    if (g_ready[dev]) return RCD_OK;
    for (int v = 0; v < 8; ++v) {
        const hipError_t e = (hipError_t)with_variant(v & 1 ? RCD_F32 : RCD_BF16, v & 2 ? 128 : 64, (v & 4) != 0, [&](auto t, auto dp, auto bias) {
            using T = decltype(t);
            constexpr int DP = decltype(dp)::value;
            constexpr bool BIAS = decltype(bias)::value;
            hipError_t e = raise_lds(&k_attention<T, DP, 1, false, BIAS>);
            if (e == hipSuccess) e = raise_lds(&k_attention<T, DP, 1, true, BIAS>);
            if (e == hipSuccess) e = raise_lds(&k_attention_dq<T, DP, BIAS>);
            if (e == hipSuccess) e = raise_lds(&k_attention_dkv<T, DP, BIAS>);
            return (int)e;
        });
        ENC_HIP_TRY(e);
    }
    g_ready[dev] = true;
    return RCD_OK;
}

template <typename K> int launch(K kernel, int64_t groups, int lds, const Args &a, hipStream_t stream)
{
    if (lds > MOST_LDS) return RCD_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(attn_rules::ceil_div(groups, 8) * 8)), dim3(THREADS), lds, stream, a);
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
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

// Workgroups of 128 rows for each sequence and head of the gradients' kernels.
int64_t tiles_of(int64_t longest, int64_t across)
{
    const int64_t tiles = std::max<int64_t>(1, attn_rules::ceil_div(longest, 128));
    return std::max<int64_t>(1, std::min(tiles, attn_rules::MOST_WORKGROUPS / std::max<int64_t>(across, 1)));
}
int64_t dq_tiles(const rcd_attention_shape &s)
{
    return tiles_of(attn_rules::longest_of(s.longest_q, s.q_rows, s.batch, s.q_offsets_dev != nullptr), (s.batch + 1) * s.heads);
}

size_t backward_bytes(const rcd_attention_shape &s, void *base, Args *a)
{
    Pieces room(base);
    const size_t plane = up256((size_t)all_rows(s.q_offsets_dev, s.q_rows, s.batch) * s.heads * 4) / 4;
    float *const stats = room.take(4 * plane);
    float *const parts = s.bias_dev ? room.take((size_t)s.heads * s.batch * dq_tiles(s) * s.buckets) : nullptr;
    if (a) {
        a->stats = stats;
        a->plane = (long long)plane;
        a->part_bias = parts;
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
    ENC_TRY(check_heads(out, s->q_rows, s->batch, s->dt));
    if (s->q_rows == 0 || s->batch == 0) return RCD_OK;
    const attn_rules::Cut c = forward_cut(*s);
    Args a = args_of(*s);
    ENC_TRY(check_workspace(workspace_dev, workspace_bytes, forward_bytes(*s, c, workspace_dev, &a)));
    ENC_TRY(set_up());
    a.q = heads_of(q, s->dt);
    a.k = heads_of(k, s->dt);
    a.v = heads_of(v, s->dt);
    a.o = heads_of(out, s->dt);
    a.saved = saved_dev;
    a.direct = aligned(a.k, s->d, s->dt) && aligned(a.v, s->d, s->dt);
    a.clear = clear && s->q_offsets_dev;
    a.pack = c.pack;
    a.tiles = (int)c.tiles;
    a.splits = (int)c.splits;
    const int64_t groups = c.tiles * (s->heads / c.pack) * (s->batch + (a.clear ? 1 : 0)) * c.splits;
    const int bias_bytes = (int)entries_of(*s) * c.pack * 4;
    ENC_TRY(with_variant(s->dt, s->d, s->bias_dev != nullptr, [&](auto t, auto dp, auto bias) {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool BIAS = decltype(bias)::value;
        if (c.keys) return launch(&k_attention<T, DP, 1, true, BIAS>, groups, Forward<T, DP, true>::TILES_BYTES + bias_bytes, a, stream);
        return launch(&k_attention<T, DP, 1, false, BIAS>, groups, Forward<T, DP, false>::TILES_BYTES + bias_bytes, a, stream);
    }));
    if (c.splits > 1) {
        const int64_t slots = a.q_all * s->heads;
        const dim3 grid((unsigned)attn_rules::ceil_div(slots, 4));
        if (s->dt == RCD_F32) hipLaunchKernelGGL((k_attention_join<float>), grid, dim3(THREADS), 0, stream, a);
        else hipLaunchKernelGGL((k_attention_join<__bf16>), grid, dim3(THREADS), 0, stream, a);
        ENC_HIP_TRY(hipGetLastError());
    }
    return RCD_OK;
}

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
    for (const rcd_heads *h : {dout, q, out, dq}) ENC_TRY(check_heads(h, s->q_rows, s->batch, s->dt));
    for (const rcd_heads *h : {k, v, dk, dv}) ENC_TRY(check_heads(h, s->k_rows, s->batch, s->dt));
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
    const int entries = (int)entries_of(*s);
    const int64_t parts = s->batch * dq_tiles(*s);
    return with_variant(s->dt, s->d, s->bias_dev != nullptr, [&](auto t, auto dp, auto bias) -> int {
        using T = decltype(t);
        constexpr int DP = decltype(dp)::value;
        constexpr bool BIAS = decltype(bias)::value;
        using W = Backward<T, DP, BIAS>;
        if (s->q_rows > 0 && s->batch > 0) {
            Args x = a;
            x.direct = aligned(a.k, s->d, s->dt) && aligned(a.v, s->d, s->dt);
            x.tiles = (int)dq_tiles(*s);
            if (!dbias_dev) x.part_bias = nullptr;
            const int64_t groups = x.tiles * s->heads * (s->batch + (a.clear && a.q_offsets ? 1 : 0));
            ENC_TRY(launch(&k_attention_dq<T, DP, BIAS>, groups, W::TILES_BYTES + (BIAS ? 5 * entries * 4 + 4 * W::TURN_BYTES : 0), x, stream));
        }
        if (dbias_dev) {
            const int64_t count = s->q_rows > 0 ? parts : 0;
            const dim3 grid((unsigned)(s->buckets * s->heads));
            if (s->bias_dt == RCD_F32)
                hipLaunchKernelGGL((k_bias_gradient<float>), grid, dim3(THREADS), 0, stream, a.part_bias, (long long)count, (int)s->buckets, (int)s->heads, (float *)dbias_dev);
            else
                hipLaunchKernelGGL((k_bias_gradient<__bf16>), grid, dim3(THREADS), 0, stream, a.part_bias, (long long)count, (int)s->buckets, (int)s->heads, (__bf16 *)dbias_dev);
            ENC_HIP_TRY(hipGetLastError());
        }
        if (s->k_rows > 0 && s->batch > 0) {
            Args x = a;
            x.direct = aligned(a.q, s->d, s->dt) && aligned(a.dout, s->d, s->dt);
            x.tiles = (int)tiles_of(attn_rules::longest_of(s->longest_k, s->k_rows, s->batch, s->k_offsets_dev != nullptr), (s->batch + 1) * s->kv_heads);
            const int64_t groups = x.tiles * s->kv_heads * (s->batch + (a.clear && a.k_offsets ? 1 : 0));
            ENC_TRY(launch(&k_attention_dkv<T, DP, BIAS>, groups, W::TILES_BYTES + W::FACTS_BYTES + (BIAS ? entries * 4 : 0), x, stream));
        }
        return RCD_OK;
    });
}

} // extern "C"

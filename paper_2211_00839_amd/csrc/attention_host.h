// Host side that attention and its gradients share: argument checks, workspace layout, the choice of a variant.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <mutex>
#include <type_traits>

#include "attention_common.h"
#include "attention_rules.h"
#include "host_error.h"

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
        attn_rules::units_of(s->batch, s->kv_heads) * (s->heads / s->kv_heads) > attn_rules::MOST_WORKGROUPS)
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

int reach_of(const rcd_attention_shape &s) { return s.bias_dev ? s.borders_host[(s.causal ? s.buckets : s.buckets / 2) - 2] : 0; }
int width_of(const rcd_attention_shape &s) { return s.bias_dev ? bias_width(reach_of(s), s.causal != 0) : 0; }

int check_heads(const rcd_heads *h, int64_t rows, int64_t batch, int dt)
{
    if (!h) return RCD_ERR_INVALID_ARG;
    if (h->batch < 0 || h->row < 0 || h->head < 0) return RCD_ERR_INVALID_ARG;
    if (rows > 0 && batch > 0 && !h->p) return RCD_ERR_INVALID_ARG;
    if (h->row * size_of(dt) >= MOST_PITCH) return RCD_ERR_UNSUPPORTED;
    return RCD_OK;
}

// Results of a call without sequences: there is a kernel all the same where rows that belong to none are to become zeros.
bool works_on(int64_t rows, int64_t batch, bool clear, const int32_t *offsets) { return rows > 0 && (batch > 0 || (clear && offsets)); }
int check_result(const rcd_heads *h, int64_t rows, int64_t batch, int dt, bool clear, const int32_t *offsets)
{
    ENC_TRY(check_heads(h, rows, batch, dt));
    return works_on(rows, batch, clear, offsets) && !h->p ? RCD_ERR_INVALID_ARG : RCD_OK;
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
    a.k_all = all_rows(s.k_offsets_dev, s.k_rows, s.batch);
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

// Calls go(type, DP, bias or not, direct or not) with the variant.
template <typename Go> int with_variant(int dt, int64_t d, bool bias, bool direct, Go go)
{
    using std::integral_constant;
    auto by_way = [&](auto t, auto dp, auto b) { return direct ? go(t, dp, b, std::true_type{}) : go(t, dp, b, std::false_type{}); };
    auto by_bias = [&](auto t, auto dp) { return bias ? by_way(t, dp, std::true_type{}) : by_way(t, dp, std::false_type{}); };
    auto by_d = [&](auto t) { return d <= 64 ? by_bias(t, integral_constant<int, 64>{}) : by_bias(t, integral_constant<int, 128>{}); };
    return dt == RCD_F32 ? by_d(float{}) : by_d(__bf16{});
}

// What is set up once per device and kind of kernel: they use more LDS than a kernel may by default.  raise(type, DP, bias or not, direct or not)
// asks for it.
constexpr int MAX_DEVICES = 64;

template <typename K> hipError_t raise_lds(K kernel)
{
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, MOST_LDS);
}

struct SetUp {
    std::mutex mutex;
    bool ready[MAX_DEVICES] = {};
    template <typename Raise> int operator()(Raise raise)
    {
        int dev = 0;
        ENC_HIP_TRY(hipGetDevice(&dev));
        if (dev < 0 || dev >= MAX_DEVICES) return RCD_ERR_UNSUPPORTED;
        std::lock_guard<std::mutex> lock(mutex);
        if (ready[dev]) return RCD_OK;
        for (int v = 0; v < 16; ++v) {
            const hipError_t e = (hipError_t)with_variant(v & 1 ? RCD_F32 : RCD_BF16, v & 2 ? 128 : 64, (v & 4) != 0, (v & 8) != 0,
                                                          [&](auto... which) { return (int)raise(which...); });
            ENC_HIP_TRY(e);
        }
        ready[dev] = true;
        return RCD_OK;
    }
};

// How a kernel's workgroups are counted.  each: those of a sequence and head of k and v.  packed_tiles: where sequences lie end to end by offsets, the
// most tiles that all of them together have (0: not so), and heads: workgroups of one such tile.  most: how many are launched, where each goes on
// to others; 0: all of them.
struct Grid {
    int64_t sequences, each, packed_tiles, heads, most;
    bool of_keys = false;       // those are parts of keys
};
template <typename K> int launch(K kernel, const Grid &g, int threads, int lds, Args &a, hipStream_t stream)
{
    if (lds > MOST_LDS) return RCD_ERR_UNSUPPORTED;
    // (one slot more than there are tiles: its workgroups clear rows that belong to no sequence)
    const int64_t packed = g.packed_tiles > 0 ? (g.packed_tiles + 1) * g.heads : 0;
    a.packed = packed > 0 && packed <= attn_rules::MOST_WORKGROUPS ? g.of_keys ? 2 : 1 : 0;
    a.slots = a.packed ? (int)g.packed_tiles : 0;
    const int64_t all = a.packed ? packed : workgroups_of(g.sequences, a.kv_heads, g.each);
    if (all > attn_rules::MOST_WORKGROUPS + 8) return RCD_ERR_UNSUPPORTED;
    const int64_t launched = g.most > 0 ? std::min(all, g.most) : all;
    a.workgroups = (int)all;
    a.by_heads = Divisor(std::max<int64_t>(g.heads, 1));
    a.by_round = Divisor(launched < all ? std::max<int64_t>(1, launched / 8 / g.each) : (int64_t)1 << 30);
    a.by_each = Divisor(g.each);
    a.by_tiles = Divisor(a.tiles);
    a.by_packs = Divisor(a.group / a.pack);
    a.by_pack = Divisor(a.pack);
    a.by_kv_heads = Divisor(a.kv_heads);
    a.by_splits = Divisor(a.splits);
    a.by_group = Divisor(a.group);
    hipLaunchKernelGGL(kernel, dim3((unsigned)launched), dim3(threads), lds, stream, a);
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

} // namespace

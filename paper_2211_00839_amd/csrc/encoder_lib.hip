// Host side of the feature encoder's operators: argument checks, workspace layout, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <mutex>
#include <type_traits>

#include "host_error.h"
#include "encoder_rules.h"
#include "norm_kernels.hip"
#include "product_kernels.hip"
#include "direct_kernels.hip"
#include "few_rows_kernels.hip"

namespace {

using namespace enc;

constexpr int64_t MAX_EXTENT = 0x7fffff00;          // rows
constexpr int64_t MAX_NORM_LENGTH = (int64_t)1 << 30;
// Lengths of a product: 255 rows of two packed ones side by side (a gated block's gradients) stay within the tile kernels' 32-bit
// byte offsets.
constexpr int64_t MAX_LENGTH = (int64_t)1 << 22;

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool is_matrix_type(int dt) { return dt == RCD_F32 || dt == RCD_BF16; }
inline int64_t size_of(int dt) { return dt == RCD_F32 ? 4 : dt == RCD_BF16 ? 2 : 1; }
inline int64_t blocks_of(int64_t d) { return (d + MX_BLOCK - 1) / MX_BLOCK; }

// Rows that may be accessed `bytes` at a time.
inline bool rows_aligned(const void *p, int64_t ld, int64_t esz, int64_t bytes = 16)
{
    return !p || ((reinterpret_cast<uintptr_t>(p) % bytes) == 0 && (ld * esz) % bytes == 0);
}

// Takes pieces of a workspace, or (base null) only adds up what they need.
struct Pieces {
    char *base;
    size_t used = 0;
    explicit Pieces(void *p) : base((char *)p) {}
    template <typename T> T *take(size_t count)
    {
        T *p = base ? reinterpret_cast<T *>(base + used) : nullptr;
        used += up256(count * sizeof(T));
        return p;
    }
};

int check_pieces(const void *ws, size_t bytes, size_t need)
{
    if (need == 0) return RCD_OK;
    return !ws || (reinterpret_cast<uintptr_t>(ws) & 255) != 0 || bytes < need ? RCD_ERR_WORKSPACE : RCD_OK;
}

// ---- norm -----------------------------------------------------------------------------------------------------------------

// Calls go(waves per row, chunks per thread) with the variant for rows of d: a wave holds up to 1024 elements of its row in
// registers, a workgroup up to 8192; longer rows are read twice.
template <typename Go> void with_row_variant(int64_t d, Go go)
{
    using std::integral_constant;
    if (d <= 512) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    else if (d <= 1024) go(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    else if (d <= 2048) go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (d <= 4096) go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    else if (d <= 8192) go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    else go(integral_constant<int, 4>{}, integral_constant<int, 0>{});
}
inline int rows_per_workgroup(int64_t d) { return d <= 1024 ? 4 : 1; }

// (One launch unless there are 2^24 rows or more.)
template <bool MX, bool NORM> int launch_norm(NormArgs a, int dt, hipStream_t stream)
{
    static_assert(NORM_THREADS == 256, "the rule counts workgroups of 256");
    const int64_t rows = a.rows;
    for (int64_t done = 0; done < rows; done = a.rows) {
        a.first = done;
        a.rows = done + enc_rules::rows_of_launch(rows - done, rows_per_workgroup(a.d));
        with_row_variant(a.d, [&](auto wpr, auto chunks) {
            constexpr int W = decltype(wpr)::value, C = decltype(chunks)::value;
            const dim3 grid((unsigned)((a.rows - a.first + RowOf<W>::ROWS - 1) / RowOf<W>::ROWS));
            if (dt == RCD_F32) hipLaunchKernelGGL((k_norm<float, W, C, MX, NORM>), grid, dim3(NORM_THREADS), 0, stream, a);
            else hipLaunchKernelGGL((k_norm<__bf16, W, C, MX, NORM>), grid, dim3(NORM_THREADS), 0, stream, a);
        });
        ENC_HIP_TRY(hipGetLastError());
    }
    return RCD_OK;
}

// Row groups of the backward kernel, each with its own sums for the weight's gradient.  Rows of a workgroup of their own: as
// many workgroups as the device holds at once (50 000 x 2048 bf16: 161 us and 8 for the sums; with half of them 187 and 6).
inline int64_t norm_groups(int64_t rows, int64_t d)
{
    const int64_t per = rows_per_workgroup(d);
    return std::min<int64_t>((rows + per - 1) / per, per == 1 ? 2048 : 1024) * per;
}
inline int64_t part_pitch(int64_t d) { return (d + 63) / 64 * 64; }

// ---- products -------------------------------------------------------------------------------------------------------------

// What is set up once per device: the tile kernels use more LDS than a kernel may by default.
constexpr int MAX_DEVICES = 64;
std::mutex g_setup_mutex;
bool g_ready[MAX_DEVICES] = {};

template <int WT, int KA, int KB, bool MX, int TO> hipError_t raise_lds_limit()
{
    return hipFuncSetAttribute(reinterpret_cast<const void *>(&tile::k_tile<WT, KA, KB, MX, TO>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, tile::Shape<WT, MX>::LDS_BYTES);
}

// Calls go(WT, KA, KB, MX, TO) as constants, for the variants that there are: both operands with k contiguous (bf16, pieces of
// fp32, 8 bits; linear or gated), and for the gradients a K_RUNS by ROWS_RUN and a ROWS_RUN by ROWS_RUN product.
template <typename Go> int with_tile_variant(int wt, int ka, int kb, bool mx, int to, Go go)
{
    using std::integral_constant;
    auto by_target = [&](auto w, auto a, auto b, auto x) {
        constexpr int A = decltype(a)::value;
        constexpr int B = decltype(b)::value;
        if (to == tile::TO_LINEAR) return go(w, a, b, x, integral_constant<int, tile::TO_LINEAR>{});
        if (to == tile::TO_PARTS) return go(w, a, b, x, integral_constant<int, tile::TO_PARTS>{});
        if constexpr (!decltype(x)::value)
            if (to == tile::TO_LINEAR_PIECES) return go(w, a, b, x, integral_constant<int, tile::TO_LINEAR_PIECES>{});
        if constexpr (A == tile::K_RUNS && B == tile::K_RUNS) {
            if (to == tile::TO_GATED) return go(w, a, b, x, integral_constant<int, tile::TO_GATED>{});
            if (to == tile::TO_GATED_PARTS) return go(w, a, b, x, integral_constant<int, tile::TO_GATED_PARTS>{});
            if constexpr (!decltype(x)::value)
                if (to == tile::TO_GATED_PIECES) return go(w, a, b, x, integral_constant<int, tile::TO_GATED_PIECES>{});
        }
        return (int)RCD_ERR_UNSUPPORTED;
    };
    using K = integral_constant<int, tile::K_RUNS>;
    using R = integral_constant<int, tile::ROWS_RUN>;
    auto by_order = [&](auto w) {
        if (mx) return by_target(w, K{}, K{}, std::true_type{});
        if (ka == tile::K_RUNS && kb == tile::K_RUNS) return by_target(w, K{}, K{}, std::false_type{});
        if (ka == tile::K_RUNS) return by_target(w, K{}, R{}, std::false_type{});
        return by_target(w, R{}, R{}, std::false_type{});
    };
    return wt == 128 ? by_order(integral_constant<int, 128>{}) : by_order(integral_constant<int, 64>{});
}

int set_up()
{
    int dev = 0;
    ENC_HIP_TRY(hipGetDevice(&dev));
    if (dev < 0 || dev >= MAX_DEVICES) return rcd_note_hip_error("device index beyond 63", hipErrorInvalidDevice);
    std::lock_guard<std::mutex> lock(g_setup_mutex);
    if (!g_ready[dev]) {
        for (int wt : {64, 128})
            for (int order = 0; order < 4; ++order)
                for (int to : {tile::TO_LINEAR, tile::TO_GATED, tile::TO_PARTS, tile::TO_GATED_PARTS, tile::TO_LINEAR_PIECES, tile::TO_GATED_PIECES}) {
                    const bool mx = order == 3;
                    const int ka = order == 2 ? tile::ROWS_RUN : tile::K_RUNS, kb = order == 1 || order == 2 ? tile::ROWS_RUN : tile::K_RUNS;
                    if ((kb == tile::ROWS_RUN && tile::is_gated(to)) || (mx && (to == tile::TO_LINEAR_PIECES || to == tile::TO_GATED_PIECES))) continue;
                    ENC_TRY(with_tile_variant(wt, ka, kb, mx, to, [](auto w, auto a, auto b, auto x, auto t) {
                        ENC_HIP_TRY((raise_lds_limit<decltype(w)::value, decltype(a)::value, decltype(b)::value, decltype(x)::value,
                                                     decltype(t)::value>()));
                        return (int)RCD_OK;
                    }));
                }
        for (const void *both : {reinterpret_cast<const void *>(&tile::k_tile_both<false>), reinterpret_cast<const void *>(&tile::k_tile_both<true>)})
            ENC_HIP_TRY(hipFuncSetAttribute(both, hipFuncAttributeMaxDynamicSharedMemorySize, (tile::Shape<64, false>::LDS_BYTES)));
        g_ready[dev] = true;
    }
    return RCD_OK;
}

// A matrix as the tile kernel reads it: where it lies if its rows can go into LDS 16 bytes at a time, else its packed copy.
struct Laid {
    const unsigned char *p = nullptr;
    const uint8_t *scale = nullptr;
    int64_t pitch = 0, scale_pitch = 0;     // bytes
    int64_t plane = 0;                      // bytes between the pieces of fp32
    int64_t cols = 0;                       // what may be read of a row, a multiple of 8
};

inline int64_t up64(int64_t n) { return (n + 63) / 64 * 64; }
inline int64_t up128(int64_t n) { return (n + 127) / 128 * 128; }

// 8-bit products go to the scaled matrix instruction from this many k on, and only where nothing but a bf16 result leaves the
// call (`narrow`); all others are computed in bf16, from widened copies, which is exact.  The instruction lines
// up the 64 products that it adds with the largest of them and cuts off what lies some 2^-11 below: measured, over all bit patterns, up
// to 2^-12.3 of the sum of the products' sizes, towards zero.  On random operands that is 1.5e-5 of a result's size at every K (an fp32 sum 5e-8), with
// ten-fold outlier channels 3.3e-5, with operands that cancel to 1/4000 of their products' sizes 1.9e-4; rounding to bf16 alone is off by 1.7e-3.  So it stays
// below a bf16 result's own rounding, and is two orders above that of an fp32 one.  Below 2048 it would pass what an fp32 sum of K
// terms may be off at worst, (K + 8) 2^-23 of the products' sizes.
constexpr int64_t MX_INSTRUCTION_FROM = 2048;
inline int product_type(int dt, int64_t K, bool narrow)
{
    return dt == RCD_MXFP8 && (K < MX_INSTRUCTION_FROM || !narrow) ? RCD_BF16 : dt;
}

// Room for a matrix's packed copy as an operand of type dt, whatever its alignment (8 bits: its scales too).
size_t packed_bytes(int64_t rows, int64_t cols, int dt)
{
    if (dt == RCD_MXFP8) return up256((size_t)rows * up128(cols)) + up256((size_t)rows * (up128(cols) / MX_BLOCK));
    return up256((size_t)rows * up64(cols) * 2 * (dt == RCD_F32 ? 3 : 1));
}

inline unsigned copy_grid(int64_t items) { return (unsigned)std::min<int64_t>((items + 255) / 256, 8192); }

// Packs what of up to three matrices cannot be read in place (fp32: all of them, in pieces), in one launch.
struct Packer {
    int dt, type;                       // of the matrices, and of the product (8 bits are widened where they differ)
    PackJobs jobs{};
    ByteJobs bytes{};
    WidenJobs wide{};
    int njobs = 0, nbytes = 0, nwide = 0;
    int64_t most = 0;
    bool always = false;

    Laid lay(Pieces &room, const void *src, const uint8_t *scale, int64_t ld_scale, int64_t rows, int64_t cols, int64_t ld)
    {
        Laid l;
        // offsets inside a tile are 32 bits: rows too far apart are brought together first
        const int64_t far = (int64_t)1 << 23;
        if (dt != type) {
            __bf16 *q = room.take<__bf16>((size_t)rows * up64(cols));
            l.p = (const unsigned char *)q;
            l.pitch = up64(cols) * 2;
            l.cols = up64(cols);
            wide.job[nwide++] = WidenJob{(const uint8_t *)src, scale, q, (long long)ld, (long long)ld_scale, (long long)up64(cols),
                                         (int)rows, (int)cols};
            most = std::max(most, rows * up64(cols) / 8);
            return l;
        }
        if (dt == RCD_MXFP8) {
            uint8_t *q = room.take<uint8_t>((size_t)rows * up128(cols));
            uint8_t *s = room.take<uint8_t>((size_t)rows * (up128(cols) / MX_BLOCK));
            l.p = (const unsigned char *)src;
            l.pitch = ld;
            if (always || !rows_aligned(src, ld, 1) || cols % 16 || ld > far) {
                l.p = q;
                l.pitch = up128(cols);
                add(ByteJob{(const uint8_t *)src, q, (long long)ld, (long long)l.pitch, (int)rows, (int)cols});
            }
            l.scale = scale;
            l.scale_pitch = ld_scale;
            if (always || !rows_aligned(scale, ld_scale, 1, 4) || cols % 128 || ld_scale > far) {
                l.scale = s;
                l.scale_pitch = up128(cols) / MX_BLOCK;
                add(ByteJob{scale, s, (long long)ld_scale, (long long)l.scale_pitch, (int)rows, (int)blocks_of(cols)});
            }
            return l;
        }
        const bool f32 = dt == RCD_F32;
        __bf16 *q = room.take<__bf16>((size_t)rows * up64(cols) * (f32 ? 3 : 1));
        l.p = (const unsigned char *)src;
        l.pitch = ld * 2;
        l.cols = cols;
        if (always || f32 || !rows_aligned(src, ld, 2) || cols % 8 || l.pitch > far) {
            l.p = (const unsigned char *)q;
            l.pitch = up64(cols) * 2;
            l.plane = rows * l.pitch;
            l.cols = up64(cols);
            jobs.job[njobs++] = PackJob{src, q, (long long)ld, (long long)up64(cols), (long long)(rows * up64(cols)), (int)rows,
                                        (int)cols};
            most = std::max(most, rows * up64(cols) / 8);
        }
        return l;
    }
    void add(const ByteJob &j)
    {
        bytes.job[nbytes++] = j;
        most = std::max<int64_t>(most, (int64_t)j.rows * j.pitch / 4);
    }
    int launch(hipStream_t stream)
    {
        if (njobs) {
            const dim3 grid(copy_grid(most), (unsigned)njobs);
            if (dt == RCD_F32) hipLaunchKernelGGL((k_pack<float, 3>), grid, dim3(256), 0, stream, jobs);
            else hipLaunchKernelGGL((k_pack<__bf16, 1>), grid, dim3(256), 0, stream, jobs);
        }
        if (nbytes) hipLaunchKernelGGL(k_pack_bytes, dim3(copy_grid(most), (unsigned)nbytes), dim3(256), 0, stream, bytes);
        if (nwide) hipLaunchKernelGGL(k_widen, dim3(copy_grid(most), (unsigned)nwide), dim3(256), 0, stream, wide);
        ENC_HIP_TRY(hipGetLastError());
        return RCD_OK;
    }
};

// C (M x N) = sum over pairs of a_i b_i, over k of K.
struct Product {
    int64_t M, N, K;
    int dt;                             // RCD_F32: operands in pieces
    int ka, kb;                         // tile::K_RUNS or ROWS_RUN
    bool gated;
    int pairs;                          // 1, or 2 products summed
    Laid a[2], b[2];                    // gated: b[1] is the second weight
    int64_t a_shift;                    // bytes from the first pair's a to the second's (same matrix)
    Epilogue e;
};

int64_t stages_of(int64_t K, int dt, int pairs)
{
    const int64_t per = dt == RCD_MXFP8 ? 128 : 64;
    return (K + per - 1) / per * (dt == RCD_F32 ? 6 : 1) * pairs;
}
inline int64_t parts_pitch(int64_t N, bool gated) { return (N + 7) / 8 * 8 * (gated ? 2 : 1); }

using enc_rules::Cut;
Cut cut_of(int64_t M, int64_t N, int64_t K, int dt, int pairs, bool gated)
{
    Cut c = enc_rules::cut_of(M, N, stages_of(K, dt, pairs), gated);
    return c;
}
size_t parts_bytes(const Cut &c, int64_t M, int64_t N, bool gated)
{
    return c.splits > 1 ? up256((size_t)c.splits * M * parts_pitch(N, gated) * 4) : 0;
}

using enc_rules::launchable;
inline unsigned grid_size(const Cut &c) { return (unsigned)enc_rules::grid_of(c); }

void take_parts(tile::Args &x, bool gated, Pieces &room)
{
    if (x.splits == 1) return;
    x.parts_pitch = parts_pitch(x.N, gated);
    x.parts_half = (int)(x.parts_pitch / 2);
    x.parts = room.take<float>((size_t)x.splits * x.M * x.parts_pitch);
}

int sum_columns(const tile::Columns &c, hipStream_t stream)
{
    const dim3 grid((unsigned)((c.d + 15) / 16));
    if (c.f32)
        hipLaunchKernelGGL(k_column_sums<float>, grid, dim3(1024), 0, stream, c.part, c.pitch, c.groups, c.d, (float *)c.out);
    else
        hipLaunchKernelGGL(k_column_sums<__bf16>, grid, dim3(1024), 0, stream, c.part, c.pitch, c.groups, c.d, (__bf16 *)c.out);
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

// Workgroups that join a product's parts.
int64_t join_groups(const tile::Args &x)
{
    if (x.splits == 1) return 1;
    const int64_t M = x.M, N = x.N;
    const int64_t groups = x.pieces.a[0] ? (M + 31) / 32 * ((N + 63) / 64) : (M * ((N + 7) / 8) + 255) / 256;
    return std::min<int64_t>(groups, 8192);
}

int launch_join_both(const tile::Args &x, const tile::Args &y, const tile::Columns &c, hipStream_t stream)
{
    if (x.splits > 1 || y.splits > 1 || c.part) {
        const dim3 grid((unsigned)std::max({join_groups(x), join_groups(y), std::min<int64_t>((c.d + 15) / 16, 8192)}), 3);
        if (x.pieces.a[0]) hipLaunchKernelGGL(tile::k_join_both<true>, grid, dim3(256), 0, stream, x, y, c);
        else hipLaunchKernelGGL(tile::k_join_both<false>, grid, dim3(256), 0, stream, x, y, c);
    }
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

void launch_join(const tile::Args &x, bool gated, hipStream_t stream)
{
    const dim3 grid((unsigned)join_groups(x));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, x); };
    if (x.pieces.a[0]) gated ? launch(tile::k_join<true, true>) : launch(tile::k_join<false, true>);
    else gated ? launch(tile::k_join<true, false>) : launch(tile::k_join<false, false>);
}

// The kernel's arguments; parts are taken from `room`.
tile::Args plan_product(const Product &p, const Cut &c, Pieces &room)
{
    const bool mx = p.dt == RCD_MXFP8;
    tile::Args x{};
    auto side = [](const Laid &l, const Laid &second, int64_t rows, int kind) {
        Side s{};
        s.p = l.p;
        s.p2 = second.p;
        s.scale = l.scale;
        s.scale2 = second.scale;
        s.pitch = l.pitch;
        s.scale_pitch = l.scale_pitch;
        s.extent = (int)(kind == tile::K_RUNS ? rows : l.cols);
        return s;
    };
    x.a = side(p.a[0], p.a[0], p.M, p.ka);
    x.b = side(p.b[0], p.gated ? p.b[1] : p.b[0], p.N, p.kb);
    const int64_t per = mx ? 128 : 64;
    x.seg.stages = (int)((p.K + per - 1) / per);
    x.seg.rem = (int)(p.K % per);
    const int pieces = p.dt == RCD_F32 ? 6 : 1;
    for (int pair = 0; pair < p.pairs; ++pair)
        for (int i = 0; i < pieces; ++i) {
            const int s = x.seg.count++;
            x.seg.a[s] = pair * p.a_shift + (pieces == 6 ? PIECE_PAIRS[i][0] * p.a[0].plane : 0);
            x.seg.b[s] = (pair ? p.b[1].p - p.b[0].p : 0) + (pieces == 6 ? PIECE_PAIRS[i][1] * p.b[pair].plane : 0);
        }
    if (p.dt == RCD_F32) {
        Pieces3 &q = x.pieces;
        q.pairs = p.pairs;
        q.K = (int)p.K;
        for (int i = 0; i < 2; ++i) {
            q.a[i] = (const __bf16 *)(p.a[0].p + (i < p.pairs ? i * p.a_shift : 0));
            q.b[i] = (const __bf16 *)p.b[i < p.pairs || p.gated ? i : 0].p;
        }
        q.a_plane = p.a[0].plane / 2;
        q.b_plane = p.b[0].plane / 2;
        q.a_row = p.ka == tile::K_RUNS ? p.a[0].pitch / 2 : 1;
        q.a_k = p.ka == tile::K_RUNS ? 1 : p.a[0].pitch / 2;
        q.b_row = p.kb == tile::K_RUNS ? p.b[0].pitch / 2 : 1;
        q.b_k = p.kb == tile::K_RUNS ? 1 : p.b[0].pitch / 2;
    }
    x.e = p.e;
    x.M = (int)p.M;
    x.N = (int)p.N;
    x.tiles_m = (int)c.tiles_m;
    x.tiles_n = (int)c.tiles_n;
    x.splits = c.splits;
    take_parts(x, p.gated, room);
    return x;
}

int launch_planned(const Product &p, const Cut &c, const tile::Args &x, hipStream_t stream)
{
    const bool mx = p.dt == RCD_MXFP8;
    const bool pieces = p.dt == RCD_F32;
    const int to = c.splits > 1 ? (p.gated ? tile::TO_GATED_PARTS : tile::TO_PARTS)
                   : p.gated    ? (pieces ? tile::TO_GATED_PIECES : tile::TO_GATED)
                                : (pieces ? tile::TO_LINEAR_PIECES : tile::TO_LINEAR);
    ENC_TRY(with_tile_variant(c.wt, p.ka, p.kb, mx, to, [&](auto w, auto a, auto b, auto m, auto t) {
        constexpr int W = decltype(w)::value;
        constexpr bool X = decltype(m)::value;
        hipLaunchKernelGGL((tile::k_tile<W, decltype(a)::value, decltype(b)::value, X, decltype(t)::value>), dim3(grid_size(c)),
                           dim3(tile::THREADS), (tile::Shape<W, X>::LDS_BYTES), stream, x);
        return (int)RCD_OK;
    }));
    if (c.splits > 1) launch_join(x, p.gated, stream);
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

int launch_product(const Product &p, Pieces &room, hipStream_t stream)
{
    ENC_TRY(set_up());
    const Cut c = cut_of(p.M, p.N, p.K, p.dt, p.pairs, p.gated);
    if (!launchable(c)) return RCD_ERR_UNSUPPORTED;
    return launch_planned(p, c, plan_product(p, c, room), stream);
}

enc_rules::Both both_of(int64_t M, int64_t N, int64_t K, int dt, int pairs)
{
    // dA: M x K over N (`pairs` of them), dW: pairs N x K over M
    return enc_rules::both_of(M, K, stages_of(N, dt, pairs), pairs == 2 ? 2 * up64(N) : N, K, stages_of(M, dt, 1));
}

// A backward call's two products (either may be missing) and the bias's column sums.
int launch_both(const Product *da, const Product *dw, const enc_rules::Both &cut, Pieces &room, const tile::Columns &cols,
                hipStream_t stream)
{
    ENC_TRY(set_up());
    if ((da && !launchable(cut.first)) || (dw && !launchable(cut.second))) return RCD_ERR_UNSUPPORTED;
    if (da && dw && cut.together) {
        const tile::Args x = plan_product(*da, cut.first, room), y = plan_product(*dw, cut.second, room);
        const unsigned first = grid_size(cut.first);
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(first + grid_size(cut.second)), dim3(tile::THREADS), (tile::Shape<64, false>::LDS_BYTES), stream, x, y,
                               (int)first);
        };
        if (da->dt == RCD_F32) launch(tile::k_tile_both<true>);
        else launch(tile::k_tile_both<false>);
        return launch_join_both(x, y, cols, stream);
    }
    if (cols.part) ENC_TRY(sum_columns(cols, stream));
    const size_t mark = room.used;
    if (da) ENC_TRY(launch_planned(*da, cut.first, plan_product(*da, cut.first, room), stream));
    room.used = mark;
    if (dw) ENC_TRY(launch_planned(*dw, cut.second, plan_product(*dw, cut.second, room), stream));
    return RCD_OK;
}
size_t both_parts(const enc_rules::Both &b, int64_t M, int64_t N, int64_t M2, int64_t N2)
{
    const size_t first = parts_bytes(b.first, M, N, false), second = parts_bytes(b.second, M2, N2, false);
    return b.together ? first + second : std::max(first, second);
}

// fp32 operands in place.
struct DirectProduct {
    int64_t M, N, K;
    int ka, kb, pairs;
    bool gated;
    const float *a[2], *b[2];
    int64_t a_pitch, b_pitch[2];
    int64_t a_extent, b_extent;         // rows
    int64_t a_cols, b_cols;             // what may be read of a contiguous run: of a row (k contiguous) or of a line (rows contiguous)
    Epilogue e;
};
// Whether both operands can go into LDS 16 bytes a lane.
bool is_wide(const DirectProduct &p)
{
    auto side = [&](const float *x, int64_t pitch, int kind, int64_t cols) {
        return !x || (rows_aligned(x, pitch, 4) && (kind == tile::K_RUNS ? (p.K + 3) / 4 * 4 <= cols : cols % 4 == 0 && pitch <= ((int64_t)1 << 23)));
    };
    const bool second = p.pairs == 2;
    return side(p.a[0], p.a_pitch, p.ka, p.a_cols) && side(second ? p.a[1] : nullptr, p.a_pitch, p.ka, p.a_cols) &&
           side(p.b[0], p.b_pitch[0], p.kb, p.b_cols) && side(second || p.gated ? p.b[1] : nullptr, p.b_pitch[1], p.kb, p.b_cols);
}
Cut direct_cut(int64_t M, int64_t N, int64_t K, int pairs, bool gated)
{
    return enc_rules::direct_cut_of(M, N, enc_rules::ceil_div(K, enc_rules::DIRECT_STAGE) * pairs, gated);
}

size_t direct_parts(int64_t M, int64_t N, int64_t K, int pairs, bool gated, int dt)
{
    return dt == RCD_F32 ? parts_bytes(direct_cut(M, N, K, pairs, gated), M, N, gated) : 0;
}

// Rows of these pitches lie near enough for the direct kernel's 32-bit offsets inside a tile.
inline bool near_enough(int64_t ld_a, int64_t ld_b = 0, int64_t ld_c = 0) { return std::max({ld_a, ld_b, ld_c}) <= ((int64_t)1 << 23); }

direct::Args plan_direct(const DirectProduct &p, const Cut &c, Pieces &room)
{
    static_assert(enc_rules::DIRECT_STAGE == direct::KS, "the rule counts the kernel's stages");
    direct::Args x{};
    for (int i = 0; i < 2; ++i) {
        x.a[i] = p.a[i];
        x.b[i] = p.b[i];
        x.b_pitch[i] = p.b_pitch[i];
    }
    x.a_pitch = p.a_pitch;
    x.a_extent = (int)(p.ka == tile::K_RUNS ? p.a_extent : p.a_cols);
    x.b_extent = (int)(p.kb == tile::K_RUNS ? p.b_extent : p.b_cols);
    x.pairs = p.pairs;
    x.K = (int)p.K;
    x.t.e = p.e;
    x.t.M = (int)p.M;
    x.t.N = (int)p.N;
    x.t.tiles_m = (int)c.tiles_m;
    x.t.tiles_n = (int)c.tiles_n;
    x.t.splits = c.splits;
    take_parts(x.t, p.gated, room);
    return x;
}

int launch_planned(const DirectProduct &p, const Cut &c, const direct::Args &x, hipStream_t stream)
{
    const dim3 grid(grid_size(c));
    constexpr int K = tile::K_RUNS, R = tile::ROWS_RUN;
    auto go = [&](auto wide) {
        constexpr bool W = decltype(wide)::value;
        auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, x); };
        if (p.gated) {
            if (c.splits > 1) launch(direct::k_direct<K, K, tile::TO_GATED_PARTS, W>);
            else launch(direct::k_direct<K, K, tile::TO_GATED, W>);
        } else if (p.ka == R) {
            if (c.splits > 1) launch(direct::k_direct<R, R, tile::TO_PARTS, W>);
            else launch(direct::k_direct<R, R, tile::TO_LINEAR, W>);
        } else if (p.kb == R) {
            if (c.splits > 1) launch(direct::k_direct<K, R, tile::TO_PARTS, W>);
            else launch(direct::k_direct<K, R, tile::TO_LINEAR, W>);
        } else {
            if (c.splits > 1) launch(direct::k_direct<K, K, tile::TO_PARTS, W>);
            else launch(direct::k_direct<K, K, tile::TO_LINEAR, W>);
        }
    };
    if (is_wide(p)) go(std::true_type{});
    else go(std::false_type{});
    if (c.splits > 1) launch_join(x.t, p.gated, stream);
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

int launch_direct(const DirectProduct &p, Pieces &room, hipStream_t stream)
{
    const Cut c = direct_cut(p.M, p.N, p.K, p.pairs, p.gated);
    if (!launchable(c)) return RCD_ERR_UNSUPPORTED;
    return launch_planned(p, c, plan_direct(p, c, room), stream);
}

int launch_both(const DirectProduct *da, const DirectProduct *dw, const enc_rules::Both &cut, Pieces &room, const tile::Columns &cols,
                hipStream_t stream)
{
    if ((da && !launchable(cut.first)) || (dw && !launchable(cut.second))) return RCD_ERR_UNSUPPORTED;
    if (da && dw) {
        const direct::Args x = plan_direct(*da, cut.first, room), y = plan_direct(*dw, cut.second, room);
        const unsigned first = grid_size(cut.first);
        const dim3 grid(first + grid_size(cut.second));
        if (is_wide(*da) && is_wide(*dw)) hipLaunchKernelGGL(direct::k_direct_both<true>, grid, dim3(256), 0, stream, x, y, (int)first);
        else hipLaunchKernelGGL(direct::k_direct_both<false>, grid, dim3(256), 0, stream, x, y, (int)first);
        return launch_join_both(x.t, y.t, cols, stream);
    }
    if (cols.part) ENC_TRY(sum_columns(cols, stream));
    if (da) ENC_TRY(launch_planned(*da, cut.first, plan_direct(*da, cut.first, room), stream));
    if (dw) ENC_TRY(launch_planned(*dw, cut.second, plan_direct(*dw, cut.second, room), stream));
    return RCD_OK;
}

// Parts of a backward call's two products, whichever way they go.
size_t backward_parts(int64_t M, int64_t N, int64_t K, int dt, int pairs)
{
    const int64_t rows = pairs == 2 ? 2 * up64(N) : N;
    size_t need = both_parts(both_of(M, N, K, dt, pairs), M, K, rows, K);
    if (dt == RCD_F32) need = std::max(need, both_parts(enc_rules::direct_both(M, N, K, pairs == 2), M, K, rows, K));
    return need;
}


// Workspace of a forward product, whichever way it goes (8 bits: whatever its result's type).
size_t forward_bytes(int64_t M, int64_t N, int64_t K, int dt, bool gated)
{
    size_t most = 0;
    for (bool narrow : {false, true}) {
        const int type = product_type(dt, K, narrow);
        const size_t parts = std::max(parts_bytes(cut_of(M, N, K, type, 1, gated), M, N, gated), direct_parts(M, N, K, 1, gated, dt));
        most = std::max(most, packed_bytes(M, K, type) + (gated ? 2 : 1) * packed_bytes(N, K, type) + parts);
    }
    return most;
}

inline bool few_rows(int64_t M, int64_t N, int64_t K, int dt) { return enc_rules::few_rows(M, N, K, dt == RCD_F32, dt == RCD_MXFP8); }

int launch_few(int dt, bool gated, const few::Args &x, hipStream_t stream)
{
    if (dt == RCD_F32) {
        const int cols = gated ? 4 : 8;
        auto go = [&](auto mr) {
            constexpr int MR = decltype(mr)::value;
            const dim3 grid((unsigned)((x.N + cols - 1) / cols), (unsigned)((x.M + MR - 1) / MR));
            if (gated) hipLaunchKernelGGL((few::k_few_f32<MR, true>), grid, dim3(256), 0, stream, x);
            else hipLaunchKernelGGL((few::k_few_f32<MR, false>), grid, dim3(256), 0, stream, x);
        };
        if (x.M == 1) go(std::integral_constant<int, 1>{});
        else if (x.M <= 4) go(std::integral_constant<int, 4>{});
        else go(std::integral_constant<int, 8>{});
    } else {
        const dim3 grid((unsigned)((x.N + 15) / 16));
        auto go = [&](auto mt, auto waves) {
            constexpr int MT = decltype(mt)::value, W = decltype(waves)::value;
            if (dt == RCD_MXFP8) {
                if (gated) hipLaunchKernelGGL((few::k_few<MT, W, true, true>), grid, dim3(64 * W), 0, stream, x);
                else hipLaunchKernelGGL((few::k_few<MT, W, true, false>), grid, dim3(64 * W), 0, stream, x);
            } else {
                if (gated) hipLaunchKernelGGL((few::k_few<MT, W, false, true>), grid, dim3(64 * W), 0, stream, x);
                else hipLaunchKernelGGL((few::k_few<MT, W, false, false>), grid, dim3(64 * W), 0, stream, x);
            }
        };
        using std::integral_constant;
        if (x.M <= 16 && grid.x < 256) go(integral_constant<int, 1>{}, integral_constant<int, 16>{});
        else if (x.M <= 16) go(integral_constant<int, 1>{}, integral_constant<int, 8>{});
        else if (x.M <= 32) go(integral_constant<int, 2>{}, integral_constant<int, 4>{});
        else go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    }
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

int zero_matrix(void *p, int dt, int64_t ld, int64_t rows, int64_t cols, hipStream_t stream)
{
    if (!p) return RCD_OK;
    const dim3 grid((unsigned)std::min<int64_t>(rows, 4096));
    if (dt == RCD_F32) hipLaunchKernelGGL(k_zero<float>, grid, dim3(256), 0, stream, (float *)p, (long long)ld, (int)rows, (int)cols);
    else hipLaunchKernelGGL(k_zero<__bf16>, grid, dim3(256), 0, stream, (__bf16 *)p, (long long)ld, (int)rows, (int)cols);
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

// The pass before a backward product: threads side by side over eight columns each, groups of rows.
struct SlopeCut {
    int across;
    int64_t pieces, groups;
};
SlopeCut slope_cut(int64_t M, int64_t cols)
{
    SlopeCut c;
    c.across = 1;
    while (c.across < 256 && c.across * 8 < cols) c.across *= 2;
    c.pieces = (cols + 8 * c.across - 1) / (8 * c.across);
    const int64_t down = 256 / c.across;
    c.groups = std::max<int64_t>(1, std::min<int64_t>((M + 4 * down - 1) / (4 * down), 1024 / std::min<int64_t>(c.pieces, 4)));
    return c;
}

template <typename Go> void with_act_value(int act, Go go)
{
    using std::integral_constant;
    if (act == RCD_ACT_NONE) go(integral_constant<int, 0>{});
    else if (act == RCD_ACT_RELU) go(integral_constant<int, 1>{});
    else if (act == RCD_ACT_SILU) go(integral_constant<int, 2>{});
    else go(integral_constant<int, 3>{});
}

// Workspace of the linear backward call.
struct LinearBack {
    __bf16 *dz;
    float *part;
    size_t used;
};
LinearBack linear_back(Pieces &w, int64_t M, int64_t N, int dt)
{
    LinearBack p;
    p.dz = w.take<__bf16>((size_t)M * up64(N) * (dt == RCD_F32 ? 3 : 1));
    p.part = w.take<float>((size_t)slope_cut(M, up64(N)).groups * part_pitch(N));
    return p;
}

// Types and extents of a product's call.
int check_product(int dt, int out_dt, int64_t M, int64_t N, int64_t K, int act)
{
    if (dt != RCD_F32 && dt != RCD_BF16 && dt != RCD_MXFP8) return RCD_ERR_UNSUPPORTED;
    if (!is_matrix_type(out_dt) || (dt == RCD_F32 && out_dt != RCD_F32)) return RCD_ERR_UNSUPPORTED;
    if (act < RCD_ACT_NONE || act > RCD_ACT_GELU) return RCD_ERR_UNSUPPORTED;
    if (M < 0 || N < 1 || K < 1) return RCD_ERR_INVALID_ARG;
    if (M > MAX_EXTENT || N > MAX_LENGTH || K > MAX_LENGTH) return RCD_ERR_UNSUPPORTED;
    return RCD_OK;
}

inline bool product_sizes_ok(int64_t M, int64_t N, int64_t K)
{
    return M >= 1 && M <= MAX_EXTENT && N >= 1 && N <= MAX_LENGTH && K >= 1 && K <= MAX_LENGTH;
}

Epilogue one_output(void *out, int64_t ld, int dt, int act)
{
    Epilogue e{};
    e.out = out;
    e.ld_o = ld;
    e.act = act;
    e.split_row = e.rows_each = 0x7fffffff;
    e.out_f32 = dt == RCD_F32;
    return e;
}

few::Args few_args(int dt, const void *a, const uint8_t *scale, int64_t ld, int64_t ld_scale, int64_t M, int64_t N, int64_t K, const Epilogue &e)
{
    few::Args x{};
    x.a = (const unsigned char *)a;
    x.a_pitch = ld * size_of(dt);
    x.sa = scale;
    x.sa_pitch = ld_scale;
    x.e = e;
    x.M = (int)M; x.N = (int)N; x.K = (int)K;
    return x;
}
void few_weight(few::Args &x, int dt, bool second, const void *w, const uint8_t *scale, int64_t ld, int64_t ld_scale)
{
    (second ? x.b2 : x.b) = (const unsigned char *)w;
    (second ? x.b2_pitch : x.b_pitch) = ld * size_of(dt);
    (second ? x.sb2 : x.sb) = scale;
    (second ? x.sb2_pitch : x.sb_pitch) = ld_scale;
}

// The gated block's two weights.  The tile kernel wants one pitch for both: if they differ, or one can be read in place
// and the other not, both are packed.
int lay_pair(Packer &pack, Pieces &room, Laid (&b)[2], int dt, const void *wg, const uint8_t *sg, int64_t ld_g, int64_t ld_sg,
             const void *wu, const uint8_t *su, int64_t ld_u, int64_t ld_su, int64_t F, int64_t K)
{
    const int jobs = pack.njobs, bytes = pack.nbytes;
    const size_t used = room.used;
    b[0] = pack.lay(room, wg, sg, ld_sg, F, K, ld_g);
    b[1] = pack.lay(room, wu, su, ld_su, F, K, ld_u);
    if (b[0].pitch == b[1].pitch && b[0].scale_pitch == b[1].scale_pitch && b[0].plane == b[1].plane) return RCD_OK;
    pack.njobs = jobs;
    pack.nbytes = bytes;
    room.used = used;
    pack.always = true;
    b[0] = pack.lay(room, wg, sg, ld_sg, F, K, ld_g);
    b[1] = pack.lay(room, wu, su, ld_su, F, K, ld_u);
    return RCD_OK;
}

int check_mx_operand(int dt, const uint8_t *scale, int64_t ld_scale, int64_t K)
{
    if (dt != RCD_MXFP8) return RCD_OK;
    return scale && ld_scale >= blocks_of(K) ? RCD_OK : RCD_ERR_INVALID_ARG;
}

} // namespace

int rcd_set_up_encoder() { return set_up(); }

extern "C" {

int rcd_rms_norm(const void *X_dev, int dt, int64_t rows, int64_t d, int64_t ld_x, const void *residual_dev, int64_t ld_r,
                 const void *weight_dev, float eps, void *sum_dev, int64_t ld_s, void *Y_dev, int out_dt, int64_t ld_y,
                 uint8_t *scale_dev, int64_t ld_scale, float *rstd_dev, void *stream)
{
    if (!is_matrix_type(dt) || (out_dt != dt && out_dt != RCD_MXFP8)) return RCD_ERR_UNSUPPORTED;
    const bool mx = out_dt == RCD_MXFP8;
    if (rows < 0 || d < 1 || ld_x < d || ld_y < d || (residual_dev && ld_r < d) || (sum_dev && ld_s < d) ||
        (mx && ld_scale < blocks_of(d)) || !(eps >= 0.f) || !std::isfinite(eps))
        return RCD_ERR_INVALID_ARG;
    if (rows > MAX_EXTENT || d > MAX_NORM_LENGTH) return RCD_ERR_UNSUPPORTED;
    if (rows == 0) return RCD_OK;
    if (!X_dev || !Y_dev || (mx && !scale_dev)) return RCD_ERR_INVALID_ARG;
    if (sum_dev == Y_dev) return RCD_ERR_INVALID_ARG;
    NormArgs a{};
    a.x = X_dev; a.r = residual_dev; a.w = weight_dev;
    a.sum = sum_dev; a.y = Y_dev; a.scale = scale_dev; a.rstd = rstd_dev;
    a.ld_x = ld_x; a.ld_r = ld_r; a.ld_s = ld_s; a.ld_y = ld_y; a.ld_scale = ld_scale;
    a.rows = rows; a.d = (int)d; a.eps = eps;
    return mx ? launch_norm<true, true>(a, dt, (hipStream_t)stream) : launch_norm<false, true>(a, dt, (hipStream_t)stream);
}

int rcd_quantize_mxfp8(const void *X_dev, int dt, int64_t rows, int64_t d, int64_t ld_x, uint8_t *Q_dev, int64_t ld_q,
                       uint8_t *scale_dev, int64_t ld_scale, void *stream)
{
    if (!is_matrix_type(dt)) return RCD_ERR_UNSUPPORTED;
    if (rows < 0 || d < 1 || ld_x < d || ld_q < d || ld_scale < blocks_of(d)) return RCD_ERR_INVALID_ARG;
    if (rows > MAX_EXTENT || d > MAX_NORM_LENGTH) return RCD_ERR_UNSUPPORTED;
    if (rows == 0) return RCD_OK;
    if (!X_dev || !Q_dev || !scale_dev) return RCD_ERR_INVALID_ARG;
    NormArgs a{};
    a.x = X_dev; a.y = Q_dev; a.scale = scale_dev;
    a.ld_x = ld_x; a.ld_y = ld_q; a.ld_scale = ld_scale;
    a.rows = rows; a.d = (int)d;
    return launch_norm<true, false>(a, dt, (hipStream_t)stream);
}

size_t rcd_rms_norm_backward_workspace_bytes(int64_t rows, int64_t d)
{
    if (rows < 1 || rows > MAX_EXTENT || d < 1 || d > MAX_NORM_LENGTH) return 0;
    return up256((size_t)norm_groups(rows, d) * part_pitch(d) * 4);
}

int rcd_rms_norm_backward(const void *dY_dev, int dt, int64_t rows, int64_t d, int64_t ld_dy, const void *H_dev, int64_t ld_h,
                          const float *rstd_dev, const void *weight_dev, const void *dsum_dev, int64_t ld_ds,
                          void *dX_dev, int64_t ld_dx, void *dweight_dev,
                          void *workspace_dev, size_t workspace_bytes, void *stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    if (!is_matrix_type(dt)) return RCD_ERR_UNSUPPORTED;
    if (rows < 0 || d < 1 || ld_dy < d || ld_h < d || ld_dx < d || (dsum_dev && ld_ds < d)) return RCD_ERR_INVALID_ARG;
    if (rows > MAX_EXTENT || d > MAX_NORM_LENGTH) return RCD_ERR_UNSUPPORTED;
    if (rows == 0) return zero_matrix(dweight_dev, dt, d, 1, d, stream);
    if (!dY_dev || !H_dev || !rstd_dev || !dX_dev) return RCD_ERR_INVALID_ARG;
    const int64_t groups = norm_groups(rows, d);
    if (dweight_dev) ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_rms_norm_backward_workspace_bytes(rows, d)));
    NormBackArgs a{};
    a.dy = dY_dev; a.h = H_dev; a.w = weight_dev; a.dsum = dsum_dev; a.rstd = rstd_dev;
    a.dx = dX_dev; a.part = dweight_dev ? (float *)workspace_dev : nullptr;
    a.ld_dy = ld_dy; a.ld_h = ld_h; a.ld_ds = ld_ds; a.ld_dx = ld_dx; a.part_pitch = part_pitch(d);
    a.rows = rows; a.d = (int)d;
    with_row_variant(d, [&](auto wpr, auto chunks) {
        constexpr int W = decltype(wpr)::value, C = decltype(chunks)::value;
        const dim3 grid((unsigned)(groups / RowOf<W>::ROWS));
        if (dt == RCD_F32) hipLaunchKernelGGL((k_norm_backward<float, W, C>), grid, dim3(NORM_THREADS), 0, stream, a);
        else hipLaunchKernelGGL((k_norm_backward<__bf16, W, C>), grid, dim3(NORM_THREADS), 0, stream, a);
    });
    ENC_HIP_TRY(hipGetLastError());
    if (!dweight_dev) return RCD_OK;
    return sum_columns(tile::Columns{a.part, dweight_dev, a.part_pitch, (int)groups, (int)d, dt == RCD_F32}, stream);
}

size_t rcd_linear_workspace_bytes(int64_t M, int64_t N, int64_t K, int dt)
{
    if (!product_sizes_ok(M, N, K) || dt < RCD_F32 || dt > RCD_MXFP8 || few_rows(M, N, K, dt)) return 0;
    return forward_bytes(M, N, K, dt, false);
}

int rcd_linear(const void *A_dev, const uint8_t *A_scale_dev, int64_t ld_a, int64_t ld_a_scale,
               const void *W_dev, const uint8_t *W_scale_dev, int64_t ld_w, int64_t ld_w_scale, int dt, int out_dt,
               int64_t M, int64_t N, int64_t K, const void *bias_dev, int act, const void *residual_dev, int64_t ld_r,
               float *preact_dev, int64_t ld_p, void *Y_dev, int64_t ld_y,
               void *workspace_dev, size_t workspace_bytes, void *stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    ENC_TRY(check_product(dt, out_dt, M, N, K, act));
    if (ld_a < K || ld_w < K || ld_y < N || (residual_dev && ld_r < N) || (preact_dev && ld_p < N)) return RCD_ERR_INVALID_ARG;
    if (M == 0) return RCD_OK;
    if (!A_dev || !W_dev || !Y_dev) return RCD_ERR_INVALID_ARG;
    ENC_TRY(check_mx_operand(dt, A_scale_dev, ld_a_scale, K));
    ENC_TRY(check_mx_operand(dt, W_scale_dev, ld_w_scale, K));
    ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_linear_workspace_bytes(M, N, K, dt)));
    Epilogue e = one_output(Y_dev, ld_y, out_dt, act);
    e.bias = bias_dev;
    e.residual = residual_dev;
    e.preact = preact_dev;
    e.ld_r = ld_r;
    e.ld_p = ld_p;
    if (few_rows(M, N, K, dt)) {
        few::Args x = few_args(dt, A_dev, A_scale_dev, ld_a, ld_a_scale, M, N, K, e);
        few_weight(x, dt, false, W_dev, W_scale_dev, ld_w, ld_w_scale);
        return launch_few(dt, false, x, stream);
    }
    Pieces room(workspace_dev);
    if (dt == RCD_F32 && enc_rules::direct_forward(M, N, K, false) && near_enough(ld_a, ld_w)) {
        DirectProduct p{};
        p.M = M; p.N = N; p.K = K;
        p.ka = p.kb = tile::K_RUNS;
        p.pairs = 1;
        p.a[0] = (const float *)A_dev;
        p.b[0] = (const float *)W_dev;
        p.a_pitch = ld_a;
        p.b_pitch[0] = ld_w;
        p.a_extent = M;
        p.b_extent = N;
        p.a_cols = p.b_cols = K;
        p.e = e;
        return launch_direct(p, room, stream);
    }
    Packer pack{dt, product_type(dt, K, out_dt == RCD_BF16 && !preact_dev)};
    Product p{};
    p.M = M; p.N = N; p.K = K;
    p.dt = pack.type;
    p.pairs = 1;
    p.a[0] = pack.lay(room, A_dev, A_scale_dev, ld_a_scale, M, K, ld_a);
    p.b[0] = pack.lay(room, W_dev, W_scale_dev, ld_w_scale, N, K, ld_w);
    p.e = e;
    ENC_TRY(pack.launch(stream));
    return launch_product(p, room, stream);
}

size_t rcd_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int dt)
{
    if (!product_sizes_ok(M, N, K) || !is_matrix_type(dt)) return 0;
    Pieces w(nullptr);
    linear_back(w, M, N, dt);
    return w.used + packed_bytes(M, K, dt) + packed_bytes(N, K, dt) + backward_parts(M, N, K, dt, 1);
}

int rcd_linear_backward(const void *dY_dev, int64_t ld_dy, const void *A_dev, int64_t ld_a, const void *W_dev, int64_t ld_w,
                        int dt, int64_t M, int64_t N, int64_t K, const float *preact_dev, int64_t ld_p, int act,
                        void *dA_dev, int64_t ld_da, void *dW_dev, int64_t ld_dw, void *dbias_dev,
                        void *workspace_dev, size_t workspace_bytes, void *stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    ENC_TRY(check_product(dt, dt, M, N, K, act));
    if (!is_matrix_type(dt)) return RCD_ERR_UNSUPPORTED;
    if (ld_dy < N || ld_a < K || ld_w < K || (act != RCD_ACT_NONE && ld_p < N) || (dA_dev && ld_da < K) || (dW_dev && ld_dw < K))
        return RCD_ERR_INVALID_ARG;
    if (M == 0) {
        ENC_TRY(zero_matrix(dW_dev, dt, ld_dw, N, K, stream));
        return zero_matrix(dbias_dev, dt, N, 1, N, stream);
    }
    if (!dY_dev || (dW_dev && !A_dev) || (dA_dev && !W_dev) || (act != RCD_ACT_NONE && !preact_dev)) return RCD_ERR_INVALID_ARG;
    ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_linear_backward_workspace_bytes(M, N, K, dt)));
    const bool f32 = dt == RCD_F32;
    Pieces room(workspace_dev);
    const LinearBack w = linear_back(room, M, N, dt);
    Packer pack{dt, dt};
    const bool in_place = f32 && enc_rules::direct_backward(M, N, K, false) && near_enough(ld_dy, up64(N));     // (no pieces)
    // dz itself, in place, where there is no activation and its rows can be read as they are
    Laid dz;
    Laid a, b;
    if (dW_dev && !in_place) a = pack.lay(room, A_dev, nullptr, 0, M, K, ld_a);
    if (dA_dev && !in_place) b = pack.lay(room, W_dev, nullptr, 0, N, K, ld_w);
    ENC_TRY(pack.launch(stream));
    const bool as_it_is = act == RCD_ACT_NONE &&
                          (in_place || (!f32 && rows_aligned(dY_dev, ld_dy, 2) && N % 8 == 0 && ld_dy * 2 <= ((int64_t)1 << 23)));
    const int64_t pitch = up64(N);
    if (as_it_is) {
        dz.p = (const unsigned char *)dY_dev;
        dz.pitch = ld_dy * 2;
        dz.cols = N;
    } else {
        dz.p = (const unsigned char *)w.dz;
        dz.pitch = pitch * 2;
        dz.plane = M * pitch * 2;
        dz.cols = pitch;
    }
    tile::Columns cols{};
    if (!as_it_is || dbias_dev) {
        const SlopeCut c = slope_cut(M, pitch);
        SlopeArgs x{};
        x.dy = dY_dev;
        x.z = preact_dev;
        x.dz = as_it_is ? nullptr : w.dz;
        x.part = dbias_dev ? w.part : nullptr;
        x.ld_dy = ld_dy; x.ld_z = ld_p; x.pitch = pitch; x.plane = M * pitch; x.part_pitch = part_pitch(N);
        x.M = (int)M; x.N = (int)N; x.across = c.across;
        const dim3 grid((unsigned)c.pieces, (unsigned)c.groups);
        with_act_value(act, [&](auto a) {
            constexpr int A = decltype(a)::value;
            if (in_place) hipLaunchKernelGGL((k_slope<float, 0, A>), grid, dim3(256), 0, stream, x);
            else if (f32) hipLaunchKernelGGL((k_slope<float, 3, A>), grid, dim3(256), 0, stream, x);
            else hipLaunchKernelGGL((k_slope<__bf16, 1, A>), grid, dim3(256), 0, stream, x);
        });
        ENC_HIP_TRY(hipGetLastError());
        if (dbias_dev) cols = tile::Columns{w.part, dbias_dev, x.part_pitch, (int)c.groups, (int)N, f32};
    }
    if (in_place) {
        DirectProduct p{}, q{};
        p.pairs = q.pairs = 1;
        p.a[0] = q.a[0] = as_it_is ? (const float *)dY_dev : (const float *)w.dz;
        p.a_pitch = q.a_pitch = as_it_is ? ld_dy : pitch;
        p.M = M; p.N = K; p.K = N;
        p.ka = tile::K_RUNS;
        p.kb = tile::ROWS_RUN;
        p.b[0] = (const float *)W_dev;
        p.b_pitch[0] = ld_w;
        p.a_extent = M;
        p.a_cols = q.a_cols = as_it_is ? N : pitch;       // (packed rows end in zeros)
        p.b_cols = q.b_cols = K;
        p.e = one_output(dA_dev, ld_da, dt, RCD_ACT_NONE);
        q.M = N; q.N = K; q.K = M;
        q.ka = q.kb = tile::ROWS_RUN;
        q.b[0] = (const float *)A_dev;
        q.b_pitch[0] = ld_a;
        q.e = one_output(dW_dev, ld_dw, dt, RCD_ACT_NONE);
        return launch_both(dA_dev ? &p : nullptr, dW_dev ? &q : nullptr, enc_rules::direct_both(M, N, K, false), room, cols, stream);
    }
    Product p{}, q{};
    p.dt = q.dt = dt;
    p.pairs = q.pairs = 1;
    p.a[0] = q.a[0] = dz;
    p.M = M; p.N = K; p.K = N;
    p.ka = tile::K_RUNS;
    p.kb = tile::ROWS_RUN;
    p.b[0] = b;
    p.e = one_output(dA_dev, ld_da, dt, RCD_ACT_NONE);
    q.M = N; q.N = K; q.K = M;
    q.ka = q.kb = tile::ROWS_RUN;
    q.b[0] = a;
    q.e = one_output(dW_dev, ld_dw, dt, RCD_ACT_NONE);
    return launch_both(dA_dev ? &p : nullptr, dW_dev ? &q : nullptr, both_of(M, N, K, dt, 1), room, cols, stream);
}

size_t rcd_gated_linear_workspace_bytes(int64_t M, int64_t F, int64_t K, int dt)
{
    if (!product_sizes_ok(M, F, K) || dt < RCD_F32 || dt > RCD_MXFP8 || few_rows(M, F, K, dt)) return 0;
    return forward_bytes(M, F, K, dt, true);
}

int rcd_gated_linear(const void *A_dev, const uint8_t *A_scale_dev, int64_t ld_a, int64_t ld_a_scale,
                     const void *Wg_dev, const uint8_t *Wg_scale_dev, int64_t ld_wg, int64_t ld_wg_scale,
                     const void *Wu_dev, const uint8_t *Wu_scale_dev, int64_t ld_wu, int64_t ld_wu_scale,
                     int dt, int out_dt, int64_t M, int64_t F, int64_t K, int act, float *saved_dev,
                     void *H_dev, int64_t ld_h, void *workspace_dev, size_t workspace_bytes, void *stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    ENC_TRY(check_product(dt, out_dt, M, F, K, act));
    if (ld_a < K || ld_wg < K || ld_wu < K || ld_h < F) return RCD_ERR_INVALID_ARG;
    if (M == 0) return RCD_OK;
    if (!A_dev || !Wg_dev || !Wu_dev || !H_dev) return RCD_ERR_INVALID_ARG;
    ENC_TRY(check_mx_operand(dt, A_scale_dev, ld_a_scale, K));
    ENC_TRY(check_mx_operand(dt, Wg_scale_dev, ld_wg_scale, K));
    ENC_TRY(check_mx_operand(dt, Wu_scale_dev, ld_wu_scale, K));
    ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_gated_linear_workspace_bytes(M, F, K, dt)));
    Epilogue e = one_output(H_dev, ld_h, out_dt, act);
    e.preact = saved_dev;
    e.ld_p = 2 * F;
    if (few_rows(M, F, K, dt)) {
        few::Args x = few_args(dt, A_dev, A_scale_dev, ld_a, ld_a_scale, M, F, K, e);
        few_weight(x, dt, false, Wg_dev, Wg_scale_dev, ld_wg, ld_wg_scale);
        few_weight(x, dt, true, Wu_dev, Wu_scale_dev, ld_wu, ld_wu_scale);
        return launch_few(dt, true, x, stream);
    }
    Pieces room(workspace_dev);
    if (dt == RCD_F32 && enc_rules::direct_forward(M, F, K, true) && near_enough(ld_a, ld_wg, ld_wu)) {
        DirectProduct p{};
        p.M = M; p.N = F; p.K = K;
        p.ka = p.kb = tile::K_RUNS;
        p.pairs = 1;
        p.gated = true;
        p.a[0] = (const float *)A_dev;
        p.b[0] = (const float *)Wg_dev;
        p.b[1] = (const float *)Wu_dev;
        p.a_pitch = ld_a;
        p.b_pitch[0] = ld_wg;
        p.b_pitch[1] = ld_wu;
        p.a_extent = M;
        p.b_extent = F;
        p.a_cols = p.b_cols = K;
        p.e = e;
        return launch_direct(p, room, stream);
    }
    Packer pack{dt, product_type(dt, K, out_dt == RCD_BF16 && !saved_dev)};
    Product p{};
    p.M = M; p.N = F; p.K = K;
    p.dt = pack.type;
    p.gated = true;
    p.pairs = 1;
    p.a[0] = pack.lay(room, A_dev, A_scale_dev, ld_a_scale, M, K, ld_a);
    ENC_TRY(lay_pair(pack, room, p.b, dt, Wg_dev, Wg_scale_dev, ld_wg, ld_wg_scale, Wu_dev, Wu_scale_dev, ld_wu, ld_wu_scale, F, K));
    p.e = e;
    ENC_TRY(pack.launch(stream));
    return launch_product(p, room, stream);
}

size_t rcd_gated_linear_backward_workspace_bytes(int64_t M, int64_t F, int64_t K, int dt)
{
    if (!product_sizes_ok(M, F, K) || !is_matrix_type(dt)) return 0;
    Pieces w(nullptr);
    w.take<__bf16>((size_t)M * 2 * up64(F) * (dt == RCD_F32 ? 3 : 1));
    return w.used + packed_bytes(M, K, dt) + 2 * packed_bytes(F, K, dt) +
           backward_parts(M, F, K, dt, 2);
}

int rcd_gated_linear_backward(const void *dH_dev, int64_t ld_dh, const void *A_dev, int64_t ld_a,
                              const void *Wg_dev, int64_t ld_wg, const void *Wu_dev, int64_t ld_wu,
                              int dt, int64_t M, int64_t F, int64_t K, const float *saved_dev, int act,
                              void *dA_dev, int64_t ld_da, void *dWg_dev, int64_t ld_dwg, void *dWu_dev, int64_t ld_dwu,
                              void *workspace_dev, size_t workspace_bytes, void *stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    ENC_TRY(check_product(dt, dt, M, F, K, act));
    if (!is_matrix_type(dt)) return RCD_ERR_UNSUPPORTED;
    if (ld_dh < F || ld_a < K || ld_wg < K || ld_wu < K || (dA_dev && ld_da < K) || (dWg_dev && ld_dwg < K) ||
        (dWu_dev && ld_dwu < K) || !dWg_dev != !dWu_dev)
        return RCD_ERR_INVALID_ARG;
    if (M == 0) {
        ENC_TRY(zero_matrix(dWg_dev, dt, ld_dwg, F, K, stream));
        return zero_matrix(dWu_dev, dt, ld_dwu, F, K, stream);
    }
    if (!dH_dev || !saved_dev || (dWg_dev && !A_dev) || (dA_dev && (!Wg_dev || !Wu_dev))) return RCD_ERR_INVALID_ARG;
    ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_gated_linear_backward_workspace_bytes(M, F, K, dt)));
    const bool f32 = dt == RCD_F32;
    const int64_t half = up64(F), pitch = 2 * half;
    Pieces room(workspace_dev);
    __bf16 *dgu = room.take<__bf16>((size_t)M * pitch * (f32 ? 3 : 1));
    const bool in_place = f32 && enc_rules::direct_backward(M, F, K, true) && near_enough(2 * up64(F));      // (no pieces)
    Packer pack{dt, dt};
    Product p{};
    p.dt = dt;
    Laid a;
    if (dWg_dev && !in_place) a = pack.lay(room, A_dev, nullptr, 0, M, K, ld_a);
    if (dA_dev && !in_place) ENC_TRY(lay_pair(pack, room, p.b, dt, Wg_dev, nullptr, ld_wg, 0, Wu_dev, nullptr, ld_wu, 0, F, K));
    ENC_TRY(pack.launch(stream));
    const SlopeCut c = slope_cut(M, half);
    SlopeArgs x{};
    x.dy = dH_dev;
    x.z = saved_dev;
    x.dz = dgu;
    x.ld_dy = ld_dh; x.ld_z = 2 * F; x.pitch = pitch; x.plane = M * pitch;
    x.M = (int)M; x.N = (int)F; x.across = c.across; x.half = (int)half;
    const dim3 grid((unsigned)c.pieces, (unsigned)c.groups);
    with_act_value(act, [&](auto a) {
        constexpr int A = decltype(a)::value;
        if (in_place) hipLaunchKernelGGL((k_gated_slope<float, 0, A>), grid, dim3(256), 0, stream, x);
        else if (f32) hipLaunchKernelGGL((k_gated_slope<float, 3, A>), grid, dim3(256), 0, stream, x);
        else hipLaunchKernelGGL((k_gated_slope<__bf16, 1, A>), grid, dim3(256), 0, stream, x);
    });
    ENC_HIP_TRY(hipGetLastError());
    Epilogue both = one_output(dWg_dev, ld_dwg, dt, RCD_ACT_NONE);       // dg's columns and du's are the rows of one product
    both.out2 = dWu_dev;
    both.ld_o2 = ld_dwu;
    both.split_row = (int)half;
    both.rows_each = (int)F;
    if (in_place) {
        DirectProduct p{}, q{};
        p.a[0] = q.a[0] = (const float *)dgu;
        p.a[1] = p.a[0] + half;
        p.a_pitch = q.a_pitch = pitch;
        p.M = M; p.N = K; p.K = F;
        p.ka = tile::K_RUNS;
        p.kb = tile::ROWS_RUN;
        p.pairs = 2;
        p.b[0] = (const float *)Wg_dev;
        p.b[1] = (const float *)Wu_dev;
        p.b_pitch[0] = ld_wg;
        p.b_pitch[1] = ld_wu;
        p.a_extent = M;
        p.a_cols = half;                                  // (packed rows end in zeros)
        p.b_cols = q.b_cols = K;
        p.e = one_output(dA_dev, ld_da, dt, RCD_ACT_NONE);
        q.M = pitch; q.N = K; q.K = M;
        q.ka = q.kb = tile::ROWS_RUN;
        q.pairs = 1;
        q.b[0] = (const float *)A_dev;
        q.b_pitch[0] = ld_a;
        q.a_cols = pitch;
        q.e = both;
        return launch_both(dA_dev ? &p : nullptr, dWg_dev ? &q : nullptr, enc_rules::direct_both(M, F, K, true), room, tile::Columns{}, stream);
    }
    Laid d;
    d.p = (const unsigned char *)dgu;
    d.pitch = pitch * 2;
    d.plane = M * pitch * 2;
    d.cols = pitch;
    p.a[0] = d;
    p.M = M; p.N = K; p.K = F;
    p.ka = tile::K_RUNS;
    p.kb = tile::ROWS_RUN;
    p.pairs = 2;
    p.a_shift = half * 2;
    p.e = one_output(dA_dev, ld_da, dt, RCD_ACT_NONE);
    Product q{};
    q.dt = dt;
    q.a[0] = d;
    q.M = pitch; q.N = K; q.K = M;
    q.ka = q.kb = tile::ROWS_RUN;
    q.pairs = 1;
    q.b[0] = a;
    q.e = both;
    return launch_both(dA_dev ? &p : nullptr, dWg_dev ? &q : nullptr, both_of(M, F, K, dt, 2), room, tile::Columns{}, stream);
}

} // extern "C"

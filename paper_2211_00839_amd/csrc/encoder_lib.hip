// Host side of the feature encoder's operators: argument checks, workspace layout, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "host_error.h"
#include "norm_kernels.hip"
#include "product_kernels.hip"

namespace {

using namespace enc;

constexpr int64_t MAX_EXTENT = 0x7fffff00;

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool is_matrix_type(int dt) { return dt == RCD_F32 || dt == RCD_BF16; }
inline int64_t size_of(int dt) { return dt == RCD_F32 ? 4 : dt == RCD_BF16 ? 2 : 1; }
inline int64_t blocks_of(int64_t d) { return (d + MX_BLOCK - 1) / MX_BLOCK; }
inline bool extent_ok(int64_t n) { return n >= 1 && n <= MAX_EXTENT; }

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

template <bool MX, bool NORM> int launch_norm(const NormArgs &a, int dt, hipStream_t stream)
{
    with_row_variant(a.d, [&](auto wpr, auto chunks) {
        constexpr int W = decltype(wpr)::value, C = decltype(chunks)::value;
        const dim3 grid((unsigned)((a.rows + RowOf<W>::ROWS - 1) / RowOf<W>::ROWS));
        if (dt == RCD_F32) hipLaunchKernelGGL((k_norm<float, W, C, MX, NORM>), grid, dim3(NORM_THREADS), 0, stream, a);
        else hipLaunchKernelGGL((k_norm<__bf16, W, C, MX, NORM>), grid, dim3(NORM_THREADS), 0, stream, a);
    });
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

// Row groups of the backward kernel, each with its own sums for the weight's gradient.
inline int64_t norm_groups(int64_t rows, int64_t d)
{
    const int64_t per = rows_per_workgroup(d);
    return std::min<int64_t>((rows + per - 1) / per, 1024) * per;
}
inline int64_t part_pitch(int64_t d) { return (d + 63) / 64 * 64; }

// ---- products -------------------------------------------------------------------------------------------------------------

int launch_product(bool gated, const Operand &a, const Operand &b, const Operand &a2, const Operand &b2, int pairs, int64_t M,
                   int64_t N, int64_t K, const Epilogue &e, hipStream_t stream)
{
    const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
    if (tiles > 0x7fffffff) return RCD_ERR_UNSUPPORTED;
    if (gated)
        hipLaunchKernelGGL(k_product<true>, dim3((unsigned)tiles), dim3(256), 0, stream, a, b, a2, b2, pairs, (int)M, (int)N, (int)K, e);
    else
        hipLaunchKernelGGL(k_product<false>, dim3((unsigned)tiles), dim3(256), 0, stream, a, b, a2, b2, pairs, (int)M, (int)N, (int)K, e);
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

int sum_columns(const float *part, int64_t pitch, int64_t groups, int64_t d, void *out, int dt, hipStream_t stream)
{
    const dim3 grid((unsigned)((d + 15) / 16));
    if (dt == RCD_F32)
        hipLaunchKernelGGL(k_column_sums<float>, grid, dim3(1024), 0, stream, part, (long long)pitch, (int)groups, (int)d, (float *)out);
    else
        hipLaunchKernelGGL(k_column_sums<__bf16>, grid, dim3(1024), 0, stream, part, (long long)pitch, (int)groups, (int)d, (__bf16 *)out);
    ENC_HIP_TRY(hipGetLastError());
    return RCD_OK;
}

constexpr int64_t SLOPE_GROUPS = 256;

struct LinearBack {
    float *dz, *part;
};
size_t linear_back_pieces(void *ws, int64_t M, int64_t N, LinearBack *p)
{
    Pieces w(ws);
    p->dz = w.take<float>((size_t)M * N);
    p->part = w.take<float>((size_t)std::min(SLOPE_GROUPS, std::max<int64_t>(M, 1)) * part_pitch(N));
    return w.used;
}
struct GatedBack {
    float *dg, *du;
};
size_t gated_back_pieces(void *ws, int64_t M, int64_t F, GatedBack *p)
{
    Pieces w(ws);
    p->dg = w.take<float>((size_t)M * F);
    p->du = w.take<float>((size_t)M * F);
    return w.used;
}

// Types and extents of a product's call.
int check_product(int dt, int out_dt, int64_t M, int64_t N, int64_t K, int act)
{
    if (dt != RCD_F32 && dt != RCD_BF16 && dt != RCD_MXFP8) return RCD_ERR_UNSUPPORTED;
    if (!is_matrix_type(out_dt) || (dt == RCD_F32 && out_dt != RCD_F32)) return RCD_ERR_UNSUPPORTED;
    if (act < RCD_ACT_NONE || act > RCD_ACT_GELU) return RCD_ERR_UNSUPPORTED;
    if (M < 0 || N < 1 || K < 1) return RCD_ERR_INVALID_ARG;
    if (M > MAX_EXTENT || N > MAX_EXTENT || K > MAX_EXTENT) return RCD_ERR_UNSUPPORTED;
    return RCD_OK;
}

int check_mx_operand(int dt, const uint8_t *scale, int64_t ld_scale, int64_t K)
{
    if (dt != RCD_MXFP8) return RCD_OK;
    return scale && ld_scale >= blocks_of(K) ? RCD_OK : RCD_ERR_INVALID_ARG;
}

} // namespace

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
    if (rows > MAX_EXTENT || d > MAX_EXTENT) return RCD_ERR_UNSUPPORTED;
    if (rows == 0) return RCD_OK;
    if (!X_dev || !Y_dev || (mx && !scale_dev)) return RCD_ERR_INVALID_ARG;
    if (sum_dev == Y_dev) return RCD_ERR_INVALID_ARG;
    const int64_t esz = size_of(dt);
    NormArgs a{};
    a.x = X_dev; a.r = residual_dev; a.w = weight_dev;
    a.sum = sum_dev; a.y = Y_dev; a.scale = scale_dev; a.rstd = rstd_dev;
    a.ld_x = ld_x; a.ld_r = ld_r; a.ld_s = ld_s; a.ld_y = ld_y; a.ld_scale = ld_scale;
    a.rows = rows; a.d = (int)d; a.eps = eps;
    a.vec = rows_aligned(X_dev, ld_x, esz) && rows_aligned(residual_dev, ld_r, esz) && rows_aligned(weight_dev, 0, esz) &&
            rows_aligned(sum_dev, ld_s, esz) && (mx ? rows_aligned(Y_dev, ld_y, 1, 8) : rows_aligned(Y_dev, ld_y, esz));
    return mx ? launch_norm<true, true>(a, dt, (hipStream_t)stream) : launch_norm<false, true>(a, dt, (hipStream_t)stream);
}

int rcd_quantize_mxfp8(const void *X_dev, int dt, int64_t rows, int64_t d, int64_t ld_x, uint8_t *Q_dev, int64_t ld_q,
                       uint8_t *scale_dev, int64_t ld_scale, void *stream)
{
    if (!is_matrix_type(dt)) return RCD_ERR_UNSUPPORTED;
    if (rows < 0 || d < 1 || ld_x < d || ld_q < d || ld_scale < blocks_of(d)) return RCD_ERR_INVALID_ARG;
    if (rows > MAX_EXTENT || d > MAX_EXTENT) return RCD_ERR_UNSUPPORTED;
    if (rows == 0) return RCD_OK;
    if (!X_dev || !Q_dev || !scale_dev) return RCD_ERR_INVALID_ARG;
    NormArgs a{};
    a.x = X_dev; a.y = Q_dev; a.scale = scale_dev;
    a.ld_x = ld_x; a.ld_y = ld_q; a.ld_scale = ld_scale;
    a.rows = rows; a.d = (int)d;
    a.vec = rows_aligned(X_dev, ld_x, size_of(dt)) && rows_aligned(Q_dev, ld_q, 1, 8);
    return launch_norm<true, false>(a, dt, (hipStream_t)stream);
}

size_t rcd_rms_norm_backward_workspace_bytes(int64_t rows, int64_t d)
{
    if (rows < 1 || !extent_ok(d)) return 0;
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
    if (rows > MAX_EXTENT || d > MAX_EXTENT) return RCD_ERR_UNSUPPORTED;
    if (rows == 0) return zero_matrix(dweight_dev, dt, d, 1, d, stream);
    if (!dY_dev || !H_dev || !rstd_dev || !dX_dev) return RCD_ERR_INVALID_ARG;
    const int64_t esz = size_of(dt), groups = norm_groups(rows, d);
    if (dweight_dev) ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_rms_norm_backward_workspace_bytes(rows, d)));
    NormBackArgs a{};
    a.dy = dY_dev; a.h = H_dev; a.w = weight_dev; a.dsum = dsum_dev; a.rstd = rstd_dev;
    a.dx = dX_dev; a.part = dweight_dev ? (float *)workspace_dev : nullptr;
    a.ld_dy = ld_dy; a.ld_h = ld_h; a.ld_ds = ld_ds; a.ld_dx = ld_dx; a.part_pitch = part_pitch(d);
    a.rows = rows; a.d = (int)d;
    a.vec = rows_aligned(dY_dev, ld_dy, esz) && rows_aligned(H_dev, ld_h, esz) && rows_aligned(weight_dev, 0, esz) &&
            rows_aligned(dsum_dev, ld_ds, esz) && rows_aligned(dX_dev, ld_dx, esz);
    with_row_variant(d, [&](auto wpr, auto chunks) {
        constexpr int W = decltype(wpr)::value, C = decltype(chunks)::value;
        const dim3 grid((unsigned)(groups / RowOf<W>::ROWS));
        if (dt == RCD_F32) hipLaunchKernelGGL((k_norm_backward<float, W, C>), grid, dim3(NORM_THREADS), 0, stream, a);
        else hipLaunchKernelGGL((k_norm_backward<__bf16, W, C>), grid, dim3(NORM_THREADS), 0, stream, a);
    });
    ENC_HIP_TRY(hipGetLastError());
    return dweight_dev ? sum_columns(a.part, a.part_pitch, groups, d, dweight_dev, dt, stream) : RCD_OK;
}

size_t rcd_linear_workspace_bytes(int64_t, int64_t, int64_t, int) { return 0; }

int rcd_linear(const void *A_dev, const uint8_t *A_scale_dev, int64_t ld_a, int64_t ld_a_scale,
               const void *W_dev, const uint8_t *W_scale_dev, int64_t ld_w, int64_t ld_w_scale, int dt, int out_dt,
               int64_t M, int64_t N, int64_t K, const void *bias_dev, int act, const void *residual_dev, int64_t ld_r,
               float *preact_dev, int64_t ld_p, void *Y_dev, int64_t ld_y,
               void *workspace_dev, size_t workspace_bytes, void *stream)
{
    ENC_TRY(check_product(dt, out_dt, M, N, K, act));
    if (ld_a < K || ld_w < K || ld_y < N || (residual_dev && ld_r < N) || (preact_dev && ld_p < N)) return RCD_ERR_INVALID_ARG;
    if (M == 0) return RCD_OK;
    if (!A_dev || !W_dev || !Y_dev) return RCD_ERR_INVALID_ARG;
    ENC_TRY(check_mx_operand(dt, A_scale_dev, ld_a_scale, K));
    ENC_TRY(check_mx_operand(dt, W_scale_dev, ld_w_scale, K));
    ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_linear_workspace_bytes(M, N, K, dt)));
    const Operand a{A_dev, A_scale_dev, ld_a, 1, ld_a_scale, dt}, b{W_dev, W_scale_dev, ld_w, 1, ld_w_scale, dt};
    const Epilogue e{bias_dev, residual_dev, preact_dev, Y_dev, ld_r, ld_p, ld_y, act, out_dt == RCD_F32};
    return launch_product(false, a, b, a, b, 1, M, N, K, e, (hipStream_t)stream);
}

size_t rcd_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, int dt)
{
    LinearBack p;
    return M >= 1 && extent_ok(N) && extent_ok(K) && is_matrix_type(dt) ? linear_back_pieces(nullptr, M, N, &p) : 0;
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
    LinearBack p;
    linear_back_pieces(workspace_dev, M, N, &p);
    const int64_t groups = std::min(SLOPE_GROUPS, M), pitch = part_pitch(N);
    const dim3 grid((unsigned)((N + 255) / 256), (unsigned)groups);
    if (dt == RCD_F32)
        hipLaunchKernelGGL(k_slope<float>, grid, dim3(256), 0, stream, (const float *)dY_dev, (long long)ld_dy, preact_dev,
                           (long long)ld_p, act, (int)M, (int)N, p.dz, p.part, (long long)pitch);
    else
        hipLaunchKernelGGL(k_slope<__bf16>, grid, dim3(256), 0, stream, (const __bf16 *)dY_dev, (long long)ld_dy, preact_dev,
                           (long long)ld_p, act, (int)M, (int)N, p.dz, p.part, (long long)pitch);
    ENC_HIP_TRY(hipGetLastError());
    if (dbias_dev) ENC_TRY(sum_columns(p.part, pitch, groups, N, dbias_dev, dt, stream));
    Epilogue e{};
    e.out_f32 = dt == RCD_F32;
    if (dA_dev) {
        e.out = dA_dev;
        e.ld_o = ld_da;
        const Operand a{p.dz, nullptr, N, 1, 0, RCD_F32}, b{W_dev, nullptr, 1, ld_w, 0, dt};
        ENC_TRY(launch_product(false, a, b, a, b, 1, M, K, N, e, stream));
    }
    if (dW_dev) {
        e.out = dW_dev;
        e.ld_o = ld_dw;
        const Operand a{p.dz, nullptr, 1, N, 0, RCD_F32}, b{A_dev, nullptr, 1, ld_a, 0, dt};
        ENC_TRY(launch_product(false, a, b, a, b, 1, N, K, M, e, stream));
    }
    return RCD_OK;
}

size_t rcd_gated_linear_workspace_bytes(int64_t, int64_t, int64_t, int) { return 0; }

int rcd_gated_linear(const void *A_dev, const uint8_t *A_scale_dev, int64_t ld_a, int64_t ld_a_scale,
                     const void *Wg_dev, const uint8_t *Wg_scale_dev, int64_t ld_wg, int64_t ld_wg_scale,
                     const void *Wu_dev, const uint8_t *Wu_scale_dev, int64_t ld_wu, int64_t ld_wu_scale,
                     int dt, int out_dt, int64_t M, int64_t F, int64_t K, int act, float *saved_dev,
                     void *H_dev, int64_t ld_h, void *workspace_dev, size_t workspace_bytes, void *stream)
{
    ENC_TRY(check_product(dt, out_dt, M, F, K, act));
    if (ld_a < K || ld_wg < K || ld_wu < K || ld_h < F) return RCD_ERR_INVALID_ARG;
    if (M == 0) return RCD_OK;
    if (!A_dev || !Wg_dev || !Wu_dev || !H_dev) return RCD_ERR_INVALID_ARG;
    ENC_TRY(check_mx_operand(dt, A_scale_dev, ld_a_scale, K));
    ENC_TRY(check_mx_operand(dt, Wg_scale_dev, ld_wg_scale, K));
    ENC_TRY(check_mx_operand(dt, Wu_scale_dev, ld_wu_scale, K));
    ENC_TRY(check_pieces(workspace_dev, workspace_bytes, rcd_gated_linear_workspace_bytes(M, F, K, dt)));
    const Operand a{A_dev, A_scale_dev, ld_a, 1, ld_a_scale, dt}, b{Wg_dev, Wg_scale_dev, ld_wg, 1, ld_wg_scale, dt},
        b2{Wu_dev, Wu_scale_dev, ld_wu, 1, ld_wu_scale, dt};
    Epilogue e{};
    e.preact = saved_dev;
    e.ld_p = 2 * F;
    e.out = H_dev;
    e.ld_o = ld_h;
    e.act = act;
    e.out_f32 = out_dt == RCD_F32;
    return launch_product(true, a, b, a, b2, 1, M, F, K, e, (hipStream_t)stream);
}

size_t rcd_gated_linear_backward_workspace_bytes(int64_t M, int64_t F, int64_t K, int dt)
{
    GatedBack p;
    return M >= 1 && extent_ok(F) && extent_ok(K) && is_matrix_type(dt) ? gated_back_pieces(nullptr, M, F, &p) : 0;
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
    GatedBack p;
    gated_back_pieces(workspace_dev, M, F, &p);
    const dim3 grid((unsigned)((F + 255) / 256), (unsigned)std::min<int64_t>(SLOPE_GROUPS, M));
    if (dt == RCD_F32)
        hipLaunchKernelGGL(k_gated_slope<float>, grid, dim3(256), 0, stream, (const float *)dH_dev, (long long)ld_dh, saved_dev, act,
                           (int)M, (int)F, p.dg, p.du);
    else
        hipLaunchKernelGGL(k_gated_slope<__bf16>, grid, dim3(256), 0, stream, (const __bf16 *)dH_dev, (long long)ld_dh, saved_dev, act,
                           (int)M, (int)F, p.dg, p.du);
    ENC_HIP_TRY(hipGetLastError());
    Epilogue e{};
    e.out_f32 = dt == RCD_F32;
    if (dA_dev) {
        e.out = dA_dev;
        e.ld_o = ld_da;
        const Operand a{p.dg, nullptr, F, 1, 0, RCD_F32}, b{Wg_dev, nullptr, 1, ld_wg, 0, dt};
        const Operand a2{p.du, nullptr, F, 1, 0, RCD_F32}, b2{Wu_dev, nullptr, 1, ld_wu, 0, dt};
        ENC_TRY(launch_product(false, a, b, a2, b2, 2, M, K, F, e, stream));
    }
    if (dWg_dev) {
        const Operand b{A_dev, nullptr, 1, ld_a, 0, dt};
        for (int i = 0; i < 2; ++i) {
            const Operand a{i ? p.du : p.dg, nullptr, 1, F, 0, RCD_F32};
            e.out = i ? dWu_dev : dWg_dev;
            e.ld_o = i ? ld_dwu : ld_dwg;
            ENC_TRY(launch_product(false, a, b, a, b, 1, F, K, M, e, stream));
        }
    }
    return RCD_OK;
}

} // extern "C"

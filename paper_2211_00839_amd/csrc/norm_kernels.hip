// Root-mean-square norm of rows with the residual's addition, its gradients, and rows in 8 bits with scales.
//
//   h = x + r,  rstd = (mean h^2 + eps)^(-1/2),  y = h rstd w
//   g = dy w, xh = h rstd:  dx = rstd (g - xh mean(g xh)) + dsum,  dw = sum over rows of dy xh
//
// All of it is a handful of operations per element: bandwidth bounds it, so a row is read once and stays in registers
// between its statistics and its outputs, eight elements (16 bytes of bf16) to a thread and access.
#pragma once
#include "encoder_math.h"

namespace enc {

constexpr int NORM_THREADS = 256;

// What a row belongs to: WPR waves (1 or 4) of the four of a workgroup; the column of this thread's chunk c is
// chunk_col(c).  C: chunks of eight that a thread holds in registers; C = 0: rows of any length, read twice.
template <int WPR> struct RowOf {
    static constexpr int ROWS = 4 / WPR, LANES = 64 * WPR;
    __device__ static int sub() { return WPR == 4 ? 0 : (int)threadIdx.x >> 6; }
    __device__ static int lane() { return WPR == 4 ? (int)threadIdx.x : (int)threadIdx.x & 63; }
};

// Sum over the lanes of a row, the same bits in every one of them; `scratch`: 4 floats of LDS that nobody else is using.
template <int WPR> __device__ __forceinline__ float row_sum(float v, float *scratch)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
    if constexpr (WPR == 4) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
    }
    return v;
}

struct NormArgs {
    const void *x, *r, *w;          // r, w nullable
    void *sum, *y;                  // sum nullable
    uint8_t *scale;
    float *rstd;                    // nullable
    long long ld_x, ld_r, ld_s, ld_y, ld_scale;
    long long first, rows;          // this launch's rows are first .. rows - 1
    int d;
    float eps;
};

// One chunk of a row in 8 bits: the four lanes of a block share their largest finite magnitude.  Every lane of a block of
// 32 has to come along (count 0 for what is past the row's end).
__device__ __forceinline__ void store_mx(const NormArgs &a, size_t row, int col, int count, const float (&v)[8])
{
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = fabsf(v[i]);
        m = f <= 3.402823466e38f ? fmaxf(m, f) : m;
    }
    m = fmaxf(m, __shfl_xor(m, 1));
    m = fmaxf(m, __shfl_xor(m, 2));
    if (count <= 0) return;
    const int e = mx_exponent(m);
    const float inv = pow2(-e);
    const unsigned lo = to_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    const unsigned hi = to_e4m3x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    uint8_t *q = (uint8_t *)a.y + row * a.ld_y + col;
    if (count >= 8) {
        typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
        *reinterpret_cast<u32x2_any *>(q) = u32x2{lo, hi};
    } else {
        for (int i = 0; i < min(count, 8); ++i) q[i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
    }
    if ((threadIdx.x & 3) == 0) a.scale[row * a.ld_scale + col / MX_BLOCK] = (uint8_t)(e + 127);
}

// One wave to a row of up to 1024 elements, four to a longer one (past 8192 it is read twice).  Bound by memory: 50 000 x 2048
// bf16 with residual and sum 135 us (819 MB, 6.1 TB/s: part of it stays in the last-level cache), 5000 x 2048 into 8 bits 14
// to 16 us (72 MB); one row of 2048 2.6 us: a launch, two waits for memory and a barrier.
// NORM = false: the rows themselves in 8 bits (no statistics).
template <typename T, int WPR, int C, bool MX, bool NORM>
__global__ void __launch_bounds__(NORM_THREADS)
k_norm(const NormArgs a)
{
    __shared__ float scratch[4];
    using R = RowOf<WPR>;
    const size_t row = (size_t)a.first + (size_t)blockIdx.x * R::ROWS + R::sub();
    if (WPR == 1 && row >= (size_t)a.rows) return;        // (a whole wave)
    const T *x = (const T *)a.x + row * a.ld_x;
    const T *r = a.r ? (const T *)a.r + row * a.ld_r : nullptr;
    const T *w = (const T *)a.w;
    T *sum = a.sum ? (T *)a.sum + row * a.ld_s : nullptr;
    constexpr int HELD = C > 0 ? C : 1;
    const int chunks = C > 0 ? C : (a.d + 8 * R::LANES - 1) / (8 * R::LANES);
    float h[HELD][8];
    auto fetch = [&](int c, float (&v)[8]) {
        const int col = (c * R::LANES + R::lane()) * 8, count = a.d - col;
        load8(x + col, count, v);
        if (r) {
            float u[8];
            load8(r + col, count, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[i];
        }
    };
    auto emit = [&](int c, const float (&v)[8], float rstd) {
        const int col = (c * R::LANES + R::lane()) * 8, count = a.d - col;
        float y[8];
        if constexpr (NORM) {
            if (sum && count > 0) store8(sum + col, count, v);
            if (w) {
                float u[8];
                load8(w + col, count, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = v[i] * rstd * u[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = v[i] * rstd;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[i];
        }
        if constexpr (MX) store_mx(a, row, col, count, y);
        else if (count > 0) store8((T *)a.y + row * a.ld_y + col, count, y);
    };
    float rstd = 1.f;
    if constexpr (NORM || C > 0) {
        float ss = 0.f;
        if constexpr (C > 0) {
#pragma unroll
            for (int c = 0; c < C; ++c) fetch(c, h[c]);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(h[c][i], h[c][i], ss);
        } else {
            for (int c = 0; c < chunks; ++c) {
                fetch(c, h[0]);
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(h[0][i], h[0][i], ss);
            }
        }
        if constexpr (NORM) {
            rstd = 1.f / sqrtf(row_sum<WPR>(ss, scratch) / (float)a.d + a.eps);
            if (a.rstd && R::lane() == 0) a.rstd[row] = rstd;
        }
    }
    if constexpr (C > 0) {
#pragma unroll
        for (int c = 0; c < C; ++c) emit(c, h[c], rstd);
    } else {
        for (int c = 0; c < chunks; ++c) {
            fetch(c, h[0]);
            emit(c, h[0], rstd);
        }
    }
}

struct NormBackArgs {
    const void *dy, *h, *w, *dsum;  // w, dsum nullable
    const float *rstd;
    void *dx;
    float *part;                    // [groups][part_pitch] sums of dy xh over the rows of a group (nullable)
    long long ld_dy, ld_h, ld_ds, ld_dx, part_pitch;
    long long rows;
    int d;
};

// A group of WPR waves walks the rows group, group + groups, ...: its sums of dy xh stay in registers from row to row
// (C = 0: in its row of `part`).  Bound by memory: 50 000 x 2048 bf16 161 us (819 MB, 5.1 TB/s).  Adding to dw with atomics would
// need no second launch, but its bits would change from run to run.
template <typename T, int WPR, int C>
__global__ void __launch_bounds__(NORM_THREADS)
k_norm_backward(const NormBackArgs a)
{
    __shared__ float scratch[4];
    using R = RowOf<WPR>;
    const int group = blockIdx.x * R::ROWS + R::sub(), groups = gridDim.x * R::ROWS;
    constexpr int HELD = C > 0 ? C : 1;
    const int chunks = C > 0 ? C : (a.d + 8 * R::LANES - 1) / (8 * R::LANES);
    float dw[HELD][8];
#pragma unroll
    for (int c = 0; c < HELD; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = 0.f;
    float *part = a.part ? a.part + (size_t)group * a.part_pitch : nullptr;
    const T *w = (const T *)a.w;
    const float inv_d = 1.f / (float)a.d;
    // g, xh of chunk c, and the chunk's share of sum g xh
    auto fetch = [&](size_t row, int c, float rstd, float (&g)[8], float (&xh)[8], float (&dwc)[8], bool add) {
        const int col = (c * R::LANES + R::lane()) * 8, count = a.d - col;
        load8((const T *)a.dy + row * a.ld_dy + col, count, g);
        load8((const T *)a.h + row * a.ld_h + col, count, xh);
#pragma unroll
        for (int i = 0; i < 8; ++i) xh[i] *= rstd;
        if (add) {
#pragma unroll
            for (int i = 0; i < 8; ++i) dwc[i] = fmaf(g[i], xh[i], dwc[i]);
        }
        if (w) {
            float u[8];
            load8(w + col, count, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] *= u[i];
        }
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(g[i], xh[i], s);
        return s;
    };
    auto emit = [&](size_t row, int c, float rstd, float mean, const float (&g)[8], const float (&xh)[8]) {
        const int col = (c * R::LANES + R::lane()) * 8, count = a.d - col;
        if (count <= 0) return;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = rstd * fmaf(-xh[i], mean, g[i]);
        if (a.dsum) {
            float u[8];
            load8((const T *)a.dsum + row * a.ld_ds + col, count, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[i];
        }
        store8((T *)a.dx + row * a.ld_dx + col, count, v);
    };
    for (long long row = group; row < a.rows; row += groups) {
        const float rstd = a.rstd[row];
        float g[HELD][8], xh[HELD][8], s = 0.f;
        if constexpr (C > 0) {
#pragma unroll
            for (int c = 0; c < C; ++c) s += fetch(row, c, rstd, g[c], xh[c], dw[c], true);
        } else {
            for (int c = 0; c < chunks; ++c) {
                const int col = (c * R::LANES + R::lane()) * 8;
                if (part && col < a.d) {       // (part_pitch is a multiple of 8: whole chunks)
                    if (row != group) load8(part + col, 8, dw[0]);
                    else
#pragma unroll
                        for (int i = 0; i < 8; ++i) dw[0][i] = 0.f;
                }
                s += fetch(row, c, rstd, g[0], xh[0], dw[0], true);
                if (part && col < a.d) store8(part + col, 8, dw[0]);
            }
        }
        const float mean = row_sum<WPR>(s, scratch) * inv_d;
        if constexpr (C > 0) {
#pragma unroll
            for (int c = 0; c < C; ++c) emit(row, c, rstd, mean, g[c], xh[c]);
        } else {
            for (int c = 0; c < chunks; ++c) {
                fetch(row, c, rstd, g[0], xh[0], dw[0], false);
                emit(row, c, rstd, mean, g[0], xh[0]);
            }
        }
    }
    if constexpr (C > 0) {
        if (part) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * R::LANES + R::lane()) * 8;
                if (col < a.d) store8(part + col, 8, dw[c]);
            }
        }
    }
}

// out[c] = sum over the first `groups` rows of part, in a fixed order: 16 columns to a workgroup of 16 DOWN threads, DOWN
// rows side by side.
template <typename T, int DOWN>
__device__ __forceinline__ void column_sums(const float *__restrict__ part, long long pitch, int groups, int d, T *__restrict__ out,
                                            int block, float (&sums)[DOWN][17])
{
    const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int col = block * 16 + c;
    float s = 0.f;
    if (col < d) {
#pragma unroll 4
        for (int g = r; g < groups; g += DOWN) s += part[(size_t)g * pitch + col];
    }
    sums[r][c] = s;
    __syncthreads();
    for (int half = DOWN / 2; half >= 1; half >>= 1) {
        if (r < half) sums[r][c] += sums[r + half][c];
        __syncthreads();
    }
    if (r == 0 && col < d) out[col] = (T)sums[0][c];
}

// grid = ceil(d / 16).  Latency: 2048 columns of 2048 groups 8 us
template <typename T>
__global__ void __launch_bounds__(1024)
k_column_sums(const float *__restrict__ part, long long pitch, int groups, int d, T *__restrict__ out)
{
    __shared__ float sums[64][17];
    column_sums<T, 64>(part, pitch, groups, d, out, (int)blockIdx.x, sums);
}

} // namespace enc

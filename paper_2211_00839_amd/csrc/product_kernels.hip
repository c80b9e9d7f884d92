// Matrix products of the feature encoder with what goes before and after them.
#include "encoder_math.h"

namespace enc {

// Element (row, k) of an operand lies at p + row * rs + k * ks (elements of its type).
struct Operand {
    const void *p;
    const uint8_t *scale;           // RCD_MXFP8: one byte for 32 elements of a row
    long long rs, ks, ld_scale;
    int dt;                         // rcd_dtype
};

__device__ __forceinline__ float element(const Operand &o, long long row, long long k)
{
    const long long at = row * o.rs + k * o.ks;
    if (o.dt == 0) return ((const float *)o.p)[at];
    if (o.dt == 1) return (float)((const __bf16 *)o.p)[at];
    const int s = o.scale[row * o.ld_scale + k / MX_BLOCK];
    const float v = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)o.p)[at], 0);
    return s == 255 ? __builtin_nanf("") : v * ldexpf(1.f, s - 127);
}

// What becomes of a product's sums.  act(z + bias) + residual, or the gated block's act(g) * u.
struct Epilogue {
    const void *bias, *residual;    // of the output's type, nullable
    float *preact;                  // z in fp32 (gated: g and u side by side), nullable
    void *out;
    long long ld_r, ld_p, ld_o;
    int act;
    bool out_f32;
};

__device__ __forceinline__ float read_as(const void *p, long long at, bool f32)
{
    return f32 ? ((const float *)p)[at] : (float)((const __bf16 *)p)[at];
}
__device__ __forceinline__ void write_as(void *p, long long at, bool f32, float v)
{
    if (f32) ((float *)p)[at] = v;
    else ((__bf16 *)p)[at] = (__bf16)v;
}

__device__ __forceinline__ void finish_linear(const Epilogue &e, long long m, long long n, float z)
{
    if (e.bias) z += read_as(e.bias, n, e.out_f32);
    if (e.preact) e.preact[m * e.ld_p + n] = z;
    float y = activate(z, e.act);
    if (e.residual) y += read_as(e.residual, m * e.ld_r + n, e.out_f32);
    write_as(e.out, m * e.ld_o + n, e.out_f32, y);
}

__device__ __forceinline__ void finish_gated(const Epilogue &e, long long m, long long f, float g, float u)
{
    if (e.preact) {
        e.preact[m * e.ld_p + 2 * f] = g;
        e.preact[m * e.ld_p + 2 * f + 1] = u;
    }
    write_as(e.out, m * e.ld_o + f, e.out_f32, activate(g, e.act) * u);
}

// sum over k of a(m, k) b(n, k), plus the same of a2 and b2 where there are two pairs; GATED: the sums with b and with b2
// apart.  One 64 x 64 tile per workgroup, 4 x 4 sums per thread.
template <bool GATED>
__global__ void __launch_bounds__(256)
k_product(const Operand a, const Operand b, const Operand a2, const Operand b2, int pairs, int M, int N, int K, const Epilogue e)
{
    __shared__ float sa[16][65], sb[GATED ? 2 : 1][16][65];
    const int tn = (N + 63) / 64;
    const long long m0 = (long long)(blockIdx.x / tn) * 64, n0 = (long long)(blockIdx.x % tn) * 64;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    float acc[GATED ? 2 : 1][4][4] = {};
    for (int pair = 0; pair < (GATED ? 1 : pairs); ++pair) {
        const Operand &pa = pair ? a2 : a, &pb = pair ? b2 : b;
        for (int k0 = 0; k0 < K; k0 += 16) {
            for (int i = tid; i < 64 * 16; i += 256) {
                const int k = i & 15, r = i >> 4;
                const bool ink = k0 + k < K;
                sa[k][r] = ink && m0 + r < M ? element(pa, m0 + r, k0 + k) : 0.f;
                sb[0][k][r] = ink && n0 + r < N ? element(pb, n0 + r, k0 + k) : 0.f;
                if constexpr (GATED) sb[1][k][r] = ink && n0 + r < N ? element(b2, n0 + r, k0 + k) : 0.f;
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 16; ++k)
#pragma unroll
                for (int s = 0; s < (GATED ? 2 : 1); ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            acc[s][i][j] = fmaf(sa[k][ty * 4 + i], sb[s][k][tx + 16 * j], acc[s][i][j]);
            __syncthreads();
        }
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const long long m = m0 + ty * 4 + i, n = n0 + tx + 16 * j;
            if (m >= M || n >= N) continue;
            if constexpr (GATED) finish_gated(e, m, n, acc[0][i][j], acc[1][i][j]);
            else finish_linear(e, m, n, acc[0][i][j]);
        }
}

// dz = dy act'(z) of a group of rows and the group's column sums of it.  A thread owns a column; grid = (ceil(N / 256), groups).
template <typename T>
__global__ void __launch_bounds__(256)
k_slope(const T *__restrict__ dy, long long ld_dy, const float *__restrict__ z, long long ld_z, int act, int M, int N,
        float *__restrict__ dz, float *__restrict__ part, long long part_pitch)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    float sum = 0.f;
    for (long long m = blockIdx.y; m < M; m += gridDim.y) {
        float v = to_f32(dy[m * ld_dy + n]);
        if (act != 0) {
            float value, slope;
            activate_both(z[m * ld_z + n], act, &value, &slope);
            v *= slope;
        }
        sum += v;
        dz[m * N + n] = v;
    }
    if (part) part[(size_t)blockIdx.y * part_pitch + n] = sum;
}

// dg = dh u act'(g), du = dh act(g).
template <typename T>
__global__ void __launch_bounds__(256)
k_gated_slope(const T *__restrict__ dh, long long ld_dh, const float *__restrict__ saved, int act, int M, int F,
              float *__restrict__ dg, float *__restrict__ du)
{
    const int f = blockIdx.x * 256 + threadIdx.x;
    if (f >= F) return;
    for (long long m = blockIdx.y; m < M; m += gridDim.y) {
        const float g = saved[2 * (m * F + f)], u = saved[2 * (m * F + f) + 1], d = to_f32(dh[m * ld_dh + f]);
        float value, slope;
        activate_both(g, act, &value, &slope);
        dg[m * F + f] = d * u * slope;
        du[m * F + f] = d * value;
    }
}

// Zeros where there is no row to sum over.
template <typename T>
__global__ void __launch_bounds__(256)
k_zero(T *__restrict__ p, long long ld, int rows, int cols)
{
    for (long long i = blockIdx.x; i < rows; i += gridDim.x)
        for (int c = threadIdx.x; c < cols; c += 256) p[i * ld + c] = (T)0.f;
}

} // namespace enc

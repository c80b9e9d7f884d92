// Products of few rows (single samples and small batches): the weights are all there is to read, so each is read once,
// straight into registers, by as many waves as there are.
#include "encoder_math.h"

namespace enc {
namespace few {

struct Args {
    const unsigned char *a, *b, *b2;            // b2: the gated block's second weight
    const uint8_t *sa, *sb, *sb2;
    long long a_pitch, b_pitch, b2_pitch;       // bytes
    long long sa_pitch, sb_pitch, sb2_pitch;
    Epilogue e;
    int M, N, K;
};

// 16 bytes of a row from byte `at` on; what lies past `bytes` is zero.
__device__ __forceinline__ uint4 chunk(const unsigned char *row, int at, int bytes)
{
    if (at + 16 <= bytes) {
        const u32x4_any t = *reinterpret_cast<const u32x4_any *>(row + at);
        return make_uint4(t[0], t[1], t[2], t[3]);
    }
    unsigned w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (at + i < bytes) w[i >> 2] |= (unsigned)row[at + i] << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void widen(const uint4 (&c)[2], float s0, float s1, bf16x8 (&out)[4])
{
    out[0] = widen8(c[0].x, c[0].y, s0);
    out[1] = widen8(c[0].z, c[0].w, s0);
    out[2] = widen8(c[1].x, c[1].y, s1);
    out[3] = widen8(c[1].z, c[1].w, s1);
}

// Sums of 16 columns and up to 16 MT rows on 16 x 16 MFMA blocks, bf16 or 8 bits (widened to bf16 in registers, which is
// exact and costs nothing beside the weights' way from memory).  The waves of a workgroup take the
// chunks of 128 bytes of k in turn and add up their sums through LDS, wave by wave.  Bound by the weights' reading: 8 rows, twice 8192 x 2048
// bf16 15.8 us (67 MB, 4.2 TB/s); one row, 2048 x 2048 6.3 us (8.4 MB: 128 workgroups of sixteen waves, whose start, one wait for memory, sum and
// epilogue are most of it).
template <int MT, int WAVES, bool MX, bool GATED>
__global__ void __launch_bounds__(64 * WAVES)
k_few(const Args x)
{
    constexpr int G = GATED ? 2 : 1;
    __shared__ float sums[WAVES][G][MT * 16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
    const int n0 = blockIdx.x * 16, n = min(n0 + (lane & 15), x.N - 1);
    const int bytes = x.K * (MX ? 1 : 2), chunks = (bytes + 127) / 128;
    const unsigned char *b[G], *a[MT];
    const uint8_t *sb[G], *sa[MT];
    b[0] = x.b + n * x.b_pitch;
    if constexpr (MX) sb[0] = x.sb + n * x.sb_pitch;
    if constexpr (GATED) {
        b[1] = x.b2 + n * x.b2_pitch;
        if constexpr (MX) sb[1] = x.sb2 + n * x.sb2_pitch;
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = min(t * 16 + (lane & 15), x.M - 1);
        a[t] = x.a + m * x.a_pitch;
        if constexpr (MX) sa[t] = x.sa + m * x.sa_pitch;
    }
    f32x4 acc[G][MT];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[g][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // what the epilogue needs from memory is asked for ahead of the sums: eight columns of a row to a thread
    static_assert(2 * 16 * MT <= 64 * WAVES, "a thread for every eight columns");
    const int em = threadIdx.x >> 1, ecol = n0 + (threadIdx.x & 1) * 8, ecount = em < x.M ? x.N - ecol : 0;
    float bias[8], residual[8];
    if constexpr (!GATED) {
        bias8(x.e, ecol, ecount, bias);
        residual8(x.e, em, ecol, ecount, residual);
    }
    const int blocks = (x.K + MX_BLOCK - 1) / MX_BLOCK;
#pragma unroll 4
    for (int c = wave; c < chunks; c += WAVES) {
        // lane group q: bytes 16 q .. of the chunk's first and of its second 64
        const int at = c * 128 + q * 16;
        uint4 w[G][2], v[MT][2];
        int ws[G][2], vs[MT][2];      // (16 k lie in one scale block)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            w[g][0] = chunk(b[g], at, bytes);
            w[g][1] = chunk(b[g], at + 64, bytes);
            if constexpr (MX)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = c * 4 + 2 * h + (q >> 1);
                    ws[g][h] = k < blocks ? sb[g][k] : 127;
                }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            v[t][0] = chunk(a[t], at, bytes);
            v[t][1] = chunk(a[t], at + 64, bytes);
            if constexpr (MX)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = c * 4 + 2 * h + (q >> 1);
                    vs[t][h] = k < blocks ? sa[t][k] : 127;
                }
        }
        if constexpr (MX) {
            bf16x8 vw[MT][4];
#pragma unroll
            for (int t = 0; t < MT; ++t) widen(v[t], mx_scale(vs[t][0]), mx_scale(vs[t][1]), vw[t]);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                bf16x8 ww[4];
                widen(w[g], mx_scale(ws[g][0]), mx_scale(ws[g][1]), ww);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        acc[g][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ww[h], vw[t][h], acc[g][t], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        acc[g][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[g][h]),
                                                                            __builtin_bit_cast(bf16x8, v[t][h]), acc[g][t], 0, 0, 0);
        }
    }
    // a lane holds row lane & 15 of each block, columns 4 q ..
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[wave][g][t * 16 + (lane & 15)][q * 4 + i] = acc[g][t][i];
    __syncthreads();
    if (ecount <= 0) return;
    float z[G][8];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = (threadIdx.x & 1) * 8 + i;
            float s = sums[0][g][em][c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += sums[w][g][em][c];
            z[g][i] = s;
        }
    if constexpr (GATED) finish_gated8(x.e, em, ecol, ecount, z[0], z[1]);
    else finish_ahead8(x.e, em, ecol, ecount, z[0], bias, residual);
}

// Sums over the 64 lanes of LEFT values each: at each step a lane keeps half of its values and sends the others to the lane
// that keeps those, so all of them take about as many shuffles as there are values, not six times as many.  A lane ends
// with the whole sum number `mine` in v[0]; of the lanes that hold the same one, one is the `first`.
template <int LEFT, int OFF, int N>
__device__ __forceinline__ void spread_sums(float (&v)[N], int lane, int &mine, bool &first)
{
    if constexpr (OFF >= 1) {
        const bool up = (lane & OFF) != 0;
        if constexpr (LEFT > 1) {
            constexpr int HALF = LEFT / 2;
#pragma unroll
            for (int i = 0; i < HALF; ++i) {
                const float keep = up ? v[i + HALF] : v[i], send = up ? v[i] : v[i + HALF];
                v[i] = keep + __shfl_xor(send, OFF);
            }
            mine += up ? HALF : 0;
            spread_sums<HALF, OFF / 2>(v, lane, mine, first);
        } else {
            v[0] += __shfl_xor(v[0], OFF);
            first = first && !up;
            spread_sums<1, OFF / 2>(v, lane, mine, first);
        }
    }
}

// fp32: 8 columns to a workgroup, MR rows, plain multiply-adds (fp32 matrix instructions have no more).  Each of four waves
// takes 256 of every 1024 k; grid = (ceil(N / 8), ceil(M / MR)).  16 rows: 2048 x 2048 7.7 us (16.8 MB of weights, twice through the caches).
template <int MR, bool GATED>
__global__ void __launch_bounds__(256)
k_few_f32(const Args x)
{
    constexpr int G = GATED ? 2 : 1, COLS = 8 / G;
    constexpr int SUMS = 8 * MR;
    __shared__ float sums[4][SUMS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = blockIdx.x * COLS, m0 = blockIdx.y * MR;
    const float *b[8], *a[MR];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int n = min(n0 + j % COLS, x.N - 1);
        b[j] = j < COLS ? reinterpret_cast<const float *>(x.b + n * x.b_pitch) : reinterpret_cast<const float *>(x.b2 + n * x.b2_pitch);
    }
#pragma unroll
    for (int i = 0; i < MR; ++i) a[i] = reinterpret_cast<const float *>(x.a + min(m0 + i, x.M - 1) * x.a_pitch);
    float acc[8][MR];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < MR; ++i) acc[j][i] = 0.f;
    auto four = [&](const float *p, int k) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (k + 4 <= x.K) return (f32x4)*reinterpret_cast<const f32x4_any *>(p + k);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k + e < x.K) v[e] = p[k + e];
        return v;
    };
    for (int k = (wave * 64 + lane) * 4; k < x.K; k += 1024) {
        f32x4 w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = four(b[j], k);
#pragma unroll
        for (int i = 0; i < MR; ++i) {
            const f32x4 v = four(a[i], k);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][i] = fmaf(w[j][e], v[e], acc[j][i]);
        }
    }
    float v[SUMS];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < MR; ++i) v[i * 8 + j] = acc[j][i];
    int mine = 0;
    bool first = true;
    spread_sums<SUMS, 32>(v, lane, mine, first);
    if (first) sums[wave][mine] = v[0];
    __syncthreads();
    const int i = threadIdx.x, m = m0 + i, count = x.N - n0;
    if (i >= MR || m >= x.M) return;
    float z[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = ((sums[0][i * 8 + j] + sums[1][i * 8 + j]) + sums[2][i * 8 + j]) + sums[3][i * 8 + j];
    if constexpr (GATED) {
        float g[8], u[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            g[j] = z[j];
            u[j] = z[4 + j];
            g[4 + j] = u[4 + j] = 0.f;
        }
        finish_gated8(x.e, m, n0, min(count, 4), g, u);
    } else {
        finish_linear8(x.e, m, n0, count, z);
    }
}

} // namespace few
} // namespace enc

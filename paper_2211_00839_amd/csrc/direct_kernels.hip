// fp32 products too small to pay for their operands' pieces: the operands go to the fp32 matrix instruction as they are,
// in one launch.
//
// That instruction multiplies at a sixteenth of bf16's rate, against six products of pieces; but the pieces are a launch and a
// trip through memory of their own, and what is left of a small product's time is launches.  A workgroup of four waves (2 x 2)
// computes 64 x 64 sums (gated: 64 rows of 64 columns of both products), each wave 32 x 32 as one MFMA block (two).  k
// advances 32 at a time; a stage goes from memory into LDS 16 bytes a lane or, where rows do not lie so, 4 (any alignment and any
// length will do), three stages ahead of its multiplies (gated two), which take less time than a load.
#include "product_kernels.hip"

namespace enc {
namespace direct {

constexpr int KS = 32;                      // k of a stage
constexpr int SIDE = 64 * KS;               // floats of one operand and stage
constexpr int LDS_FLOATS = 9 * SIDE;        // three stages of three operands, or four of two

struct Args {
    tile::Args t;                           // epilogue, sizes, cut, parts (its sides and segments are not used)
    const float *a[2], *b[2];               // per pair of a summed product; gated: b[1] is the second weight
    long long a_pitch, b_pitch[2];          // from row to row (k contiguous) or from k to k (rows contiguous)
    int a_extent, b_extent;                 // rows of either side that may be read
    int pairs, K;
};

// One operand's way into LDS.  Each wave brings a quarter of a stage, with eight loads of 64 elements or (WIDE: rows that lie
// 16 bytes apart, lengths that are multiples of four) two of 256.
// k contiguous: rows of 32 floats, the four of k / 4 = c of row r at place c ^ (r & 7) (spreads what one pass of a
// ds_read_b128 touches over the banks).  Rows contiguous: lines of 64 rows, turned by 32 where k has bit 2 set (the two
// halves of a wave read lines four apart).
template <int KIND, bool WIDE> struct Feed {
    static constexpr int LOADS = WIDE ? 2 : 8, LANE = WIDE ? 4 : 1;     // loads of a wave and stage, elements of a lane
    static constexpr int ROWS = 2 * LANE;       // K_RUNS: rows of a load.  ROWS_RUN: LANE lines
    unsigned row_off[KIND == tile::K_RUNS ? LOADS : 2];     // byte offsets: of a load's row, or of this lane's rows in straight and turned lines
    unsigned kpos[LOADS];                       // K_RUNS: place in k
    const float *p;
    long long pitch;

    __device__ __forceinline__ void init(const float *p_, long long pitch_, int row0, int extent, int wave, int lane)
    {
        pitch = pitch_;
        constexpr int ACROSS = 32 / LANE;       // lanes side by side in a row's 32 k
        if constexpr (KIND == tile::K_RUNS) {
            p = p_ + row0 * pitch;
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int r = wave * 16 + u * ROWS + lane / ACROSS, at = lane % ACROSS * LANE;
                row_off[u] = (unsigned)((min(row0 + r, extent - 1) - row0) * pitch * 4);
                kpos[u] = (((at >> 2) ^ (r & 7)) << 2) | (at & 3);
            }
        } else {
            p = p_ + row0;
            const int at = lane % (64 / LANE) * LANE;
            row_off[0] = (unsigned)(min(row0 + at, extent - LANE) - row0) * 4;
            row_off[1] = (unsigned)(min(row0 + (at ^ 32), extent - LANE) - row0) * 4;
        }
    }
    // The stage from k0 on; from `there` k on there is nothing, what lies past them in LDS is some element of them.
    __device__ __forceinline__ void load(const float *from, int k0, int there, int wave, int lane, unsigned lds)
    {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const unsigned to = lds + (wave * LOADS + u) * (256 * LANE);
            if constexpr (KIND == tile::K_RUNS) {
                // (WIDE: the four k of the last one that there is)
                const unsigned k = min(kpos[u], (unsigned)(there - 1) & ~(unsigned)(LANE - 1));
                send(from + k0, row_off[u] + k * 4, to);
            } else if constexpr (WIDE) {
                const int k = wave * 8 + u * 4 + lane / 16;         // (bit 2 of k is u)
                send(from + (long long)k0 * pitch, row_off[u] + (unsigned)(min(k, there - 1) * pitch * 4), to);
            } else {
                const int k = wave * 8 + u;
                send(from + (long long)(k0 + min(k, there - 1)) * pitch, row_off[(k >> 2) & 1], to);
            }
        }
    }
    static __device__ __forceinline__ void send(const float *from, unsigned offset, unsigned to)
    {
        if constexpr (WIDE) tile::load16_to_lds(from, offset, to);
        else tile::load4_to_lds(from, offset, to);
    }
};

// Four k (k8 + 4 half + 0 .. 3) of this lane's row of a wave's block.  side: the operand's stage.
template <int KIND> __device__ __forceinline__ f32x4 four(const float *side, int row, int half, int k8)
{
    if constexpr (KIND == tile::K_RUNS) {
        return *reinterpret_cast<const f32x4 *>(side + row * KS + (((k8 >> 2) + half) ^ (row & 7)) * 4);
    } else {
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = side[(k8 + half * 4 + e) * 64 + (row ^ (half * 32))];
        return v;
    }
}

template <int KA, int KB, int TO, bool WIDE>
__device__ __forceinline__ void direct_body(const Args &x, int wg, int nwg, float *lds)
{
    constexpr bool GATED = TO == tile::TO_GATED || TO == tile::TO_GATED_PARTS;
    constexpr int G = GATED ? 2 : 1, DEPTH = GATED ? 3 : 4, LOADS = (WIDE ? 2 : 8) * (1 + G);
    constexpr int STAGE = (1 + G) * SIDE;
    using Out = tile::Band<GATED ? 64 : 32, GATED>;
    static_assert(DEPTH * STAGE <= LDS_FLOATS && 4 * 32 * Out::PITCH <= DEPTH * STAGE, "the waves' turn-round regions fit where the stages were");
    int ti, tj, split;
    if (!tile::tile_of_workgroup(wg, nwg, x.t.tiles_m, x.t.tiles_n, x.t.splits, &ti, &tj, &split)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave >> 1, wc = wave & 1;
    const int m0 = ti * 64, n0 = tj * 64;
    const int per = (x.K + KS - 1) / KS, all = per * x.pairs;
    const int s0 = (int)((long long)all * split / x.t.splits), s1 = (int)((long long)all * (split + 1) / x.t.splits);
    f32x16 acc[G];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[g][r] = 0.f;
    Feed<KA, WIDE> fa;
    Feed<KB, WIDE> fb[G];
    fa.init(x.a[0], x.a_pitch, m0, x.a_extent, wave, lane);
#pragma unroll
    for (int g = 0; g < G; ++g) fb[g].init(x.b[g], x.b_pitch[g], n0, x.b_extent, wave, lane);
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) float *)lds;
    auto there = [&](int s) { return min(KS, x.K - (s >= per ? s - per : s) * KS); };       // k of stage s
    auto fetch = [&](int s) {
        const bool second = s >= per;
        const int k0 = (second ? s - per : s) * KS;
        const unsigned to = lds_base + (unsigned)((s - s0) % DEPTH) * (STAGE * 4);
        fa.load(second ? fa.p + (x.a[1] - x.a[0]) : fa.p, k0, there(s), wave, lane, to);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (!GATED && second) {
                // (the second pair's b may have a pitch of its own)
                Feed<KB, WIDE> other;
                other.init(x.b[1], x.b_pitch[1], n0, x.b_extent, wave, lane);
                other.load(other.p, k0, there(s), wave, lane, to + (1 + g) * (SIDE * 4));
            } else {
                fb[g].load(fb[g].p, k0, there(s), wave, lane, to + (1 + g) * (SIDE * 4));
            }
        }
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i)
        if (s0 + i < s1) fetch(s0 + i);
    const int half = lane >> 5, ra = wr * 32 + (lane & 31), rb = wc * 32 + (lane & 31);
    for (int s = s0; s < s1; ++s) {
        // stage s is there, in every wave, and nobody reads stage s - 1 any more
        if (s + DEPTH - 2 < s1) tile::wait_loads<(DEPTH - 2) * LOADS>();
        else tile::wait_loads<0>();
        tile::wait_lds();
        tile::meet();
        if (s + DEPTH - 1 < s1) fetch(s + DEPTH - 1);
        const float *stage = lds + ((s - s0) % DEPTH) * STAGE;
        const int mine = there(s) - half * 4;
        // lanes 0-31 carry k = 0 .. 3 of each eight, lanes 32-63 k = 4 .. 7, for both operands alike.  The whole stage is read
        // ahead of its multiplies
        f32x4 a[KS / 8], b[G][KS / 8];
#pragma unroll
        for (int k = 0; k < KS / 8; ++k) {
            a[k] = four<KA>(stage, ra, half, k * 8);
#pragma unroll
            for (int g = 0; g < G; ++g) b[g][k] = four<KB>(stage + (1 + g) * SIDE, rb, half, k * 8);
        }
        tile::pin();
#pragma unroll
        for (int k = 0; k < KS / 8; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool there = k * 8 + e < mine;
                const float x = there ? a[k][e] : 0.f;
#pragma unroll
                for (int g = 0; g < G; ++g)
                    acc[g] = __builtin_amdgcn_mfma_f32_32x32x2f32(there ? b[g][k][e] : 0.f, x, acc[g], 0, 0, 0);
            }
    }
    tile::wait_lds();
    tile::meet();
    Out band;
    band.turn = lds + wave * (32 * Out::PITCH);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<f32x4 *>(band.turn + (lane & 31) * Out::PITCH + g * 32 + q * 8 + (lane >> 5) * 4) =
                f32x4{acc[g][4 * q], acc[g][4 * q + 1], acc[g][4 * q + 2], acc[g][4 * q + 3]};
    const int m = m0 + wr * 32, n = n0 + wc * 32;
    if constexpr (TO == tile::TO_PARTS || TO == tile::TO_GATED_PARTS) {
        band.parts(x.t, split, m, n);
    } else if (m0 + 64 <= x.t.M && n0 + 64 <= x.t.N && x.t.e.split_row == 0x7fffffff) {
        band.fetch_residual(x.t.e, m, n);
        band.inside(x.t.e, m, n, -1);
    } else {
        band.checked(x.t, m, n);
    }
}

// Bound by the wait from stage to stage where workgroups are few, by the fp32 instruction where they are many: 999 x 511 x 300 12.2 us
// (15.2 with bias, relu, residual and z), 2048 x 1024 x 640 31.9 us (84 TFLOP/s, 56 % of a large library product).  Loads of 4 bytes take a tenth
// more.
template <int KA, int KB, int TO, bool WIDE>
__global__ void __launch_bounds__(256)
k_direct(const Args x)
{
    __shared__ __attribute__((aligned(16))) float lds[LDS_FLOATS];
    direct_body<KA, KB, TO, WIDE>(x, (int)blockIdx.x, (int)gridDim.x, lds);
}

// A backward call's two products side by side: x's workgroups are the first `first` (a multiple of 8) of the launch.  999 x 511 x 300
// 29.8 us the call, by pieces 33.8.
template <bool WIDE>
__global__ void __launch_bounds__(256)
k_direct_both(const Args x, const Args y, int first)
{
    using namespace tile;
    __shared__ __attribute__((aligned(16))) float lds[LDS_FLOATS];
    const int wg = (int)blockIdx.x;
    if (wg < first) {
        if (x.t.splits > 1) direct_body<K_RUNS, ROWS_RUN, TO_PARTS, WIDE>(x, wg, first, lds);
        else direct_body<K_RUNS, ROWS_RUN, TO_LINEAR, WIDE>(x, wg, first, lds);
    } else {
        if (y.t.splits > 1) direct_body<ROWS_RUN, ROWS_RUN, TO_PARTS, WIDE>(y, wg - first, (int)gridDim.x - first, lds);
        else direct_body<ROWS_RUN, ROWS_RUN, TO_LINEAR, WIDE>(y, wg - first, (int)gridDim.x - first, lds);
    }
}

} // namespace direct
} // namespace enc

// Matrix products of the feature encoder with what goes before and after them:
//
//   C(m, n) = sum over k of a(m, k) b(n, k)
//
// on the matrix cores, for operands whose k is contiguous (the forward products) or whose rows are (the gradients: no matrix
// is ever transposed in memory), in bf16, in fp32 as three bf16 pieces, or in 8 bits with block scales.
#pragma once
#include "encoder_pieces.h"
#include "norm_kernels.hip"

namespace enc {

// What becomes of a product's sums: act(z + bias) + residual, the gated block's act(g) * u, or the sums themselves.
struct Epilogue {
    const void *bias, *residual;    // of the output's type, nullable
    float *preact;                  // z in fp32 (gated: g and u side by side), nullable
    void *out, *out2;               // rows from split_row on go to out2 (two weights' gradients in one product)
    long long ld_r, ld_p, ld_o, ld_o2;
    int act;
    int split_row;                  // 0x7fffffff: one output
    int rows_each;                  // rows of one output (with two of them, padding lies between)
    bool out_f32;
};

template <typename T>
__device__ __forceinline__ void finish_linear8_as(const Epilogue &e, T *out, long long row, long long m, int n, int count, float (&z)[8])
{
    float t[8];
    if (e.bias) {
        load8((const T *)e.bias + n, count, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += t[i];
    }
    if (e.preact) store8(e.preact + m * e.ld_p + n, count, z);
    if (e.act != 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = activate(z[i], e.act);
    }
    if (e.residual) {
        load8((const T *)e.residual + m * e.ld_r + n, count, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += t[i];
    }
    store8(out + row + n, count, z);
}

// Columns n .. n + count - 1 (count <= 8) of row m.
__device__ __forceinline__ void finish_linear8(const Epilogue &e, int m, int n, int count, float (&z)[8])
{
    void *out = e.out;
    long long row = (long long)m * e.ld_o;
    if (m >= e.split_row) {
        out = e.out2;
        m -= e.split_row;
        row = (long long)m * e.ld_o2;
    }
    if (m >= e.rows_each) return;
    if (e.out_f32) finish_linear8_as(e, (float *)out, row, m, n, count, z);
    else finish_linear8_as(e, (__bf16 *)out, row, m, n, count, z);
}

// The same in two halves: what is read (zeros where there is nothing), and what is made of it (one output, no second one).
__device__ __forceinline__ void bias8(const Epilogue &e, int n, int count, float (&bias)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) bias[i] = 0.f;
    if (!e.bias || count <= 0) return;
    if (e.out_f32) load8((const float *)e.bias + n, count, bias);
    else load8((const __bf16 *)e.bias + n, count, bias);
}
__device__ __forceinline__ void residual8(const Epilogue &e, int m, int n, int count, float (&residual)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) residual[i] = 0.f;
    if (!e.residual || count <= 0) return;
    if (e.out_f32) load8((const float *)e.residual + m * e.ld_r + n, count, residual);
    else load8((const __bf16 *)e.residual + m * e.ld_r + n, count, residual);
}
__device__ __forceinline__ void finish_ahead8(const Epilogue &e, int m, int n, int count, float (&z)[8], const float (&bias)[8],
                                              const float (&residual)[8])
{
    if (e.bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += bias[i];
    }
    if (e.preact) store8(e.preact + m * e.ld_p + n, count, z);
    if (e.act != 0)
        with_act(e.act, [&](auto a) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = activate_as<decltype(a)::value>(z[i]);
        });
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += residual[i];
    }
    const long long at = (long long)m * e.ld_o + n;
    if (e.out_f32) store8((float *)e.out + at, count, z);
    else store8((__bf16 *)e.out + at, count, z);
}

__device__ __forceinline__ void finish_gated8(const Epilogue &e, int m, int f, int count, const float (&g)[8], const float (&u)[8])
{
    if (e.preact) {
        float *p = e.preact + (long long)m * e.ld_p + 2 * (long long)f;
        const float lo[8] = {g[0], u[0], g[1], u[1], g[2], u[2], g[3], u[3]}, hi[8] = {g[4], u[4], g[5], u[5], g[6], u[6], g[7], u[7]};
        store8(p, 2 * count, lo);
        store8(p + 8, 2 * count - 8, hi);
    }
    float h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = activate(g[i], e.act) * u[i];
    const long long at = (long long)m * e.ld_o + f;
    if (e.out_f32) store8((float *)e.out + at, count, h);
    else store8((__bf16 *)e.out + at, count, h);
}

// One operand of a product on the matrix cores.
struct Side {
    const unsigned char *p, *p2;    // p2: the gated block's second weight
    const uint8_t *scale, *scale2;  // 8-bit elements: scale bytes, four to a stage
    long long pitch;                // bytes from row to row (k contiguous) or from k to k (rows contiguous)
    long long scale_pitch;
    int extent;                     // rows of this side; rows contiguous: what may be read of them, a multiple of 8
};

// k runs through `count` segments of `stages` stages each (fp32: pairs of pieces; two summed products: the pairs).
constexpr int MAX_SEGMENTS = 12;
struct Segments {
    int count, stages;
    int rem;                        // how many k there are in a segment's last stage; 0: all of it
    long long a[MAX_SEGMENTS], b[MAX_SEGMENTS];     // byte offsets of the segments' first elements
};

// fp32 factors as their pieces, to go back to where the pieces' products say nothing: an infinity times a piece that is
// zero, or times two of opposite signs, is a NaN.
struct Pieces3 {
    const __bf16 *a[2], *b[2];      // per pair; null: not an fp32 product
    long long a_plane, b_plane, a_row, a_k, b_row, b_k;
    int pairs, K;
};

// Factors k + 4 half .. + 3 of the row that lies `lane` elements from `row`, `step` apart; from K on zeros (rows that lie in a run are
// packed: zeros up to a multiple of 64).  row, k: the same in every lane.
__device__ __forceinline__ void whole4(const __bf16 *row, unsigned lane, long long plane, long long step, int k, int half, int K, float (&v)[4])
{
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    if (step == 1) {
        const __bf16 *p = row + k;
        const unsigned at = lane + half * 4;
        const bf16x4 a = *reinterpret_cast<const bf16x4 *>(p + at), b = *reinterpret_cast<const bf16x4 *>(p + plane + at),
                     c = *reinterpret_cast<const bf16x4 *>(p + 2 * plane + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = ((float)c[e] + (float)b[e]) + (float)a[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int first = min(k + e, K - 1);
            const __bf16 *p = row + first * step;
            const unsigned at = lane + (unsigned)(min(k + e + half * 4, K - 1) - first) * (unsigned)step;
            const float f = ((float)(p + 2 * plane)[at] + (float)(p + plane)[at]) + (float)p[at];
            v[e] = k + e + half * 4 < K ? f : 0.f;
        }
    }
}

__device__ __forceinline__ bool is_finite(float v) { return fabsf(v) <= 3.402823466e38f; }

// 32 x 32 sums of a wave, in LDS with rows `pitch` floats apart: those that are not finite (of the first `rows` rows and `cols` columns) are
// computed again, from whole numbers on the fp32 matrix instruction.  m0, n0: the block's place in the product.  Ends as soon as all of them are NaN,
// which no further term changes.  Every lane has to come along.  Bound by that instruction and by loads that nothing hides: a call whose every sum
// is infinite takes up to 14 times what a finite one does (4104 x 2056 x 1040 2.2 ms against 0.16, its gradients 2.5 against 0.29, all NaN 0.3).
__device__ __forceinline__ void mend_block(const Pieces3 &x, int which, int m0, int n0, int rows, int cols, float *block, int pitch)
{
    const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
    float *mine = block + r * pitch + half * 4;         // sum 4 q + e lies at 8 q + e
    unsigned wanted = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int c = (i >> 2) * 8 + (i & 3);
        if (r < rows && half * 4 + c < cols && !is_finite(mine[c])) wanted |= 1u << i;
    }
    if (!__any(wanted != 0)) return;
    m0 = __builtin_amdgcn_readfirstlane(m0);
    n0 = __builtin_amdgcn_readfirstlane(n0);
    const unsigned a_lane = (unsigned)min(r, rows - 1) * (unsigned)x.a_row, b_lane = (unsigned)min(r, cols - 1) * (unsigned)x.b_row;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    bool open = true;
    for (int pair = 0; pair < x.pairs && open; ++pair) {
        const __bf16 *a = x.a[pair] + m0 * x.a_row, *b = (which ? x.b[1] : x.b[pair]) + n0 * x.b_row;
#pragma unroll 1
        for (int k0 = 0; k0 < x.K && open; k0 += 64) {
            const int end = min(x.K, k0 + 64);
#pragma unroll 1
            for (int k = k0; k < end; k += 8) {
                float u[4], v[4];
                whole4(a, a_lane, x.a_plane, x.a_k, k, half, x.K, u);
                whole4(b, b_lane, x.b_plane, x.b_k, k, half, x.K, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e], u[e], acc, 0, 0, 0);
            }
            bool mine_open = false;
#pragma unroll
            for (int i = 0; i < 16; ++i) mine_open |= ((wanted >> i) & 1) != 0 && acc[i] == acc[i];
            open = __any(mine_open);
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if ((wanted >> i) & 1) mine[(i >> 2) * 8 + (i & 3)] = acc[i];
}

// ---------------------------------------------------------------------------------------------------------------------------
// The tile kernel.  A workgroup of four waves (2 x 2) computes a tile of 2 WT x 2 WT sums, each wave WT x WT of them as
// MFMA blocks of 32 x 32; WT = 128 fills a lane's 256 accumulators (one workgroup to a compute unit), WT = 64 takes
// a quarter of that (two workgroups to a compute unit).
//
// Operands go from global memory straight into LDS (lane L's 16 bytes land at base + 16 L), 128 bytes of k per row and
// stage, two stages.  k contiguous: the 16-byte chunk c of row r sits at chunk c ^ ((r >> 1) & 7) of the row's 128 bytes,
// which spreads the 16 rows that one pass of a ds_read_b128 touches over all banks.  Rows contiguous: a stage is 64 lines of k, and
// ds_read_b64_tr_b16 turns 4 x 16 elements round on their way to the registers; the 64-byte block b of line k
// sits at block b ^ f(k), so that the lines that one such read touches at once lie in different banks.
//
// The loads are inline asm whose completion is awaited by vmcnt, since the compiler would wait for all of them at every barrier.  A
// stage is four k sub-steps (8 bits: two of twice the k); fragments are read one sub-step ahead, the barrier that
// frees the stage's buffer sits early in sub-step 2, and the loads of stage s+2 are spread over what follows of stage s.
// ---------------------------------------------------------------------------------------------------------------------------
namespace tile {

constexpr int THREADS = 256;
constexpr int LINE = 128;

enum { K_RUNS = 0, ROWS_RUN = 1 };      // which of an operand's extents is contiguous
// What a tile's sums become.  _PIECES: of fp32 by pieces, whose sums that are not finite are looked at again.
enum { TO_LINEAR = 0, TO_GATED = 1, TO_PARTS = 2, TO_GATED_PARTS = 3, TO_LINEAR_PIECES = 4, TO_GATED_PIECES = 5 };
constexpr bool is_gated(int to) { return to == TO_GATED || to == TO_GATED_PARTS || to == TO_GATED_PIECES; }
constexpr bool is_parts(int to) { return to == TO_PARTS || to == TO_GATED_PARTS; }

template <int WT, bool MX> struct Shape {
    static constexpr int T = 2 * WT, NB = WT / 32;
    static constexpr int HALF = T * LINE;                       // bytes of one operand and stage
    static constexpr int SCALES = MX ? 2 * T * 4 : 0;           // four scale bytes per row
    static constexpr int STAGE = 2 * HALF + SCALES;
    static constexpr int NLOAD = 2 * HALF / (THREADS * 16);     // per lane and stage
    static constexpr int NSCALE = SCALES / (THREADS * 4);
    static constexpr int LDS_BYTES = 2 * STAGE;
    static constexpr int TURN_PITCH = WT + 4;                   // floats
    static_assert(4 * 32 * TURN_PITCH * 4 <= LDS_BYTES, "the waves' turn-round regions fit where the stages were");
};

// (M0 holds the LDS address; the instruction may follow M0's write only after a wait state)
__device__ __forceinline__ void load16_to_lds(const void *base, unsigned offset, unsigned lds_addr)
{
    asm volatile("s_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(offset), "s"(base), "{m0}"(lds_addr)
                 : "memory");
}
__device__ __forceinline__ void load4_to_lds(const void *base, unsigned offset, unsigned lds_addr)
{
    asm volatile("s_nop 0\n\t"
                 "global_load_lds_dword %0, %1"
                 :
                 : "v"(offset), "s"(base), "{m0}"(lds_addr)
                 : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// A barrier that no access to LDS is moved across.
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <int WT, int KA, int KB, bool MX, bool GATED>
struct Pipe {
    using S = Shape<WT, MX>;
    static constexpr int NB = S::NB, NM = NB * NB, T = S::T;
    static constexpr int MINE = S::NLOAD;      // this wave's loads: half of one operand's stage
    unsigned char *lds;
    unsigned lds_base, wave_dst, scale_dst;
    unsigned off[S::NLOAD];                    // byte offset of this lane's chunk from the stage's base
    unsigned soff[MX ? S::NSCALE : 1];
    bool loads_a;                              // waves 0 and 1 load a, 2 and 3 b
    const unsigned char *base, *base2;         // the next stage to load (base2: the gated block's second weight)
    const unsigned char *sbase, *sbase2;
    const unsigned char *p, *p2, *sp, *sp2;    // this wave's operand at this tile, without its segment's offset
    long long step;                            // bytes from stage to stage
    int seg, left;                             // segment of the next stage to load, its stages left
    int frag_a, frag_b, sw16, hi16;            // k contiguous: this lane's row, swizzle and k half
    int blk_a[NB], blk_b[NB];                  // rows contiguous: its block offsets
    f32x16 acc[NB][NB];                        // [block of a's rows][block of b's rows]; a lane holds one row of a

    static __device__ __forceinline__ int line_swizzle(int k) { return T == 256 ? ((k & 3) | (((k >> 3) & 1) << 2)) : (k & 3); }

    // Where load u of this lane comes from, inside the stage: row (or line of k) and 16-byte chunk of it.
    template <int KIND> static __device__ __forceinline__ void slot(int half, int u, int lane, int *row, int *chunk)
    {
        const int ci = (half * S::NLOAD + u) * 64 + lane;
        if constexpr (KIND == K_RUNS) {
            *row = ci >> 3;
            *chunk = (ci & 7) ^ ((*row >> 1) & 7);
        } else {
            constexpr int PER = T / 8;
            *row = ci / PER;
            const int pos = ci % PER;
            *chunk = ((((pos >> 2) ^ line_swizzle(*row)) << 2) | (pos & 3));
        }
    }
    template <int KIND> __device__ __forceinline__ void place(const Side &s, int tile0, int half, int lane, bool dual)
    {
#pragma unroll
        for (int u = 0; u < S::NLOAD; ++u) {
            int row, chunk;
            slot<KIND>(half, u, lane, &row, &chunk);
            if constexpr (KIND == K_RUNS) {
                int r = row;
                if (dual) r = (row / WT) * (WT / 2) + ((row % WT) >> 6) * 32 + (row & 31);     // 32 rows of the gate, 32 of the other, ...
                r = min(tile0 + r, s.extent - 1) - tile0;
                off[u] = (unsigned)((long long)r * s.pitch + chunk * 16);
            } else {
                const int c = min(tile0 / 8 + chunk, s.extent / 8 - 1) - tile0 / 8;
                off[u] = (unsigned)((long long)row * s.pitch + c * 16);
            }
        }
        const long long shift = KIND == K_RUNS ? (long long)tile0 * s.pitch : (long long)tile0 * 2;
        p = s.p + shift;
        p2 = dual ? s.p2 + shift : p;
        step = KIND == K_RUNS ? LINE : 64 * s.pitch;
        if constexpr (MX) {
#pragma unroll
            for (int v = 0; v < S::NSCALE; ++v) {
                const int row = (half * S::NSCALE + v) * 64 + lane;
                int r = row;
                if (dual) r = (row / WT) * (WT / 2) + ((row % WT) >> 6) * 32 + (row & 31);
                r = min(tile0 + r, s.extent - 1) - tile0;
                soff[v] = (unsigned)((long long)r * s.scale_pitch);
                if (dual && ((row >> 5) & 1)) soff[v] |= 0x80000000u;      // (marks the second weight's rows)
            }
            sp = s.scale + (long long)tile0 * s.scale_pitch;
            sp2 = dual ? s.scale2 + (long long)tile0 * s.scale_pitch : sp;
        }
    }
    __device__ __forceinline__ void init(unsigned char *lds_, const Side &a, const Side &b, int m0, int n0)
    {
        lds = lds_;
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wr = wave >> 1, wc = wave & 1;
        lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds;
        wave_dst = lds_base + wave * (S::NLOAD * 1024);
        scale_dst = lds_base + 2 * S::HALF + wave * (S::NSCALE * 256);
        loads_a = wave < 2;
        if (loads_a) place<KA>(a, m0, wave & 1, lane, false);
        else place<KB>(b, n0, wave & 1, lane, GATED);
        sw16 = ((lane & 31) >> 1 & 7) << 4;        // (fragment rows differ from lane & 31 by multiples of 32)
        hi16 = (lane >> 5) << 4;
        frag_a = (wr * WT + (lane & 31)) * LINE;
        frag_b = S::HALF + (wc * WT + (lane & 31)) * LINE;
        const int i16 = lane & 15, f = T == 256 ? ((i16 >> 2) | ((lane >> 5) << 2)) : (i16 >> 2);
        const int inside = ((lane >> 5) * 8 + (i16 >> 2)) * (T * 2) + ((lane >> 4) & 1) * 32 + (i16 & 3) * 8;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            blk_a[i] = inside + (((wr * NB + i) ^ f) << 6);
            blk_b[i] = S::HALF + inside + (((wc * NB + i) ^ f) << 6);
        }
    }
    // The base of stage `stage` (of all segments end to end) becomes the next one to load.
    __device__ __forceinline__ void seek(const Segments &g, int stage)
    {
        seg = stage / g.stages;
        const int in = stage - seg * g.stages;
        left = g.stages - in;
        const long long o = (loads_a ? g.a[seg] : g.b[seg]) + (long long)in * step;
        base = p + o;
        base2 = p2 + o;
        if constexpr (MX) {
            sbase = sp + in * 4;
            sbase2 = sp2 + in * 4;
        }
    }
    __device__ __forceinline__ void advance(const Segments &g)
    {
        if (--left == 0) {
            seg = min(seg + 1, g.count - 1);
            left = g.stages;
            const long long o = loads_a ? g.a[seg] : g.b[seg];
            base = p + o;
            base2 = p2 + o;
        } else {
            base += step;
            base2 += step;
            if constexpr (MX) {
                sbase += 4;
                sbase2 += 4;
            }
        }
    }
    // Load u of the next stage into buffer buf.  TAIL: only the stage's first `rem` k; the rest of it becomes zeros.
    template <bool TAIL> __device__ __forceinline__ void load1(int buf, int u, int rem)
    {
        const unsigned char *from = GATED && ((u >> 2) & 1) ? base2 : base;
        const unsigned to = wave_dst + buf * S::STAGE + u * 1024;
        if constexpr (!TAIL) {
            load16_to_lds(from, off[u], to);
        } else {
            const int lane = threadIdx.x & 63, half = (threadIdx.x >> 6) & 1;
            int row, chunk;
            bool there;
            constexpr int ESZ = MX ? 1 : 2;
            if (loads_a) {
                slot<KA>(half, u, lane, &row, &chunk);
                there = KA == K_RUNS ? chunk * 16 < rem * ESZ : row < rem;
            } else {
                slot<KB>(half, u, lane, &row, &chunk);
                there = KB == K_RUNS ? chunk * 16 < rem * ESZ : row < rem;
            }
            if (there) load16_to_lds(from, off[u], to);
            else *reinterpret_cast<uint4 *>(lds + (to - lds_base) + lane * 16) = make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void load_scales(int buf)
    {
        if constexpr (MX) {
#pragma unroll
            for (int v = 0; v < S::NSCALE; ++v) {
                const unsigned to = scale_dst + buf * S::STAGE + v * 256;
                if (GATED && !loads_a) {
                    if (soff[v] & 0x80000000u) load4_to_lds(sbase2, soff[v] & 0x7fffffffu, to);
                    else load4_to_lds(sbase, soff[v], to);
                } else {
                    load4_to_lds(sbase, soff[v], to);
                }
            }
        }
    }

    struct Frags { uint4 v[2 * NB]; };          // v[0 .. NB-1]: a's blocks, v[NB ..]: b's
    // fragment i of k sub-step h (0 .. 3)
    __device__ __forceinline__ void read1(Frags &f, int buf, int h, int i)
    {
        const unsigned char *stage = lds + buf * S::STAGE;
        const bool of_a = i < NB;
        const int kind = of_a ? KA : KB, blk = of_a ? i : i - NB;
        if (kind == K_RUNS) {
            // sub-step h is 32 bytes of k, lanes 0-31 take the first half
            const int pos = h * 32 + hi16;
            f.v[i] = *reinterpret_cast<const uint4 *>(stage + (of_a ? frag_a : frag_b) + blk * 32 * LINE + (pos ^ sw16));
        } else {
            typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
            unsigned char *at = const_cast<unsigned char *>(stage) + (of_a ? blk_a[blk] : blk_b[blk]) + h * 16 * (T * 2);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * (T * 2)));
            const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            f.v[i] = __builtin_bit_cast(uint4, both);
        }
    }
    struct Frags8 { i32x8 v[2 * NB]; };         // 8 bits: both halves of a pair of sub-steps (0 and 1, or 2 and 3)
    template <int HALF> __device__ __forceinline__ void read8(Frags8 &f, int buf, int pair, int i)
    {
        // a lane holds chunk (lane >> 5) of each of a pair of scale blocks
        const unsigned char *stage = lds + buf * S::STAGE;
        const int pos = (pair * 64 + HALF * 32 + hi16) ^ sw16;
        const uint4 v = *reinterpret_cast<const uint4 *>(stage + (i < NB ? frag_a + i * 32 * LINE : frag_b + (i - NB) * 32 * LINE) + pos);
        f.v[i][HALF * 4] = (int)v.x;
        f.v[i][HALF * 4 + 1] = (int)v.y;
        f.v[i][HALF * 4 + 2] = (int)v.z;
        f.v[i][HALF * 4 + 3] = (int)v.w;
    }
    // this lane's scale words of a stage: two bytes each, byte 0 for its block of sub-steps 0/1, byte 2 for that of 2/3
    struct Words { int v[2 * NB]; };
    __device__ __forceinline__ void read_scale(Words &w, int buf, int i)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int row = i < NB ? (wave >> 1) * WT + i * 32 + (lane & 31) : T + (wave & 1) * WT + (i - NB) * 32 + (lane & 31);
        const unsigned word = *reinterpret_cast<const unsigned *>(lds + buf * S::STAGE + 2 * S::HALF + row * 4);
        w.v[i] = (int)(word >> ((lane >> 5) * 8));
    }

    // The multiplies of one sub-step (8 bits: of two), b's rows down a block's registers, a's across its lanes.  hook(i)
    // runs right behind the i-th.
    template <typename Hook> __device__ __forceinline__ void multiply(const Frags &f, Hook hook)
    {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f.v[NB + j]),
                                                                    __builtin_bit_cast(bf16x8, f.v[i]), acc[i][j], 0, 0, 0);
                pin();
                hook(i * NB + j);
                pin();
            }
    }
    template <int SEL, typename Hook> __device__ __forceinline__ void multiply8(const Frags8 &f, const Words &w, Hook hook)
    {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.v[NB + j], f.v[i], acc[i][j], 0, 0, SEL, w.v[NB + j],
                                                                            SEL, w.v[i]);
                // (keeps the multiply where it stands: this instruction alone may be moved across a branch)
                if constexpr (WT == 128) asm volatile("" : "+a"(acc[i][j]));
                else asm volatile("" : "+v"(acc[i][j]));
                pin();
                hook(i * NB + j);
                pin();
            }
    }

    // All of stages s0 .. s1 - 1.  Ends with a barrier: LDS is free in every wave.
    __device__ __forceinline__ void run(const Segments &g, int s0, int s1)
    {
        constexpr int ALL = S::NLOAD + S::NSCALE;
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        const int n = s1 - s0;
        seek(g, s0);
        auto fill = [&](int buf) {
            load_scales(buf);
            if (g.rem != 0 && left == 1) {
#pragma unroll
                for (int u = 0; u < S::NLOAD; ++u) load1<true>(buf, u, g.rem);
            } else {
#pragma unroll
                for (int u = 0; u < S::NLOAD; ++u) load1<false>(buf, u, 0);
            }
            advance(g);
        };
        fill(0);
        if (n > 1) {
            // (a tail's loads may be fewer than ALL: then all of them are awaited)
            const bool exact = !(g.rem != 0 && left == 1);
            fill(1);
            if (exact) wait_loads<ALL>();
            else wait_loads<0>();
        } else {
            wait_loads<0>();
        }
        wait_lds();
        meet();
        Frags f0, f1, f2, f3;
        Frags8 p0, p1;
        Words w, wn;
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) {
            if constexpr (MX) {
                read8<0>(p0, 0, 0, i);
                read8<1>(p0, 0, 0, i);
                read_scale(w, 0, i);
            } else {
                read1(f0, 0, 0, i);
            }
        }
        int buf = 0;
        constexpr int WAIT = NM / 4 - 1;                        // the multiply behind which the buffer is given up
        constexpr int PER = (2 * NB + NM - 1) / NM;             // reads of a sub-step's fragments per multiply
        auto nothing = [](int) {};
        auto stage = [&](auto more_tag, auto refill_tag) {
            constexpr bool MORE = decltype(more_tag)::value;
            constexpr bool REFILL = decltype(refill_tag)::value;    // a whole stage s+2 takes this stage's buffer
            auto reads = [&](Frags &f, int b, int h, int from, int count) {
#pragma unroll
                for (int i = 0; i < count; ++i)
                    if (from + i < 2 * NB) read1(f, b, h, from + i);
            };
            auto give_up = [&]() {
                wait_loads<0>();
                wait_lds();
                meet();
            };
            // the refill's loads: `done` of them are out, `count` more
            auto refill = [&](int done, int count) {
#pragma unroll
                for (int i = 0; i < count; ++i)
                    if (done + i < S::NLOAD) load1<false>(buf, done + i, 0);
            };
            if constexpr (!MX) {
                constexpr int EARLY = 6;                        // large tiles: loads behind sub-step 2's multiplies
                multiply(f0, [&](int i) { reads(f1, buf, 1, i * PER, PER); });
                multiply(f1, [&](int i) {
                    constexpr int H = NM / 2;
                    if (i < H) reads(f2, buf, 2, i * 2 * PER, 2 * PER);
                    else reads(f3, buf, 3, (i - H) * 2 * PER, 2 * PER);
                });
                multiply(f2, [&](int i) {
                    if (MORE && i == WAIT) give_up();
                    if constexpr (REFILL) {
                        // (a small tile's stage is shorter than a load takes: all of them at once)
                        if (NM == 16) {
                            if (i > WAIT && (i & 1) == 0) refill((i - WAIT - 1) / 2, 1);
                        } else if (i == WAIT) {
                            refill(0, S::NLOAD);
                        }
                    }
                });
                multiply(f3, [&](int i) {
                    if constexpr (MORE) reads(f0, buf ^ 1, 0, i * PER, PER);
                    if constexpr (REFILL) {
                        if (NM == 16) refill(EARLY + i, i < S::NLOAD - EARLY ? 1 : 0);
                    }
                });
            } else {
                multiply8<0>(p0, w, [&](int i) {
                    constexpr int EACH = (4 * NB + NM - 1) / NM;
#pragma unroll
                    for (int k = 0; k < EACH; ++k) {
                        const int r = i * EACH + k;
                        if (r < 4 * NB) {
                            if (r & 1) read8<1>(p1, buf, 1, r >> 1);
                            else read8<0>(p1, buf, 1, r >> 1);
                        }
                    }
                });
                multiply8<2>(p1, w, [&](int i) {
                    if (MORE && i == WAIT) {
                        give_up();
                        if constexpr (REFILL && NM != 16) {
                            load_scales(buf);
                            refill(0, S::NLOAD);
                        }
                    }
                    if (i > WAIT) {
                        constexpr int ROOM = NM - 1 - WAIT;
                        const int at = i - WAIT - 1;
                        if constexpr (MORE) {
                            constexpr int EACH = (4 * NB + ROOM - 1) / ROOM;
#pragma unroll
                            for (int k = 0; k < EACH; ++k) {
                                const int r = at * EACH + k;
                                if (r < 4 * NB) {
                                    if (r & 1) read8<1>(p0, buf ^ 1, 0, r >> 1);
                                    else read8<0>(p0, buf ^ 1, 0, r >> 1);
                                }
                            }
                            if (at < 2 * NB && ROOM >= 2 * NB) read_scale(wn, buf ^ 1, at);
                            if (ROOM < 2 * NB && at == 0) {
#pragma unroll
                                for (int k = 0; k < 2 * NB; ++k) read_scale(wn, buf ^ 1, k);
                            }
                        }
                        if constexpr (REFILL && NM == 16) {
                            constexpr int EACH = (S::NLOAD + ROOM - 1) / ROOM;
                            if (at == 0) load_scales(buf);
                            refill(at * EACH, EACH);
                        }
                    }
                });
                w = wn;
            }
            if constexpr (REFILL) advance(g);
            buf ^= 1;
        };
        using std::bool_constant;
        int s = 0;
#pragma unroll 1
        for (;;) {
            // as long as the stage to load is a whole one; a segment's short last stage is loaded behind its predecessor's
            // multiplies, outside of this loop
            int whole = n - 2 - s;
            if (g.rem != 0) whole = min(whole, left - 1);
#pragma unroll 1
            for (; whole > 0; --whole, ++s) stage(bool_constant<true>{}, bool_constant<true>{});
            if (s + 1 >= n) break;
            const bool another = s + 2 < n;
            stage(bool_constant<true>{}, bool_constant<false>{});
            ++s;
            if (another) fill(buf ^ 1);
        }
        stage(bool_constant<false>{}, bool_constant<false>{});
        wait_lds();
        meet();
    }
};

// Tile number t of the list for workgroup w.  Workgroups are dealt round-robin to the 8 XCDs, each with an L2 of its own:
// an XCD gets a contiguous run of the list, which walks the grid of tiles in bands of 8 tile rows, down the band first, so
// that the workgroups that an XCD runs side by side share operand rows in its L2.
__device__ __forceinline__ bool tile_of_workgroup(int w, int nwg, int tiles_m, int tiles_n, int splits, int *ti, int *tj, int *split)
{
    const int per = (nwg + 7) >> 3, tiles = tiles_m * tiles_n;
    int t = (w & 7) * per + (w >> 3);
    if (t >= tiles * splits) return false;
    *split = t / tiles;
    t -= *split * tiles;
    constexpr int BAND = 8;
    const int band = t / (BAND * tiles_n);
    const int rows = min(BAND, tiles_m - band * BAND);
    const int r = t - band * BAND * tiles_n;
    *ti = band * BAND + r % rows;
    *tj = r / rows;
    return true;
}

struct Args {
    Side a, b;
    Segments seg;
    Epilogue e;
    Pieces3 pieces;
    float *parts;                   // [split][M][parts_pitch], gated: g's columns, then u's from parts_half on
    long long parts_pitch;
    int parts_half;
    int M, N;                       // N: output columns
    int tiles_m, tiles_n, splits;
};

// One accumulator at the point of use.  WT = 128: read explicitly, so that the register allocator does not move all 256 of
// them into ordinary registers at once, which leaves room for nothing else.
template <int WT> __device__ __forceinline__ float accumulator(float a)
{
    if constexpr (WT != 128) return a;
    float v;
    asm("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(a));
    return v;
}

// 32 rows of a wave's sums in LDS, and their way out.
template <int WT, bool GATED> struct Band {
    static constexpr int PITCH = WT + 4;
    static constexpr int COLS = GATED ? WT / 2 : WT;        // output columns of the wave
    float *turn;

    // column c of the wave's: a gated wave has 32 of the gate, 32 of the other, ...
    static __device__ __forceinline__ int at(int c) { return GATED ? (c >> 5) * 64 + (c & 31) : c; }

    // the bare sums, four columns to a lane; rows and columns of `parts` reach to multiples of eight
    __device__ __forceinline__ void parts(const Args &x, int split, int m, int n)
    {
        const int lane = threadIdx.x & 63;
        constexpr int LANES = COLS / 4, ROWS = 64 / LANES;
        const int c = (lane % LANES) * 4, r0 = lane / LANES;
        if (n + c >= x.N) return;
        float *to = x.parts + ((size_t)split * x.M + m) * x.parts_pitch + n + c;
#pragma unroll
        for (int k = 0; k < 32 / ROWS; ++k) {
            const int r = r0 + k * ROWS;
            if (m + r >= x.M) break;
            *reinterpret_cast<f32x4 *>(to + r * x.parts_pitch) = *reinterpret_cast<const f32x4 *>(turn + r * PITCH + at(c));
            if constexpr (GATED)
                *reinterpret_cast<f32x4 *>(to + r * x.parts_pitch + x.parts_half) =
                    *reinterpret_cast<const f32x4 *>(turn + r * PITCH + at(c) + 32);
        }
    }

    // every check, eight columns to a lane.  The residual of four rows is on its way before the first of them is stored.  (With
    // whole tiles at the result's edge taken this way, row after row, they ended last: 5000 x 2048 x 2048 with gelu and residual 98 us,
    // 70 so.)
    __device__ __forceinline__ void checked(const Args &x, int m, int n)
    {
        const int lane = threadIdx.x & 63;
        constexpr int LANES = COLS / 8, ROWS = 64 / LANES, AHEAD = ROWS > 8 ? 32 / ROWS : 4;
        const int c = (lane % LANES) * 8, count = x.N - n - c;
        if (count <= 0) return;
        float bias[8], residual[AHEAD][8];
        if constexpr (!GATED) bias8(x.e, n + c, count, bias);
#pragma unroll 1
        for (int r0 = lane / LANES; r0 < 32; r0 += AHEAD * ROWS) {
            if constexpr (!GATED) {
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) residual8(x.e, min(m + r0 + k * ROWS, x.M - 1), n + c, count, residual[k]);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int r = r0 + k * ROWS;
                float z[8];
                load8(turn + r * PITCH + at(c), 8, z);
                if constexpr (GATED) {
                    float u[8];
                    load8(turn + r * PITCH + at(c) + 32, 8, u);
                    if (m + r < x.M) finish_gated8(x.e, m + r, n + c, count, z, u);
                } else if (m + r < x.M) {
                    if (x.e.split_row != 0x7fffffff) finish_linear8(x.e, m + r, n + c, count, z);
                    else finish_ahead8(x.e, m + r, n + c, count, z, bias, residual[k]);
                }
            }
        }
    }

    // fp32 by pieces: sums that are not finite, computed again
    __device__ __forceinline__ void mend(const Args &x, int m, int n)
    {
#pragma unroll 1
        for (int j = 0; j < WT / 32; ++j) {
            const int at = n + (GATED ? j >> 1 : j) * 32;
            if (at < x.N) mend_block(x.pieces, GATED ? j & 1 : 0, m, at, x.M - m, x.N - at, turn + j * 32, PITCH);
        }
    }

    // whether all of the band's sums are finite (the same answer in every lane)
    __device__ __forceinline__ bool finite()
    {
        const int lane = threadIdx.x & 63;
        float zero = 0.f;
#pragma unroll 4
        for (int k = 0; k < 32 * WT / 256; ++k) {
            const int at4 = k * 64 + lane;
            const f32x4 v = *reinterpret_cast<const f32x4 *>(turn + at4 / (WT / 4) * PITCH + at4 % (WT / 4) * 4);
            zero = fmaf(v[0], 0.f, zero);
            zero = fmaf(v[1], 0.f, zero);
            zero = fmaf(v[2], 0.f, zero);
            zero = fmaf(v[3], 0.f, zero);
        }
        return !__any(!(zero == 0.f));
    }

    // The residual of a band on its way, ahead of the band's sums: nothing else runs on the unit to hide that trip.
    static constexpr int HELD = GATED ? 1 : 32 * WT / 256;      // fp32: four columns to a lane; bf16 needs half of them
    f32x4 held[HELD];
    __device__ __forceinline__ void fetch_residual(const Epilogue &e, int m, int n)
    {
        if constexpr (!GATED) {
            if (!e.residual) return;
            if (e.out_f32) fetch_as<float, 4>(e, m, n);
            else fetch_as<__bf16, 8>(e, m, n);
        }
    }
    template <typename T, int V> __device__ __forceinline__ void fetch_as(const Epilogue &e, int m, int n)
    {
        const int lane = threadIdx.x & 63;
        constexpr int LANES = COLS / V, ROWS = 64 / LANES, R = 32 / ROWS;
        const T *res = (const T *)e.residual + (long long)(m + lane / LANES) * e.ld_r + n + (lane % LANES) * V;
#pragma unroll
        for (int k = 0; k < R; ++k) held[k] = *reinterpret_cast<const f32x4_any *>(res + k * ROWS * e.ld_r);
    }

    // next: the row of the band after this one, or -1
    __device__ __forceinline__ void inside(const Epilogue &e, int m, int n, int next)
    {
        if constexpr (GATED) {
            if (e.preact) save_pairs(e, m, n);
            if (e.out_f32) gated<float, 4>(e, m, n);
            else gated<__bf16, 8>(e, m, n);
        } else {
            if (e.preact) save(e, m, n);
            if (e.out_f32) linear<float, 4>(e, m, n, next);
            else linear<__bf16, 8>(e, m, n, next);
        }
    }

    // V consecutive elements, 16 bytes
    template <typename T, int V> static __device__ __forceinline__ void get(const T *p, float (&v)[V])
    {
        const typename Any<T>::type t = *reinterpret_cast<const typename Any<T>::type *>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)t[i];
    }
    template <typename T, int V> static __device__ __forceinline__ void put(T *p, const float (&v)[V])
    {
        typename Any<T>::type t;
#pragma unroll
        for (int i = 0; i < V; ++i) t[i] = (T)v[i];
        *reinterpret_cast<typename Any<T>::type *>(p) = t;
    }
    // V sums of row r from column c (of the turned band) on
    template <int V> __device__ __forceinline__ void sums(int r, int c, float (&z)[V])
    {
#pragma unroll
        for (int h = 0; h < V; h += 4) {
            const f32x4 t = *reinterpret_cast<const f32x4 *>(turn + r * PITCH + c + h);
            z[h] = t[0]; z[h + 1] = t[1]; z[h + 2] = t[2]; z[h + 3] = t[3];
        }
    }

    // z in fp32, for the backward call: read once, much later, so it passes by the caches
    __device__ __forceinline__ void save(const Epilogue &e, int m, int n)
    {
        const int lane = threadIdx.x & 63;
        constexpr int LANES = COLS / 4, ROWS = 64 / LANES;
        const int c = (lane % LANES) * 4, r0 = lane / LANES;
        float b[4] = {0.f, 0.f, 0.f, 0.f};
        if (e.bias)
            for (int i = 0; i < 4; ++i) b[i] = e.out_f32 ? ((const float *)e.bias)[n + c + i] : (float)((const __bf16 *)e.bias)[n + c + i];
        float *to = e.preact + (long long)m * e.ld_p + n + c;
#pragma unroll
        for (int k = 0; k < 32 / ROWS; ++k) {
            float z[4];
            sums<4>(r0 + k * ROWS, c, z);
            const f32x4 v = {z[0] + b[0], z[1] + b[1], z[2] + b[2], z[3] + b[3]};
            __builtin_nontemporal_store(v, reinterpret_cast<f32x4_any *>(to + (r0 + k * ROWS) * e.ld_p));
        }
    }
    // g and u side by side, two pairs to a lane
    __device__ __forceinline__ void save_pairs(const Epilogue &e, int m, int f)
    {
        const int lane = threadIdx.x & 63;
        constexpr int LANES = COLS / 2, ROWS = 64 / LANES;
        const int c = (lane % LANES) * 2, r0 = lane / LANES;
        float *to = e.preact + (long long)m * e.ld_p + 2 * (f + c);
#pragma unroll
        for (int k = 0; k < 32 / ROWS; ++k) {
            const float *from = turn + (r0 + k * ROWS) * PITCH + at(c);
            const float2 g = *reinterpret_cast<const float2 *>(from), u = *reinterpret_cast<const float2 *>(from + 32);
            const f32x4 v = {g.x, u.x, g.y, u.y};
            __builtin_nontemporal_store(v, reinterpret_cast<f32x4_any *>(to + (r0 + k * ROWS) * e.ld_p));
        }
    }

    template <typename T, int V> __device__ __forceinline__ void linear(const Epilogue &e, int m, int n, int next)
    {
        const int lane = threadIdx.x & 63;
        constexpr int LANES = COLS / V, ROWS = 64 / LANES, R = 32 / ROWS;
        const int c = (lane % LANES) * V, r0 = lane / LANES;
        const bool second = m >= e.split_row;
        T *out = (T *)(second ? e.out2 : e.out);
        const long long ld = second ? e.ld_o2 : e.ld_o;
        out += (long long)(m - (second ? e.split_row : 0) + r0) * ld + n + c;
        float z[R][V], b[V];
        if (e.bias) get<T, V>((const T *)e.bias + n + c, b);
#pragma unroll
        for (int k = 0; k < R; ++k) sums<V>(r0 + k * ROWS, c, z[k]);
        if (e.bias) {
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) z[k][i] += b[i];
        }
        if (e.act != 0)
            with_act(e.act, [&](auto a) {
#pragma unroll
                for (int k = 0; k < R; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) z[k][i] = activate_as<decltype(a)::value>(z[k][i]);
            });
        if (e.residual) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                typedef T vec __attribute__((ext_vector_type(V)));
                const vec t = __builtin_bit_cast(vec, held[k]);
#pragma unroll
                for (int i = 0; i < V; ++i) z[k][i] += (float)t[i];
            }
            if (next >= 0) fetch_residual(e, next, n);
        }
#pragma unroll
        for (int k = 0; k < R; ++k) put<T, V>(out + k * ROWS * ld, z[k]);
    }

    template <typename T, int V> __device__ __forceinline__ void gated(const Epilogue &e, int m, int f)
    {
        const int lane = threadIdx.x & 63;
        constexpr int LANES = COLS / V, ROWS = 64 / LANES, R = 32 / ROWS;
        const int c = (lane % LANES) * V, r0 = lane / LANES;
        T *out = (T *)e.out + (long long)(m + r0) * e.ld_o + f + c;
        with_act(e.act, [&](auto a) {
            float g[R][V], u[R][V];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                sums<V>(r0 + k * ROWS, at(c), g[k]);
                sums<V>(r0 + k * ROWS, at(c) + 32, u[k]);
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
#pragma unroll
                for (int i = 0; i < V; ++i) g[k][i] = activate_as<decltype(a)::value>(g[k][i]) * u[k][i];
                put<T, V>(out + k * ROWS * e.ld_o, g[k]);
            }
        });
    }
};

// Workgroup `wg` of the `nwg` that share one product.
template <int WT, int KA, int KB, bool MX, int TO>
__device__ __forceinline__ void tile_body(const Args &x, int wg, int nwg)
{
    constexpr bool GATED = is_gated(TO);
    using P = Pipe<WT, KA, KB, MX, GATED>;
    using S = typename P::S;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    int ti, tj, split;
    if (!tile_of_workgroup(wg, nwg, x.tiles_m, x.tiles_n, x.splits, &ti, &tj, &split)) return;
    constexpr int COLS = GATED ? WT : 2 * WT;      // output columns of a tile
    const int m0 = ti * S::T, n0 = tj * COLS;
    const int all = x.seg.count * x.seg.stages;
    const int s0 = (int)((long long)all * split / x.splits), s1 = (int)((long long)all * (split + 1) / x.splits);
    P p;
    p.init(lds, x.a, x.b, m0, n0);
    p.run(x.seg, s0, s1);

    // The sums, 32 rows of this wave at a time, are turned round in LDS (a region of its own for each wave), so that a
    // lane gets neighbouring columns and everything behind them is whole 16-byte accesses, whole lines by the wave.  A
    // band that lies inside the result goes without checks, its loads ahead of its stores.
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Band<WT, GATED> band;
    band.turn = reinterpret_cast<float *>(lds) + wave * (32 * S::TURN_PITCH);
    const int wm = m0 + (wave >> 1) * WT, wn = n0 + (wave & 1) * (COLS / 2);
    // whether the 32 rows from m on lie inside, in this wave's columns
    auto inside = [&](int m) {
        return m + 32 <= x.M && wn + COLS / 2 <= x.N &&
               (x.e.split_row == 0x7fffffff || m + 32 <= x.e.rows_each || (m >= x.e.split_row && m - x.e.split_row + 32 <= x.e.rows_each));
    };
    auto turn_round = [&](auto band_tag) {
        constexpr int I = decltype(band_tag)::value;
        if constexpr (I < P::NB) {
#pragma unroll
            for (int j = 0; j < P::NB; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = accumulator<WT>(p.acc[I][j][4 * q + e]);
                    *reinterpret_cast<f32x4 *>(band.turn + (lane & 31) * S::TURN_PITCH + j * 32 + q * 8 + (lane >> 5) * 4) = v;
                }
        }
    };
    if constexpr (!GATED && !is_parts(TO))
        if (inside(wm)) band.fetch_residual(x.e, wm, wn);
    // (a loop: unrolled, the code behind it would be there four times)
#pragma unroll 1
    for (int i = 0; i < P::NB && wm + i * 32 < x.M; ++i) {
        if (i == 0) turn_round(std::integral_constant<int, 0>{});
        else if (i == 1) turn_round(std::integral_constant<int, 1>{});
        else if (i == 2) turn_round(std::integral_constant<int, 2>{});
        else turn_round(std::integral_constant<int, 3>{});
        pin();
        const int m = wm + i * 32;
        if constexpr (is_parts(TO)) band.parts(x, split, m, wn);
        else {
            if constexpr (TO == TO_LINEAR_PIECES || TO == TO_GATED_PIECES)
                if (!band.finite()) band.mend(x, m, wn);
            if (inside(m)) band.inside(x.e, m, wn, i + 1 < P::NB && inside(m + 32) ? m + 32 : -1);
            else band.checked(x, m, wn);
        }
        pin();
    }
}

// Bound by the matrix cores where there are many tiles: the gradients of 16384 tokens' gated block of 8192 x 2048, in 256 x 256 tiles, 861 us
// (the tokens') and 842 (the weights'), 1.1 TFLOP each: 1.28 and 1.31 PFLOP/s, 93 and 95 % of a large library product, the clock being held down by
// power.  What the epilogue moves comes on top where workgroups end together: 16384 x 2048 x 2048 with gelu, residual and z 212 us, of which 268 MB
// of epilogue; the gated block forward, g and u kept, 1198 us of which 786 are multiplies.  8 bits: 5000 x 2048 x 8192 125 us in 160 tiles on 256 units,
// 1.3 PFLOP/s (2.1 on the units in use).
template <int WT, int KA, int KB, bool MX, int TO>
__global__ void __launch_bounds__(THREADS, WT == 128 ? 1 : 2)
k_tile(const Args x)
{
    tile_body<WT, KA, KB, MX, TO>(x, (int)blockIdx.x, (int)gridDim.x);
}

// A backward call's two products side by side: x's workgroups are the first `first` (a multiple of 8) of the launch.  Neither fills the
// device, and what is left is starts and ends: 1000 x 1024 x 1024 bf16 21.8 us the call, 31.6 one after the other.
template <bool PIECES>
__global__ void __launch_bounds__(THREADS, 2)
k_tile_both(const Args x, const Args y, int first)
{
    constexpr int WHOLE = PIECES ? TO_LINEAR_PIECES : TO_LINEAR;
    const int wg = (int)blockIdx.x;
    if (wg < first) {
        if (x.splits > 1) tile_body<64, K_RUNS, ROWS_RUN, false, TO_PARTS>(x, wg, first);
        else tile_body<64, K_RUNS, ROWS_RUN, false, WHOLE>(x, wg, first);
    } else {
        if (y.splits > 1) tile_body<64, ROWS_RUN, ROWS_RUN, false, TO_PARTS>(y, wg - first, (int)gridDim.x - first);
        else tile_body<64, ROWS_RUN, ROWS_RUN, false, WHOLE>(y, wg - first, (int)gridDim.x - first);
    }
}

// The parts of a product whose k was split among workgroups, in order (the sum's bits are the same from run to run), and what
// becomes of their sum.  Bound by memory: four parts of 2048 x 2048 13.2 us (75 MB, 5.7 TB/s).
template <bool GATED> __device__ __forceinline__ void add_parts(const Args &x, int m, int n, float (&z)[8], float (&u)[8])
{
    const long long stride = (long long)x.M * x.parts_pitch;
    const float *p = x.parts + m * x.parts_pitch + n;
    float v[8];
    load8(p, 8, z);
    if constexpr (GATED) load8(p + x.parts_half, 8, u);
    for (int s = 1; s < x.splits; ++s) {
        load8(p + s * stride, 8, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] += v[i];
        if constexpr (GATED) {
            load8(p + s * stride + x.parts_half, 8, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] += v[i];
        }
    }
}

template <bool GATED> __device__ __forceinline__ void join(const Args &x)
{
    const int groups = (x.N + 7) / 8;
    const long long all = (long long)x.M * groups;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < all; t += (long long)gridDim.x * 256) {
        const int m = (int)(t / groups), n = (int)(t % groups) * 8, count = x.N - n;
        float z[8], u[8];
        add_parts<GATED>(x, m, n, z, u);
        if constexpr (GATED) finish_gated8(x.e, m, n, count, z, u);
        else finish_linear8(x.e, m, n, count, z);
    }
}

// fp32 by pieces: a workgroup to 32 rows of 64 columns, of which the sums that are not finite are computed again in LDS.
constexpr int JOIN_PITCH = 68;
constexpr int JOIN_LDS = 32 * JOIN_PITCH;       // floats
template <bool GATED> __device__ __forceinline__ void join_pieces(const Args &x, float *lds)
{
    const int across = (x.N + 63) / 64, r = threadIdx.x >> 3, c = (threadIdx.x & 7) * 8;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long all = (long long)((x.M + 31) / 32) * across;
    for (long long t = blockIdx.x; t < all; t += gridDim.x) {
        const int m0 = (int)(t / across) * 32, n0 = (int)(t % across) * 64, count = x.N - n0 - c;
        const bool there = m0 + r < x.M && count > 0;
        float z[8], u[8];
        bool fine = true;
        if (there) {
            add_parts<GATED>(x, m0 + r, n0 + c, z, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                fine = fine && (e >= count || is_finite(z[e]));
                if constexpr (GATED) fine = fine && (e >= count || is_finite(u[e]));
            }
        }
        if (__syncthreads_or(!fine)) {
            auto mend = [&](int which, float (&v)[8]) {
                store8(lds + r * JOIN_PITCH + c, 8, v);
                __syncthreads();
                if (wave < 2 && n0 + wave * 32 < x.N)
                    mend_block(x.pieces, which, m0, n0 + wave * 32, x.M - m0, x.N - n0 - wave * 32, lds + wave * 32, JOIN_PITCH);
                __syncthreads();
                load8(lds + r * JOIN_PITCH + c, 8, v);
                __syncthreads();
            };
            mend(0, z);
            if constexpr (GATED) mend(1, u);
        }
        if (there) {
            if constexpr (GATED) finish_gated8(x.e, m0 + r, n0 + c, count, z, u);
            else finish_linear8(x.e, m0 + r, n0 + c, count, z);
        }
    }
}

template <bool GATED, bool PIECES> __device__ __forceinline__ void join_parts(const Args &x, float *lds)
{
    if constexpr (PIECES) join_pieces<GATED>(x, lds);
    else join<GATED>(x);
}
template <bool GATED, bool PIECES>
__global__ void __launch_bounds__(256)
k_join(const Args x)
{
    __shared__ __attribute__((aligned(16))) float lds[PIECES ? JOIN_LDS : 1];
    join_parts<GATED, PIECES>(x, lds);
}

// What a backward call's two products leave to be joined, and the bias's column sums.  grid.y = 3.
struct Columns {
    const float *part;              // null: none
    void *out;
    long long pitch;
    int groups, d;
    bool f32;
};
template <bool PIECES>
__global__ void __launch_bounds__(256)
k_join_both(const Args x, const Args y, const Columns c)
{
    __shared__ __attribute__((aligned(16))) float lds[PIECES ? JOIN_LDS : 16 * 17];
    float (&sums)[16][17] = *reinterpret_cast<float (*)[16][17]>(lds);
    if (blockIdx.y == 0) {
        if (x.splits > 1) join_parts<false, PIECES>(x, lds);
    } else if (blockIdx.y == 1) {
        if (y.splits > 1) join_parts<false, PIECES>(y, lds);
    } else if (c.part) {
        for (int b = (int)blockIdx.x; b < (c.d + 15) / 16; b += (int)gridDim.x) {
            if (c.f32) column_sums<float, 16>(c.part, c.pitch, c.groups, c.d, (float *)c.out, b, sums);
            else column_sums<__bf16, 16>(c.part, c.pitch, c.groups, c.d, (__bf16 *)c.out, b, sums);
            __syncthreads();
        }
    }
}

} // namespace tile

// ---- what goes before a product -------------------------------------------------------------------------------------------

// Eight values into a packed operand, from element `at` on: bf16, or the three pieces in planes `plane` elements apart, or
// (PLANES = 0) fp32 as it is.
template <int PLANES> __device__ __forceinline__ void put8(__bf16 *base, long long at, long long plane, const float (&v)[8])
{
    if constexpr (PLANES == 0) {
        store8((float *)base + at, 8, v);
        return;
    }
    __bf16 *p = base + at;
    bf16x8 a, b, c;
    auto cut = [&](auto pieces) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Piece3 q = pieces(v[i]);
            a[i] = __builtin_bit_cast(__bf16, q.a);
            b[i] = __builtin_bit_cast(__bf16, q.b);
            c[i] = __builtin_bit_cast(__bf16, q.c);
        }
    };
    if constexpr (PLANES == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = (__bf16)v[i];
    } else {
        bool ordinary = true;
#pragma unroll
        for (int i = 0; i < 8; ++i) ordinary &= is_ordinary(v[i]);
        if (ordinary) cut([](float f) { return pieces_of_ordinary(f); });
        else cut([](float f) { return pieces_of(f); });
    }
    *reinterpret_cast<bf16x8 *>(p) = a;
    if constexpr (PLANES == 3) {
        *reinterpret_cast<bf16x8 *>(p + plane) = b;
        *reinterpret_cast<bf16x8 *>(p + 2 * plane) = c;
    }
}

// Rows laid out for the tile kernel: a pitch that is a multiple of 64 elements, zeros behind the columns, fp32 in its
// pieces.  grid.y: which matrix.  Bound by memory, and by its launch where small: 2500 x 512 and 2730 x 512 fp32 6.8 us (10.7 MB in, 16 out).
struct PackJob {
    const void *src;
    __bf16 *dst;
    long long ld, pitch, plane;
    int rows, cols;
};
struct PackJobs {
    PackJob job[3];
};
template <typename T, int PLANES>
__global__ void __launch_bounds__(256)
k_pack(const PackJobs jobs)
{
    const PackJob &j = jobs.job[blockIdx.y];
    const int groups = (int)(j.pitch / 8);
    const long long all = (long long)j.rows * groups;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < all; t += (long long)gridDim.x * 256) {
        const long long row = t / groups;
        const int col = (int)(t % groups) * 8;
        float v[8];
        load8((const T *)j.src + row * j.ld + col, j.cols - col, v);
        put8<PLANES>(j.dst, row * j.pitch + col, j.plane, v);
    }
}

// The same for bytes (8-bit elements and their scales): `pitch` bytes to a row, zeros behind the columns.  Only for rows that do
// not lie 16 bytes apart, which the loads into LDS need.
struct ByteJob {
    const uint8_t *src;
    uint8_t *dst;
    long long ld, pitch;
    int rows, cols;
};
struct ByteJobs {
    ByteJob job[6];
};
__global__ void __launch_bounds__(256)
k_pack_bytes(const ByteJobs jobs)
{
    const ByteJob &j = jobs.job[blockIdx.y];
    const int groups = (int)(j.pitch / 4);
    const long long all = (long long)j.rows * groups;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < all; t += (long long)gridDim.x * 256) {
        const long long row = t / groups;
        const int col = (int)(t % groups) * 4;
        const uint8_t *s = j.src + row * j.ld + col;
        unsigned w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < j.cols) w |= (unsigned)s[i] << (8 * i);
        *reinterpret_cast<unsigned *>(j.dst + row * j.pitch + col) = w;
    }
}

// 8-bit rows as packed bf16 (exact), for the products of too short a k for the scaled matrix instruction.
struct WidenJob {
    const uint8_t *src, *scale;
    __bf16 *dst;
    long long ld, ld_scale, pitch;
    int rows, cols;
};
struct WidenJobs {
    WidenJob job[3];
};
__global__ void __launch_bounds__(256)
k_widen(const WidenJobs jobs)
{
    const WidenJob &j = jobs.job[blockIdx.y];
    const int groups = (int)(j.pitch / 8);
    const long long all = (long long)j.rows * groups;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < all; t += (long long)gridDim.x * 256) {
        const long long row = t / groups;
        const int col = (int)(t % groups) * 8, count = j.cols - col;
        const uint8_t *s = j.src + row * j.ld + col;
        uint2 w = make_uint2(0, 0);
        if (count >= 8) {
            const u32x2_any t = *reinterpret_cast<const u32x2_any *>(s);
            w = make_uint2(t[0], t[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) (i < 4 ? w.x : w.y) |= (unsigned)s[i] << (8 * (i & 3));
        }
        const float scale = count > 0 ? mx_scale(j.scale[row * j.ld_scale + col / MX_BLOCK]) : 0.f;
        bf16x8 v = widen8(w.x, w.y, scale);
        // (a NaN scale is no business of what lies behind the columns)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < count ? v[i] : (__bf16)0.f;
        *reinterpret_cast<bf16x8 *>(j.dst + row * j.pitch + col) = v;
    }
}

// dz = dy act'(z), packed, and its column sums over a group of rows.  A thread owns eight columns; `across` threads of a
// workgroup lie side by side, the others take further rows.  grid = (column pieces, groups).  Bound by memory: 16384 x 2048, z in fp32, 60 us
// (268 MB, 4.5 TB/s).
struct SlopeArgs {
    const void *dy;
    const float *z;                 // preact; gated: g and u side by side
    __bf16 *dz;                     // packed (null: column sums alone); gated: dg, and du `half` columns on
    float *part;                    // [group][part_pitch], nullable
    long long ld_dy, ld_z, pitch, plane, part_pitch;
    int M, N, across, half;
};
template <typename T, int PLANES, int ACT>
__global__ void __launch_bounds__(256)
k_slope(const SlopeArgs x)
{
    __shared__ float sums[256][9];
    const int c = threadIdx.x % x.across, r = threadIdx.x / x.across, down = 256 / x.across;
    const int n = (blockIdx.x * x.across + c) * 8, count = x.N - n;
    float sum[8] = {};
    if (n < x.pitch) {
        for (long long m = (long long)blockIdx.y * down + r; m < x.M; m += (long long)gridDim.y * down) {
            float v[8];
            load8((const T *)x.dy + m * x.ld_dy + n, count, v);
            if constexpr (ACT != 0) {
                float z[8];
                load8(x.z + m * x.ld_z + n, count, z);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float value, slope;
                    activate_both_as<ACT>(z[i], &value, &slope);
                    v[i] = i < count ? v[i] * slope : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
            if (x.dz) put8<PLANES>(x.dz, m * x.pitch + n, x.plane, v);
        }
    }
    if (!x.part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = sum[i];
    __syncthreads();
    if (r == 0 && count > 0) {
        for (int k = 1; k < down; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += sums[k * x.across + c][i];
        store8(x.part + (size_t)blockIdx.y * x.part_pitch + n, 8, sum);
    }
}

// dg = dh u act'(g) and du = dh act(g), packed side by side.  Bound by memory: 16384 x 8192 354 us (1.88 GB, 5.3 TB/s).
template <typename T, int PLANES, int ACT>
__global__ void __launch_bounds__(256)
k_gated_slope(const SlopeArgs x)
{
    const int c = threadIdx.x % x.across, r = threadIdx.x / x.across, down = 256 / x.across;
    const int n = (blockIdx.x * x.across + c) * 8, count = x.N - n;
    if (n >= x.half) return;
    for (long long m = (long long)blockIdx.y * down + r; m < x.M; m += (long long)gridDim.y * down) {
        float d[8], lo[8], hi[8], dg[8], du[8];
        load8((const T *)x.dy + m * x.ld_dy + n, count, d);
        const float *s = x.z + m * x.ld_z + 2 * (long long)n;
        load8(s, 2 * count, lo);
        load8(s + 8, 2 * count - 8, hi);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float g = i < 4 ? lo[2 * i] : hi[2 * i - 8], u = i < 4 ? lo[2 * i + 1] : hi[2 * i - 7];
            float value, slope;
            activate_both_as<ACT>(g, &value, &slope);
            dg[i] = i < count ? d[i] * u * slope : 0.f;
            du[i] = i < count ? d[i] * value : 0.f;
        }
        put8<PLANES>(x.dz, m * x.pitch + n, x.plane, dg);
        put8<PLANES>(x.dz, m * x.pitch + x.half + n, x.plane, du);
    }
}

// Zeros where there is no row to sum over (a fill of its own: a captured memset may not replay right).
template <typename T>
__global__ void __launch_bounds__(256)
k_zero(T *__restrict__ p, long long ld, int rows, int cols)
{
    for (long long i = blockIdx.x; i < rows; i += gridDim.x)
        for (int c = threadIdx.x; c < cols; c += 256) p[i * ld + c] = (T)0.f;
}

} // namespace enc

// An fp32 number as three bf16: plain code for host and device, so that it can be tested without a device.
#pragma once
#include <cstdint>

#if defined(__HIPCC__)
#define ENC_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define ENC_HOST_DEVICE inline
#endif

namespace enc {

struct Piece3 {
    uint16_t a, b, c;       // bf16
};

ENC_HOST_DEVICE uint32_t bits_of(float v) { return __builtin_bit_cast(uint32_t, v); }
ENC_HOST_DEVICE float of_bf16(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }

// The bf16 nearest to v (finite), ties to even.
ENC_HOST_DEVICE uint16_t nearest_bf16(float v)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(uint16_t, (__bf16)v);
#else
    return (uint16_t)((bits_of(v) + 0x7fffu + ((bits_of(v) >> 16) & 1u)) >> 16);
#endif
}

// Whether the nearest bf16 to v is finite.
ENC_HOST_DEVICE bool is_ordinary(float v) { return (bits_of(v) & 0x7fffffffu) < 0x7f7f8000u; }

// v = a + b + c, exactly (but for what lies below bf16's least number).  Each piece is the nearest to what is left, so |b| <= 2^-8 and
// |c| <= 2^-17 of v's power of two, of either sign.
ENC_HOST_DEVICE Piece3 pieces_of_ordinary(float v)
{
    Piece3 p;
    p.a = nearest_bf16(v);
    const float r = v - of_bf16(p.a);
    p.b = nearest_bf16(r);
    p.c = nearest_bf16(r - of_bf16(p.b));
    return p;
}
// The same for any v.  Where the nearest to a finite v is infinite, the largest below it is taken; of what is not finite the first
// piece says all.
ENC_HOST_DEVICE Piece3 pieces_of(float v)
{
    if (is_ordinary(v)) return pieces_of_ordinary(v);
    const uint32_t bits = bits_of(v);
    Piece3 p{(uint16_t)(bits >> 16), 0, 0};
    if ((bits & 0x7f800000u) == 0x7f800000u) {
        if (bits & 0x7fffffu) p.a |= 0x40u;
        return p;
    }
    const float r = v - of_bf16(p.a);
    p.b = nearest_bf16(r);
    p.c = nearest_bf16(r - of_bf16(p.b));
    return p;
}

// The pairs of pieces whose products make up an fp32 product, smallest first.  The dropped ones, (1, 2), (2, 1) and (2, 2), are
// at most 2^-24 (1 + 2^-10) of the product's size together, of either sign: over two million random pairs up to 2^-24.2, in the mean
// 4e-5 of 2^-24.
// (Pieces cut off instead of rounded would leave up to 2^-21, always of the product's own sign.)
constexpr int PIECE_PAIRS[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};

} // namespace enc

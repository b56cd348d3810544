// Random bits by counter: Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011).  Any element's bits follow from (seed, step, layer, index) alone, so a dropout mask is made where it is needed
// and never stored.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define PHILOX_FN __host__ __device__ inline
#else
#define PHILOX_FN inline
#endif

struct Words4 { uint32_t w[4]; };

PHILOX_FN uint32_t xor3(uint32_t a, uint32_t b, uint32_t c)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);      // (one instruction, which the compiler does not find by itself)
#else
    return a ^ b ^ c;
#endif
}

PHILOX_FN Words4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = xor3((uint32_t)(p1 >> 32), c1, k0);
        c1 = (uint32_t)p1;
        c2 = xor3((uint32_t)(p0 >> 32), c3, k1);
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// What a dropout is made of.  Eight elements share a counter: element e takes the 16 bits number e % 8 of group e / 8 and is
// kept where they are at least `limit`; what is kept is multiplied by `factor`, the inverse of the kept share, exactly that of
// the limit, so that the mean stays.
struct DropRule {
    uint32_t k0, k1, s0, s1, limit;
    float factor;
};

PHILOX_FN Words4 drop_bits(const DropRule &d, uint64_t group, uint32_t layer)
{
    return philox((uint32_t)group, (uint32_t)(group >> 32) | layer << 16, d.s0, d.s1, d.k0, d.k1);
}
PHILOX_FN bool drop_keeps(const DropRule &d, const Words4 &bits, int place)
{
    const uint32_t half = place & 1 ? bits.w[place >> 1] >> 16 : bits.w[place >> 1] & 0xffffu;
    return half >= d.limit;
}
// The limit for a share p, 0 <= p < 1; 65536 where nothing would be kept.
PHILOX_FN uint32_t drop_limit(double p)
{
    const double x = p * 65536.0;
    uint32_t t = (uint32_t)x;                               // to the nearest whole number, ties to even
    const double rest = x - (double)t;
    if (rest > 0.5 || (rest == 0.5 && (t & 1u))) ++t;
    return t;
}

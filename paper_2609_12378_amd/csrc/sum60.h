// Sums of products of residues below 2^60, one reduction a sum: what the basis conversions of the integer arithmetic
// spend their time on.
//
// Both factors split into halves of 30 bits, so the four partial products, below 2^60 each, add up in three 64-bit
// words without carries: ll and hh of up to 15 products and mid, two a product, of up to 8.  A product is four 32-bit
// multiply-adds and nothing else, where an exact 128-bit sum adds more carries and moves than that.  The sum S, at most
// 2^64 q, is divided by 2^64 modulo q (Montgomery 1985: one low and one high product, seven multiplies where reduce128
// takes twenty), so the constants carry a factor 2^64 from where they are staged.
#pragma once
#include "modarith.h"

struct Mod60 {
    uint64_t q, qinv;   // qinv q = 1 mod 2^64
};
__device__ __forceinline__ Mod60 mod60(uint64_t q)
{
    // q q = 1 mod 8 for odd q, and a Newton step doubles the bits: 3, 6, 12, 24, 48, 96
    uint64_t v = q;
#pragma unroll
    for (int i = 0; i < 5; i++) v *= 2 - q * v;
    return Mod60{q, v};
}

// the halves of a value below 2^60
__device__ __forceinline__ uint2 halves(uint64_t v)
{
    return make_uint2((uint32_t)v & 0x3FFFFFFFu, (uint32_t)(v >> 30));
}
// v 2^64 mod q for a staged constant
__device__ __forceinline__ uint64_t times_2_64(uint64_t v, const ModQ &m) { return reduce128(acc128{0, v}, m); }

struct Sum60 {
    uint64_t ll = 0, mid = 0, hh = 0;
    __device__ __forceinline__ void add(uint2 a, uint2 b)
    {
        ll += (uint64_t)a.x * b.x;
        mid += (uint64_t)a.x * b.y;
        mid += (uint64_t)a.y * b.x;
        hh += (uint64_t)a.y * b.y;
    }
    // n b of a small n
    __device__ __forceinline__ void add(uint32_t n, uint2 b)
    {
        ll += (uint64_t)n * b.x;
        mid += (uint64_t)n * b.y;
    }
    __device__ __forceinline__ acc128 value() const
    {
        const unsigned __int128 s = ((unsigned __int128)hh << 60) + ((unsigned __int128)mid << 30) + ll;
        return acc128{(uint64_t)s, (uint64_t)(s >> 64)};
    }
};

// s / 2^64 mod q, canonical: s < 2^64 q
__device__ __forceinline__ uint64_t redc(acc128 s, const Mod60 &m)
{
    const uint64_t r = s.hi - mulhi64(s.lo * m.qinv, m.q);
    return (int64_t)r < 0 ? r + m.q : r;
}

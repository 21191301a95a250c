// The order of a row's positions over a half wave that the fused row passes of sums work in (wsum.hip, step_f64.hip).
#pragma once
#include "wsum_args.h"

namespace wsum {

using nttc::kE8;

// The positions of thread t (of 32) in a row of 256: pairs (j, j + 1) at j = 64 c + 4 (t & 15) + 2 (t >> 4), register
// e = 2 c + (0 or 1), so a wave's access is whole cache lines.  It is the layout that the transforms end in and inverse
// ones start from (nttc::u8<2>, four adjacent positions a thread) with position bits 1 and 6 exchanged, which is one
// swap of lane rows a register (swap_1_6).
// sigma_g reads position j at j' with 2 brev(j') + 1 = (2 brev(j) + 1) g mod 2N.  Bit 0 of j is the top bit of
// 2 brev(j) + 1 modulo 2N, which an odd g leaves in place up to a carry from below: the partner j + 1 of an even j is
// read at j' ^ 1; likewise the sources of 64 aligned positions are 64 aligned positions.  So gathers are pairs and
// whole lines as well.  (8-byte accesses, or 16-byte ones at a stride of 32, cost twice the requests to L2, which bound
// the kernels.)
struct Positions {
    uint32_t at, log_n;
    __device__ Positions(uint32_t h, uint32_t t, uint32_t log_n_)
        : at(h * 256 + 4 * (t & 15u) + 2 * (t >> 4)), log_n(log_n_)
    {
    }
    __device__ uint32_t pos(int e) const { return at + 64u * (uint32_t)(e >> 1) + (uint32_t)(e & 1); }
    __device__ uint32_t start(uint32_t g) const { return (2u * (__brev(at) >> (32 - log_n)) + 1u) * g; }
    // j' of pos(e), e even; kg = start(g).  Bits 6 and 7 of the position add 2^(log_n - 6) g and 2^(log_n - 7) g.
    __device__ uint32_t source(uint32_t kg, uint32_t g, int e) const
    {
        const uint32_t dk = ((uint32_t)(e & 2) << (log_n - 7)) + ((uint32_t)(e >> 2) << (log_n - 7));
        return (__brev(kg + dk * g) >> (31 - log_n)) & ((1u << log_n) - 1);
    }
};
// u8<2> to Positions' order and back: registers e and e | 2 (e & 2 clear) exchange lane rows 1 (of e) and 0 (of e | 2)
__device__ __forceinline__ void swap_1_6(double (&x)[kE8])
{
#pragma unroll
    for (int e = 0; e < kE8; e++) {
        if (e & 2) continue;
        const uint64_t a = A::to_raw(x[e]), b = A::to_raw(x[e | 2]);
        const auto lo = __builtin_amdgcn_permlane16_swap((uint32_t)a, (uint32_t)b, false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((uint32_t)(a >> 32), (uint32_t)(b >> 32), false, false);
        x[e] = A::from_raw((uint64_t)hi[0] << 32 | lo[0]);
        x[e | 2] = A::from_raw((uint64_t)hi[1] << 32 | lo[1]);
    }
}

}  // namespace wsum

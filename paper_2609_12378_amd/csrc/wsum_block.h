// What the whole-row kernels that divide sums by P q_l share (wsum_block.hip, step_block.hip).
#pragma once
#include "ntt_block.h"
#include "wsum_args.h"

namespace wsum {

using nttc::GridSum;
using nttc::kE;

struct Tab {
    const ModQ *mods;
    const double *twf, *itwf;
};

// v = sum_i y_i m(i) mod q, |v| <= q/2 + 1, at a thread's 16 points of the K digit rows that follow yr
template <int LOGN, typename Factor>
__device__ __forceinline__ void digit_sums(double (&v)[kE], const uint64_t *yr, const Dims &d, const A &ar, Factor m)
{
    const uint32_t t = threadIdx.x;
    const int K = (int)d.K;
#pragma unroll
    for (int e0 = 0; e0 < kE; e0 += 8) {
        GridSum acc[8];
        // two sources' loads at a time
        for (int s = 0; s < K; s += 2) {
            double y[2][8];
#pragma unroll
            for (int h = 0; h < 2; h++)
#pragma unroll
                for (int e = 0; e < 8; e++)
                    y[h][e] = A::from_raw(yr[((size_t)min(s + h + 1, K) << LOGN) + blk::col_pos<LOGN>(t, e0 + e)]);
            if (s && s % GridSum::kTerms == 0) {
#pragma unroll
                for (int e = 0; e < 8; e++) acc[e].fold(ar);
            }
#pragma unroll
            for (int h = 0; h < 2; h++) {
                if (s + h >= K) break;
                const double w = m(s + h);
#pragma unroll
                for (int e = 0; e < 8; e++) acc[e].add(y[h][e], w);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e++) v[e0 + e] = ar.red(acc[e].value(ar));
    }
}

}  // namespace wsum

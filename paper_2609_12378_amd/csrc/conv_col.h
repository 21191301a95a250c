// A basis conversion with the forward column pass of its target, 16 points of a 2^LOGS-point column a thread (256
// threads, 4096 / 2^LOGS columns).  Each target reads its tile of the sources again, which no registers hold, so ring
// and number of sources are free; with the targets of a tile one after the other on one XCD those reads meet its L2.
#pragma once
#include "ckks_internal.h"
#include "ntt_core.h"

// Worth it while the reads, tiles of 4096 coefficients times targets times sources, are few: `most`.  us a call in two
// launches and in one, rotary positions of 1 to 16 ciphertexts for the ModUps, hoisted rotations for the ModDowns:
//   ModUps    2^14, 9 limbs in digits of 4: 101 and 95 (2880 reads); 2^15, 6 limbs of 2: 242 and 221 (5376), 16 limbs of 8:
//             176 and 174 (11776), 318 and 312 (23552); 2^16, 10 limbs of 10: 357 and 354 (12800), 642 and 641 (25600);
//             2^14, 24 limbs of 8: 464 and 465 (47616)
//   ModDowns  2^14, 11 limbs and 4 special primes: 96 and 88 (2816), 221 and 205 (11264); 24 and 8: 161 and 157 (12288),
//             259 and 258 (24576), 440 and 445 (49152)
constexpr size_t kConvColReads = 16384;
inline bool conv_col_few(const ckks_ctx *ctx, uint32_t polys, uint32_t sources, uint32_t targets,
                         size_t most = kConvColReads)
{
    return ((size_t)polys << (ctx->log_n - 12)) * targets * sources <= most;
}

namespace nttc {

template <int LOGS>
struct ColTile {
    static constexpr uint32_t TS = (1u << LOGS) / 16, kCols = 4096u >> LOGS, kTiles = 256 / kCols;   // tiles a row
    static constexpr uint32_t kLds = LOGS > 4 ? kCols * ((1u << LOGS) + (1u << LOGS) / 16 + 1) : 1;
    uint32_t col, t, at;
    __device__ explicit ColTile(uint32_t tile)
        : col(threadIdx.x % kCols), t(threadIdx.x / kCols), at(tile * kCols + col)
    {
    }
    __device__ void load(double (&x)[kE], const uint64_t *row) const
    {
#pragma unroll
        for (int k = 0; k < kE; k++) x[k] = Ar<true>::from_raw(row[at + (size_t)(t + TS * k) * 256]);
    }
    // S sums x[s] = sum_i (row src + i N) m[s][i stride[s]] modulo ar[s], i < ns, lazily reduced (GridSum::value); the
    // next row is asked for ahead
    template <int S>
    __device__ void sum(double (&x)[S][kE], const uint64_t *src, uint32_t log_n, uint32_t ns,
                        const double *const (&m)[S], const uint32_t (&stride)[S], const Ar<true> (&ar)[S]) const
    {
        double next[kE];
        load(next, src);
        GridSum acc[S][kE];
#pragma unroll 1
        for (uint32_t i = 0; i < ns; i++) {
#pragma unroll
            for (int k = 0; k < kE; k++) x[0][k] = next[k];
            if (i + 1 < ns) load(next, src + ((size_t)(i + 1) << log_n));
#pragma unroll
            for (int s = 0; s < S; s++) {
                const double f = m[s][i * stride[s]];
#pragma unroll
                for (int k = 0; k < kE; k++) acc[s][k].add(x[0][k], f);
                if ((i & 7u) == 7u && i + 1 < ns)
#pragma unroll
                    for (int k = 0; k < kE; k++) acc[s][k].fold(ar[s]);
            }
        }
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int k = 0; k < kE; k++) x[s][k] = acc[s][k].value(ar[s]);
    }
    // forward column pass of reduced values, the stages of kMask reducing; raw doubles out
    template <unsigned kMask>
    __device__ void forward(double (&x)[kE], uint64_t *row, const double *tw, double *lds, const Ar<true> &ar) const
    {
        fwd_top<true, kMask>(x, tw, 1, ar);
        if (LOGS > 4) {
            transpose<LOGS, true>(x, lds, col, t);
            fwd_low<LOGS, true, kMask>(x, tw, 1, t, ar);
        }
#pragma unroll
        for (int k = 0; k < kE; k++) row[at + (size_t)(LOGS > 4 ? 16 * t + k : k) * 256] = Ar<true>::to_raw(x[k]);
    }
};

// block b of a launch of `targets` blocks a tile: the tile's blocks follow one another on one XCD
__device__ __forceinline__ void target_of(uint32_t targets, uint32_t &tile, uint32_t &tt)
{
    const uint32_t xcd = blockIdx.x & 7u, rest = blockIdx.x >> 3;
    tt = rest % targets;
    tile = (rest / targets) * 8 + xcd;
}

}  // namespace nttc

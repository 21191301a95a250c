// Arguments and arithmetic that the weighted-sum kernels share (wsum.hip, wsum_block.hip).
#pragma once
#include "ks_args.h"
#include "wsum.h"

namespace wsum {

using A = nttc::Ar<true>;

struct Ct {
    const uint64_t *c, *dig;   // [2][L][N]; its ModUp digits [nd][ext][N] (rotated kinds)
    uint64_t *out[kWsumPages];
    const uint64_t *prev[kWsumPages];
    uint32_t kind;
};
struct Args {
    WsumKind kind[kWsumKinds];
    Ct ct[kWsumCts];
};

// The ring's sizes: L = level + 1 q-limbs, K special primes, ext = L + K, nd digits
struct Dims {
    uint32_t L, K, ext, nd, alpha, n_q, key_rows, log_n;
    __device__ uint32_t prime(uint32_t row) const { return row < L ? row : n_q + (row - L); }
};

// Two adjacent words, read and written in one 16-byte access (rows are 8-byte aligned).
struct __attribute__((aligned(8))) Pair {
    uint64_t x, y;
};
__device__ __forceinline__ Pair ld2(const uint64_t *p) { return *(const Pair *)p; }

// Block b of a launch over `tiles` tiles (a multiple of 8) of each of n ciphertexts: blocks go to the 8 XCDs in turn,
// and the ciphertexts of one tile, which share its keys and tables, follow one another on one XCD (16 of 13 limbs:
// k_wsum_intt8 122 us against 178 with one ciphertext after the other, k_wsum_fin8 198 against 312; two of 37 limbs in
// integers: k_wsum 195 against 284).
__device__ __forceinline__ void tile_of(uint32_t n, uint32_t &z, uint32_t &tile)
{
    const uint32_t xcd = blockIdx.x & 7u, rest = blockIdx.x >> 3;
    z = rest % n;
    tile = (rest / n) * 8 + xcd;
}

// sum_i a_i w_i mod q of at most 4 products of canonical residues under one quotient (nttc::GridSum with twice its
// grid: u = 2^51, so |sum| < 4 2^100 = 2^51 u, and lo is at most 4 2^50 = 2^52).  value(): |x| <= q/2 + 1.
struct ProductSum {
    static constexpr double kGrid = 0x1.8p+103;   // 1.5 2^52 u
    double hi, lo;
    __device__ ProductSum() : hi(kGrid), lo(0.0) {}
    __device__ void add(double a, double w)
    {
        const double t = fma(a, w, hi);
        const double h = t - hi;
        lo += fma(a, w, -h);
        hi = t;
    }
    __device__ double value(const A &ar) const
    {
        const double h = hi - kGrid;
        return ar.red(fma(-rint(h * ar.qinv), ar.q, h) + lo);
    }
    __device__ void fold(const A &ar)
    {
        lo = value(ar);
        hi = kGrid;
    }
};

// the integer r in [0, 2^52) as a word: the mantissa of 2^52 + r
__device__ __forceinline__ uint64_t to_word(double r)
{
    return (uint64_t)__double_as_longlong(r + 4503599627370496.0) & 0x000FFFFFFFFFFFFFull;
}

// x f mod q, canonical: |x| < 8 q reduced to q/2 + 1, times f in [0, q) at most 0.7 q
__device__ __forceinline__ uint64_t quotient(const A &ar, double x, double f)
{
    const double r = ar.mul(ar.red(x), f);
    return to_word(r < 0.0 ? r + ar.q : r);
}

// (-q/2, q/2] of |x| < q/2 + 2^49: the centred representative of an odd modulus
__device__ __forceinline__ double centre(const A &ar, double x)
{
    const double v = ar.red(x), h = 0.5 * ar.q;
    return v > h ? v - ar.q : v < -h ? v + ar.q : v;
}

// The division's constants: y_i takes N^-1 Qhat_i^-1, the q_l row N^-1 P^-1 (N^-1 alone for unrotated kinds)
struct Quot {
    const double *qhat_inv;    // [K]
    const double *qhat_mod;    // [K][L] centred
    const ulonglong2 *pinv, *qlinv, *pmodq;
};

// factor of source i in the conversion to q_l divided by P, [P / p_i P^-1]_{q_l}, centred
__device__ __forceinline__ double top_factor(const Quot &qt, const Dims &d, int i, const A &top)
{
    return centre(top, top.mul(qt.qhat_mod[i * d.L + d.L - 1], (double)qt.pinv[d.L - 1].x));
}

}  // namespace wsum

inline wsum::Dims wsum_dims(const ckks_ctx *ctx, uint32_t L)
{
    return wsum::Dims{L, ctx->n_p, L + ctx->n_p, n_digits(ctx, L - 1), ctx->alpha, ctx->n_q, ctx->n_primes(), ctx->log_n};
}

// The division by P q_l (q_l alone: unrotated kinds) of sums that are there, between their inverse row pass and their
// forward one (wsum.hip, two passes).  Of a it reads whose kinds are rotated.
ckks_status wsum_convert(ckks_ctx *ctx, const wsum::Args &a, uint32_t n, uint32_t pages, const wsum::Dims &d, uint64_t *up,
                         uint64_t *cw);

// N = 2^12 and 2^13 (wsum_block.hip): the sums and the division of n ciphertexts whose digits are formed;
// u: 2 n pages (level+1+n_p) N words
ckks_status wsum_blk_sums(ckks_ctx *ctx, const wsum::Args &a, uint32_t n, uint32_t pages, const wsum::Dims &d, uint64_t *u);
// ... from u that is there (raw doubles of at most q/2 + 1) to the outputs
ckks_status wsum_blk_divide(ckks_ctx *ctx, const wsum::Args &a, uint32_t n, uint32_t pages, const wsum::Dims &d,
                            uint64_t *u);

// Any ring and any primes (wsum_exact.hip): the same in exact 128-bit sums, of ciphertexts that are all of rotated
// kinds (rot) or all of unrotated ones; a.ct[z].dig's own rows are not read.  u: 2 n pages (level+1+n_p) N words, x: 2
// n pages level N
ckks_status wsum_exact_sums(ckks_ctx *ctx, const wsum::Args &a, uint32_t n, uint32_t pages, const wsum::Dims &d, bool rot,
                            uint64_t *u, uint64_t *x);
// ... from u that is there to the outputs
ckks_status wsum_exact_divide(ckks_ctx *ctx, const wsum::Args &a, uint32_t n, uint32_t pages, const wsum::Dims &d, bool rot,
                              uint64_t *u, uint64_t *x);
// c1 of the first n ciphertexts to out[n][L][N]
ckks_status wsum_gather_c1(ckks_ctx *ctx, const wsum::Args &a, uint32_t n, uint32_t L, uint64_t *out);

// Arguments that the kernels of steps share (step.hip, step_f64.hip).
#pragma once
#include "step.h"
#include "wsum_args.h"

namespace steps {

// What a step's product is: none, of ciphertexts, of a ciphertext and a plaintext, a sum of products that is there
enum : uint32_t { kNone = 0, kProduct = 1, kPlain = 2, kGiven = 3 };

// A step's operands as they travel in a launch's arguments.  Counts share words: a byte of the arguments is not a scalar
// load, and waiting for it is waiting for every load before it.
struct Operands {
    const uint64_t *a, *b, *z[kStepTerms];       // a: the sum [3][L][N] of a kGiven step
    uint64_t *out;
    int64_t k[kStepTerms + 1];                   // the terms' integers, then the constant's
    uint32_t term[kStepTerms + 1];               // their shifts, limbs and polynomials
    uint32_t info;                               // terms, kind, limbs of a and of b
    int32_t mult;
    __host__ __device__ uint32_t n() const { return info & 0xff; }
    __host__ __device__ uint32_t kind() const { return info >> 8 & 0xff; }
    __host__ __device__ uint32_t a_limbs() const { return info >> 16 & 0xff; }
    __host__ __device__ uint32_t b_limbs() const { return info >> 24; }
    __host__ __device__ bool switched() const { return kind() == kProduct || kind() == kGiven; }
    __device__ uint32_t sh(uint32_t i) const { return term[i] & 0xff; }
    __device__ uint32_t limbs(uint32_t i) const { return term[i] >> 8 & 0xff; }
    __device__ bool two(uint32_t i) const { return term[i] >> 16 == 2; }
};
struct Batch {
    Operands s[kStepBatch];
};
static_assert(sizeof(Batch) <= 4096 - 256, "a batch travels in the kernel arguments");

// m 2^sh mod q
__device__ __forceinline__ uint64_t int_mod(int64_t m, uint32_t sh, uint64_t q)
{
    const uint64_t a = m < 0 ? 0 - (uint64_t)m : (uint64_t)m;
    uint64_t r = a % q;
    for (uint32_t i = 0; i < sh; i++) r = csub(2 * r, q);
    return m < 0 && r ? q - r : r;
}
// The same in doubles, |m| <= 2^62 and q < 2^50: the two halves of m are exact, and x - c q below q where c is at most a
// unit off.
__device__ __forceinline__ double int_mod(int64_t m, uint32_t sh, const wsum::A &ar)
{
    const double hi = ar.red((double)(m >> 31) * 0x1p31);
    double r = ar.red(hi + (double)(m & 0x7fffffff));
    for (uint32_t i = 0; i < sh; i++) r = ar.red(2.0 * r);
    return r < 0.0 ? r + ar.q : r;
}

}  // namespace steps

// the products d2 of the first n_sw steps, as a ModUp reads them
PolyProd step_sources(const ckks_ctx *ctx, uint32_t L, const steps::Batch &b, uint32_t n_sw);

// n steps at L >= 2 limbs, of which the first n_sw switch a key, in `mem` of step_scratch_words(ctx, L, n, n_sw > 0) words:
// fp64 arithmetic (f64_switch) in two passes a transform, N >= 2^14 (step_f64.hip) ...
ckks_status step_f64(ckks_ctx *ctx, uint32_t L, const steps::Batch &b, uint32_t n, uint32_t n_sw, const uint64_t *rlk,
                     uint64_t *mem);
// ... or in whole rows, N = 2^12 and 2^13 (step_block.hip)
ckks_status step_blk(ckks_ctx *ctx, uint32_t L, const steps::Batch &b, uint32_t n, uint32_t n_sw, const uint64_t *rlk,
                     uint64_t *mem);

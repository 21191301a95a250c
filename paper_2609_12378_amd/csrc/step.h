// The step that polynomials, norms and the projection's epilogue are made of (step.hip), of ciphertexts at l + 1 = L limbs:
//
//   (d0, d1, d2) = m (a0 b0, a0 b1 + a1 b0, a1 b1) + sum_i k_i (z0, z1, 0)_i
//   out          = Rescale((d0, d1) + ModDown(<ModUp(d2), rlk>)) + c
#pragma once
#include <vector>

#include "ckks_internal.h"

// the integer m 2^sh
struct StepInt {
    int64_t m = 0;
    uint32_t sh = 0;
};
// The integer nearest to x (ties to even); false: x is not finite or 2^120 and more.
bool step_int(double x, StepInt *out);

constexpr uint32_t kStepTerms = 9;    // linear terms of a step: T_1 .. T_7, a remainder or T_8, a residual
constexpr uint32_t kStepBatch = 16;   // steps a launch

struct StepTerm {
    const uint64_t *z;        // [polys][limbs][N], limbs >= L; one polynomial counts for d0
    uint32_t limbs, polys;
    StepInt k;
};
struct Step {
    // a product (a null: none): b a ciphertext or (b_polys 1) a plaintext, which needs no key; limbs >= L
    const uint64_t *a = nullptr, *b = nullptr;
    uint32_t a_limbs = 0, b_limbs = 0, b_polys = 2;
    int32_t mult = 1;         // 1, 2 or -1; of a product with a plaintext 1
    // or a sum of products [3][L][N]
    const uint64_t *d = nullptr;
    uint32_t n_terms = 0;     // more than kStepTerms are counted and not kept: step_run refuses them
    StepTerm t[kStepTerms];
    StepInt c;
    uint64_t *out = nullptr;  // [2][L - 1][N]; overlaps no operand of the call's steps

    bool switched() const { return d || (a && b_polys == 2); }
    void product(const uint64_t *a_, uint32_t al, const uint64_t *b_, uint32_t bl, int32_t m = 1, uint32_t bp = 2)
    {
        a = a_, a_limbs = al, b = b_, b_limbs = bl, mult = m, b_polys = bp;
    }
    void term(const StepTerm &s)
    {
        if (n_terms < kStepTerms) t[n_terms] = s;
        n_terms++;
    }
    void term(const uint64_t *z, uint32_t limbs, StepInt k, uint32_t polys = 2) { term(StepTerm{z, limbs, polys, k}); }
};

// words of scratch for up to `steps` steps at L limbs; switched: some have a product of ciphertexts
size_t step_scratch_words(const ckks_ctx *ctx, uint32_t L, uint32_t steps, bool switched = true);
// Every step, independent of the others; rlk may be null where none has a product of ciphertexts.
ckks_status step_run(ckks_ctx *ctx, uint32_t L, const std::vector<Step> &steps, const uint64_t *rlk, uint64_t *mem);
// d [3][L][N] = sum_j the products of a[j] ([2][limbs][N], limbs >= L) with itself
ckks_status step_squares(ckks_ctx *ctx, uint32_t L, const std::vector<const uint64_t *> &a, uint32_t limbs, uint64_t *d);

// sum_i c_i T_i of ciphertexts holding T_1 (cheb.hip): what is computed at which depth below T_1's level
struct ChebTerm {
    uint32_t of;              // an earlier object
    StepInt k;
};
struct ChebObj {
    uint32_t depth;           // L1 - depth limbs
    int x = -1, y = -1;       // the product of these objects
    int32_t mult = 1;
    std::vector<ChebTerm> t;
    StepInt c;
    double scale = 0;
};
struct ChebPlan {
    uint32_t L1, depth;       // limbs of T_1; levels of the sum below it
    std::vector<ChebObj> obj; // 0: T_1; the last: the sum
};
inline uint32_t cheb_depth(uint32_t degree)
{
    uint32_t d = 0;
    while (degree >> d) d++;
    return d;
}
constexpr uint32_t kChebDegree = 127;
// coefs (degree + 1, or null: zeros) of T_1 at scale s1 with L1 > cheb_depth(degree) limbs, the sum at scale `target`
ckks_status cheb_plan(const ckks_ctx *ctx, const double *coefs, uint32_t degree, uint32_t L1, double s1, double target,
                      const char *what, ChebPlan *out);
size_t cheb_scratch_words(const ckks_ctx *ctx, const ChebPlan &plan, uint32_t cts);
// The sums of T_1 at t1[r] into out[r] ([2][L1 - depth][N]); extra (empty, or one a ciphertext): a term of the last step.
ckks_status cheb_run(ckks_ctx *ctx, const ChebPlan &plan, const std::vector<const uint64_t *> &t1,
                     const std::vector<uint64_t *> &out, const std::vector<StepTerm> &extra, const uint64_t *rlk,
                     uint64_t *mem);

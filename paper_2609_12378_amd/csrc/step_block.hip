// Steps (step.h) in the rings of 2^12 and 2^13 points with fp64 arithmetic, whole rows in a block (ntt_block.h): the two
// launches of the ModUp, which forms the products d2 where it reads them, k_step_sums, and the division by P q_l in two
// (wsum_block.hip).
#include "ops.h"
#include "step_args.h"

namespace {

using namespace wsum;
using namespace steps;

// u = P (d0, d1) + <digits, rlk> (wsum.hip) on every row, raw doubles of at most q/2 + 1: one position a thread, the loads
// of a step's product, of its digits and of their keys issued before the first product.  Formed where they are used, a
// row a block, the sums take a launch less and as long: a thread there has 16 positions, whose words do not fit the
// registers together, and a round trip to memory for each operand in turn (one ciphertext of 4 limbs at N = 2^12: 12.5 us
// in either of two launches).
template <int ND>
__global__ __launch_bounds__(256) void k_step_sums(Batch bt, const uint64_t *dig, const uint64_t *rlk, uint64_t *u, Dims d,
                                                   const ulonglong2 *__restrict__ pmodq, const ModQ *__restrict__ mods)
{
    constexpr int kDig = ND > 0 ? ND : 1;
    const uint32_t pos = blockIdx.x * 256 + threadIdx.x, row = blockIdx.y, z = blockIdx.z;
    const Operands &s = bt.s[z];
    const bool q_row = row < d.L, sw = s.switched();
    if (!sw && !q_row) return;
    const uint32_t prime = d.prime(row), kind = q_row ? s.kind() : kNone;
    const A ar(mods[prime]);
    const size_t at = ((size_t)row << d.log_n) + pos, dstride = (size_t)d.ext << d.log_n,
                 kstride = (size_t)d.key_rows << d.log_n;
    const uint64_t *dg = dig + ((size_t)z * d.nd * d.ext << d.log_n) + at,
                   *key = rlk + ((size_t)prime << d.log_n) + pos;
    uint64_t w[4] = {}, dv[kDig] = {}, bv[kDig] = {}, av[kDig] = {};
    if (kind == kGiven) {
        w[0] = s.a[at];
        w[1] = s.a[at + ((size_t)d.L << d.log_n)];
    } else if (kind != kNone) {
        w[0] = s.a[at];
        w[1] = s.a[at + ((size_t)s.a_limbs() << d.log_n)];
        w[2] = s.b[at];
        if (kind == kProduct) w[3] = s.b[at + ((size_t)s.b_limbs() << d.log_n)];
    }
    if constexpr (ND > 0) {
        if (sw) {
#pragma unroll
            for (int i = 0; i < ND; i++) {
                dv[i] = dg[i * dstride];
                bv[i] = key[2 * i * kstride];
                av[i] = key[(2 * i + 1) * kstride];
            }
        }
    }
    double u0 = 0.0, u1 = 0.0;
    if (q_row) {
        // linear terms: a product at most 0.875 q, reduced every four
        for (uint32_t i = 0; i < s.n(); i++) {
            const double k = int_mod(s.k[i], s.sh(i), ar);
            const uint64_t *zp = s.z[i] + at;
            u0 += ar.mul(A::from_u64(zp[0]), k);
            if (s.two(i)) u1 += ar.mul(A::from_u64(zp[(size_t)s.limbs(i) << d.log_n]), k);
            if ((i & 3) == 3) {
                u0 = ar.red(u0);
                u1 = ar.red(u1);
            }
        }
        if (s.k[kStepTerms]) {   // the constant c as c q_l, which the division leaves as c
            const double ql = ar.red((double)mods[d.L - 1].qd);
            u0 += ar.mul(int_mod(s.k[kStepTerms], s.sh(kStepTerms), ar), ql < 0.0 ? ql + ar.q : ql);
        }
        const double w0 = A::from_u64(w[0]), w1 = A::from_u64(w[1]), w2 = A::from_u64(w[2]), m = s.mult;
        if (kind == kGiven) {
            u0 += w0;
            u1 += w1;
        } else if (kind != kNone) {
            u0 = ar.red(u0) + m * ar.mul(w0, w2);
            u1 = ar.red(u1) + m * ar.mul(w1, w2);
            if (kind == kProduct) u1 += m * ar.mul(w0, A::from_u64(w[3]));
        }
        u0 = ar.red(u0);
        u1 = ar.red(u1);
    }
    if (sw) {
        const double pq = q_row ? (double)pmodq[row].x : 0.0;
        u0 = ar.mul(u0, pq);
        u1 = ar.mul(u1, pq);
        auto digit = [&](uint64_t v, uint64_t b, uint64_t a) {
            const double x = A::from_u64(v);
            u0 += ar.mul(x, A::from_u64(b));
            u1 += ar.mul(x, A::from_u64(a));
        };
        if constexpr (ND > 0) {
#pragma unroll
            for (int i = 0; i < ND; i++) digit(dv[i], bv[i], av[i]);
        } else {
            for (uint32_t i = 0; i < d.nd; i++) {
                digit(dg[i * dstride], key[2 * i * kstride], key[(2 * i + 1) * kstride]);
                if ((i & 3) == 3) {
                    u0 = ar.red(u0);
                    u1 = ar.red(u1);
                }
            }
        }
        u0 = ar.red(u0);
        u1 = ar.red(u1);
    }
    uint64_t *out = u + ((size_t)z * 2 * d.ext << d.log_n) + at;
    out[0] = A::to_raw(u0);
    out[(size_t)d.ext << d.log_n] = A::to_raw(u1);
}

}  // namespace

ckks_status step_blk(ckks_ctx *ctx, uint32_t L, const Batch &b, uint32_t n, uint32_t n_sw, const uint64_t *rlk,
                     uint64_t *mem)
{
    Dims d = wsum_dims(ctx, L);
    const size_t N = ctx->n;
    uint64_t *dig = mem, *stage = dig + (size_t)n_sw * d.nd * d.ext * N, *u = stage + (size_t)n_sw * L * N;
    if (n_sw) {
        CK_TRY(blk_modup(ctx, step_sources(ctx, L, b, n_sw), n_sw, L - 1, dig, stage));
    } else {
        d.K = 0;
        d.ext = L;
    }
    Args a{};
    a.kind[0].rotated = 1;
    for (uint32_t i = 0; i < n; i++) {
        a.ct[i].kind = i < n_sw ? 0 : 1;
        a.ct[i].out[0] = b.s[i].out;
    }
    const dim3 grid(ctx->n / 256, d.ext, n);
    prof_begin(ctx, K_KEYIP, 8.0 * N * d.ext * (n_sw * (d.nd + 2.0) + 4.0 * n));
#define CK_GO(ND)                                                                                                  \
    hipLaunchKernelGGL(k_step_sums<ND>, grid, dim3(256), 0, ctx->stream, b, dig, rlk, u, d, ctx->d_pmodq, ctx->d_mod)
    switch (d.nd) {
    case 1: CK_GO(1); break;
    case 2: CK_GO(2); break;
    case 3: CK_GO(3); break;
    case 4: CK_GO(4); break;
    default: CK_GO(0); break;
    }
#undef CK_GO
    prof_end(ctx, K_KEYIP);
    HIP_TRY(hipGetLastError());
    return wsum_blk_divide(ctx, a, n, 1, d, u);
}

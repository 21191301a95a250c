// Steps (step.h) in the rings of 2^12 and 2^13 points with fp64 arithmetic, whole rows in a block (ntt_block.h).  After the
// two launches of the ModUp, which forms the products d2 where it reads them:
//   k_step_top   u = P (d0, d1) + <digits, rlk> on the rows q_l and P and their inverse transforms: U P^-1 and the centred
//                digits y_i;
//   k_step_fin   u on the rows below q_l, the row's conversion x (wsum_block.hip) and its transform, (u - NTT(x)) (P q_l)^-1.
// Few ciphertexts are bounded by one row's latency a launch, so the sums are formed where they are used: a launch apart
// for them, as the weighted sums of rotations have, costs one more.
#include "ops.h"
#include "step_args.h"
#include "wsum_block.h"

namespace {

using namespace wsum;
using namespace steps;

// u of component k at a thread's 16 points of the row layout, |u| <= q/2 + 1.  q_row: the row is one of the q limbs (the P
// rows have no d0, d1); in units of q a product is at most 0.875, so four and a reduced sum stay below 4.
template <int LOGN>
__device__ __forceinline__ void step_row(double (&u)[kE], const Operands &s, uint32_t k, const uint64_t *dig,
                                         const uint64_t *rlk, const Dims &d, uint32_t row, double pq, const A &ar,
                                         const A &top)
{
    const uint32_t t = threadIdx.x;
    const bool q_row = row < d.L;
    auto reduce = [&] {
#pragma unroll
        for (int e = 0; e < kE; e++) u[e] = ar.red(u[e]);
    };
    // u += m a b at the 16 points
    auto product = [&](const uint64_t *a, const uint64_t *b, double m) {
        uint64_t v[kE], w[kE];
#pragma unroll
        for (int e = 0; e < kE; e++) v[e] = a[blk::row_pos(t, e)];
#pragma unroll
        for (int e = 0; e < kE; e++) w[e] = b[blk::row_pos(t, e)];
#pragma unroll
        for (int e = 0; e < kE; e++) u[e] += m * ar.mul(A::from_u64(v[e]), A::from_u64(w[e]));
    };
#pragma unroll
    for (int e = 0; e < kE; e++) u[e] = 0.0;
    if (q_row) {
        const size_t rw = (size_t)row << LOGN;
        for (uint32_t i = 0; i < s.n; i++) {
            if (k && s.polys[i] < 2) continue;
            const double f = int_mod(s.k[i], s.sh[i], ar);
            const uint64_t *z = s.z[i] + rw + (k ? (size_t)s.limbs[i] << LOGN : 0);
#pragma unroll
            for (int e = 0; e < kE; e++) u[e] += ar.mul(A::from_u64(z[blk::row_pos(t, e)]), f);
            if ((i & 3) == 3) reduce();
        }
        if (!k && s.k[kStepTerms]) {   // the constant c as c q_l, which the division leaves as c
            const double ql = ar.red(top.q);
            const double c = ar.mul(int_mod(s.k[kStepTerms], s.sh[kStepTerms], ar), ql < 0.0 ? ql + ar.q : ql);
#pragma unroll
            for (int e = 0; e < kE; e++) u[e] += c;
        }
        const uint64_t *a0 = s.a + rw, *b0 = s.b + rw;
        if (s.kind == kGiven) {
            const uint64_t *a = a0 + ((size_t)(k * d.L) << LOGN);
#pragma unroll
            for (int e = 0; e < kE; e++) u[e] += A::from_u64(a[blk::row_pos(t, e)]);
        } else if (s.kind != kNone) {
            const uint64_t *a1 = a0 + ((size_t)s.a_limbs << LOGN);
            reduce();
            product(k ? a1 : a0, b0, s.mult);
            if (k && s.kind == kProduct) product(a0, b0 + ((size_t)s.b_limbs << LOGN), s.mult);
        }
        reduce();
        if (!s.switched()) return;
#pragma unroll
        for (int e = 0; e < kE; e++) u[e] = ar.mul(u[e], pq);
    }
    const uint64_t *key = rlk + ((size_t)(k * d.key_rows + d.prime(row)) << LOGN);
    dig += (size_t)row << LOGN;
    for (uint32_t i = 0; i < d.nd; i++) {
        product(dig + ((size_t)i * d.ext << LOGN), key + ((size_t)2 * i * d.key_rows << LOGN), 1.0);
        if ((i & 3) == 3) reduce();
    }
    reduce();
}

// rows q_l (blockIdx.x = 0) and P of component blockIdx.y of step blockIdx.z: centred coefficients times their factor to
// y[z][k][s]
template <int LOGN>
__global__ __launch_bounds__(blk::Shape<LOGN>::NT) void k_step_top(Batch bt, const uint64_t *dig, const uint64_t *rlk,
                                                                   uint64_t *y, Dims d, Quot qt, Tab tb)
{
    __shared__ double lds[blk::Shape<LOGN>::kLds];
    const uint32_t s = blockIdx.x, k = blockIdx.y, z = blockIdx.z, t = threadIdx.x;
    const Operands &o = bt.s[z];
    if (s && !o.switched()) return;
    const uint32_t row = d.L - 1 + s, prime = d.prime(row);
    const A ar(tb.mods[prime]);
    A sc = ar;
    if (s) sc.ninv = ar.scaled_twiddle(qt.qhat_inv[s - 1]);
    else if (o.switched()) sc.ninv = ar.scaled_twiddle((double)qt.pinv[d.L - 1].x);
    const blk::ColTw<LOGN> cw(tb.itwf + ((size_t)prime << LOGN));
    const blk::RowTw<LOGN> rw(tb.itwf + ((size_t)prime << LOGN));
    double x[kE];
    step_row<LOGN>(x, o, k, dig + ((size_t)z * d.nd * d.ext << LOGN), rlk, d, row, s ? 0.0 : (double)qt.pmodq[row].x, ar, ar);
    blk::inverse<LOGN>(x, lds, cw, rw, ar, sc);
    uint64_t *out = y + ((((size_t)z * 2 + k) * (d.K + 1) + s) << LOGN);
#pragma unroll
    for (int e = 0; e < kE; e++) out[blk::col_pos<LOGN>(t, e)] = A::to_raw(centre(ar, x[e]));
}

// row i of component k of step z: grid (level, 2, steps)
template <int LOGN>
__global__ __launch_bounds__(blk::Shape<LOGN>::NT) void k_step_fin(Batch bt, const uint64_t *dig, const uint64_t *rlk,
                                                                   const uint64_t *y, Dims d, Quot qt, Tab tb)
{
    __shared__ double lds[blk::Shape<LOGN>::kLds];
    const uint32_t i = blockIdx.x, k = blockIdx.y, z = blockIdx.z, t = threadIdx.x;
    const Operands &o = bt.s[z];
    const bool sw = o.switched();
    const A ar(tb.mods[i]), top(tb.mods[d.L - 1]);
    const uint64_t *yr = y + (((size_t)z * 2 + k) * (d.K + 1) << LOGN);
    double x[kE], u[kE], f = (double)qt.qlinv[i].x;
#pragma unroll
    for (int e = 0; e < kE; e++) x[e] = A::from_raw(yr[blk::col_pos<LOGN>(t, e)]);
    const double pq = (double)qt.pmodq[i].x;
    if (sw) {
        f = centre(ar, ar.mul(f, (double)qt.pinv[i].x));
        f = f < 0.0 ? f + ar.q : f;
        double v[kE];
        digit_sums<LOGN>(v, yr, d, top, [&](int j) { return top_factor(qt, d, j, top); });
#pragma unroll
        for (int e = 0; e < kE; e++) x[e] = centre(top, x[e] - v[e]);
        digit_sums<LOGN>(v, yr, d, ar, [&](int j) { return qt.qhat_mod[j * (int)d.L + (int)i]; });
#pragma unroll
        for (int e = 0; e < kE; e++) x[e] = ar.red(v[e] + ar.mul(x[e], pq));
    } else {
#pragma unroll
        for (int e = 0; e < kE; e++) x[e] = ar.red(x[e]);
    }
    const blk::ColTw<LOGN> cw(tb.twf + ((size_t)i << LOGN));
    const blk::RowTw<LOGN> rw(tb.twf + ((size_t)i << LOGN));
    step_row<LOGN>(u, o, k, dig + ((size_t)z * d.nd * d.ext << LOGN), rlk, d, i, pq, ar, top);
    blk::forward<LOGN>(x, lds, cw, rw, ar);
    uint64_t *out = o.out + ((size_t)(k * (d.L - 1) + i) << LOGN);
#pragma unroll
    for (int e = 0; e < kE; e++) out[blk::row_pos(t, e)] = quotient(ar, u[e] - x[e], f);
}

}  // namespace

ckks_status step_blk(ckks_ctx *ctx, uint32_t L, const Batch &b, uint32_t n, uint32_t n_sw, const uint64_t *rlk,
                     uint64_t *mem)
{
    Dims d = wsum_dims(ctx, L);
    const size_t N = ctx->n;
    const uint32_t level = L - 1;
    uint64_t *dig = mem, *stage = dig + (size_t)n_sw * d.nd * d.ext * N, *y = stage + (size_t)n_sw * L * N;
    if (n_sw) {
        CK_TRY(blk_modup(ctx, step_sources(ctx, L, b, n_sw), n_sw, level, dig, stage));
    } else {
        d.K = 0;
        d.ext = L;
    }
    const ConvDev *cd;
    CK_TRY(ctx_conv(ctx, (int)level, -1, &cd));
    const Quot qt{cd->d_qhat_inv_f, cd->d_qhat_mod_f, ctx->d_pinv, ctx->d_qlinv + (size_t)level * ctx->n_q, ctx->d_pmodq};
    const Tab tb{ctx->d_mod, ctx->d_twf, ctx->d_itwf};
    const double rows1 = (2.0 * n_sw * d.K + 2.0 * n) * N, rows2 = 2.0 * n * level * N;
#define CK_BLK(KERNEL, GRID, ...)                                                                                  \
    do {                                                                                                           \
        if (ctx->log_n == 12)                                                                                      \
            hipLaunchKernelGGL(KERNEL<12>, GRID, dim3(blk::Shape<12>::NT), 0, ctx->stream, __VA_ARGS__);             \
        else                                                                                                       \
            hipLaunchKernelGGL(KERNEL<13>, GRID, dim3(blk::Shape<13>::NT), 0, ctx->stream, __VA_ARGS__);             \
    } while (0)
    prof_begin(ctx, K_KEYIP, 8.0 * rows1 * (d.nd + 1.0), rows1 * (5.0 * d.nd + kOpsButterflyF64 * d.log_n / 2));
    CK_BLK(k_step_top, dim3(d.K + 1, 2, n), b, dig, rlk, y, d, qt, tb);
    prof_end(ctx, K_KEYIP);
    HIP_TRY(hipGetLastError());
    prof_begin(ctx, K_MODDOWN, 8.0 * rows2 * (d.nd + 3.0), rows2 * (5.0 * d.nd + kOpsButterflyF64 * d.log_n / 2));
    CK_BLK(k_step_fin, dim3(level, 2, n), b, dig, rlk, y, d, qt, tb);
#undef CK_BLK
    prof_end(ctx, K_MODDOWN);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

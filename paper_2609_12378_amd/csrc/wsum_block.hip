// Weighted sums of rotations (wsum.hip) in the rings of 2^12 and 2^13 points with fp64 arithmetic, whole rows in a
// block (ntt_block.h).  After the ModUp:
//   1. k_blk_wsum   u on every row, element-wise;
//   2. k_blk_wtop   the rows q_l and P to coefficients: U P^-1 and the centred digits y_i;
//   3. k_blk_wfin   a block forms its row of the conversion, x_t = sum_i y_i [P / p_i]_t + P w with w the centred top
//      coefficient of the quotient by P, transforms it and writes (u - NTT(x)) (P q_l)^-1 (+ prev).
// With the two launches of the ModUp that is five; through the ModDown, the rescale and the additions it was eight. 
// Few ciphertexts are bounded by one row's latency a launch: one of 4 limbs at N = 2^12 takes 4, 7 and 11 us in the
// three (35 us a call, as long as the host takes to issue it), three of 6 limbs at 2^13 7, 11 and 17 (58 us a call).  The
// sums of 1 could be formed where 2 and 3 read them, a row a block, in one launch fewer; that is not tried.
#include "ntt_block.h"
#include "ops.h"
#include "wsum_args.h"

namespace {

using namespace wsum;
using nttc::GridSum;
using nttc::kE;

struct Tab {
    const ModQ *mods;
    const double *twf, *itwf;
};

// u[z P + o][k][row][n] as doubles of at most q/2 + 1: one position a thread, every load issued before the first
// product. Unrotated kinds: pt c, on the q rows alone.
template <int ND, int P>
__global__ __launch_bounds__(256) void k_blk_wsum(Args a, uint64_t *u, Dims d, const ulonglong2 *__restrict__ pmodq,
                                                  const ModQ *__restrict__ mods)
{
    constexpr int T = (int)kWsumTerms;
    const uint32_t pos = blockIdx.x * 256 + threadIdx.x, row = blockIdx.y, z = blockIdx.z;
    const Ct &ct = a.ct[z];
    const WsumKind &w = a.kind[ct.kind];
    const bool q_row = row < d.L;
    if (!w.rotated && !q_row) return;
    const uint32_t prime = d.prime(row);
    const A ar(mods[prime]);
    const size_t rw = (size_t)row << d.log_n, half = (size_t)d.L << d.log_n;
    const double pq = q_row ? (double)pmodq[row].x : 0.0;
    const uint64_t *c = ct.c + (q_row ? rw : 0);   // on the P rows read and not used
    uint64_t cv[T], dv[T][ND], bv[T][ND], av[T][ND], tv[P][T];
#pragma unroll
    for (int j = 0; j < T; j++) {
        if (j >= (int)w.n) break;
        const uint32_t sc = auto_index(pos, w.g[j], d.log_n);
        cv[j] = c[sc];
#pragma unroll
        for (int o = 0; o < P; o++) tv[o][j] = w.tab[o][j][rw + pos];
        if (!w.key[j]) {
            dv[j][0] = c[half + pos];
            continue;
        }
        const uint64_t *key = w.key[j] + ((size_t)prime << d.log_n) + pos, *dig = ct.dig + rw + sc;
#pragma unroll
        for (int i = 0; i < ND; i++) {
            dv[j][i] = dig[(size_t)i * d.ext << d.log_n];
            bv[j][i] = key[(size_t)(2 * i) * d.key_rows << d.log_n];
            av[j][i] = key[(size_t)(2 * i + 1) * d.key_rows << d.log_n];
        }
    }
    double s[P][2] = {};
#pragma unroll
    for (int j = 0; j < T; j++) {
        if (j >= (int)w.n) break;
        double t0, t1;
        if (w.key[j]) {
            ProductSum s0, s1;
            s0.add(A::from_u64(cv[j]), pq);
#pragma unroll
            for (int i = 0; i < ND; i++) {
                if (i && i % 3 == 0) {   // s0 holds the c0 term and three products
                    s0.fold(ar);
                    s1.fold(ar);
                }
                s0.add(A::from_u64(dv[j][i]), A::from_u64(bv[j][i]));
                s1.add(A::from_u64(dv[j][i]), A::from_u64(av[j][i]));
            }
            t0 = s0.value(ar);
            t1 = s1.value(ar);
        } else {
            t0 = A::from_u64(cv[j]);
            t1 = A::from_u64(dv[j][0]);
            if (w.rotated) {
                t0 = ar.mul(t0, pq);
                t1 = ar.mul(t1, pq);
            }
            if (!q_row) t0 = t1 = 0.0;
        }
#pragma unroll
        for (int o = 0; o < P; o++) {
            const double pt = A::from_u64(tv[o][j]);
            s[o][0] += ar.mul(t0, pt);
            s[o][1] += ar.mul(t1, pt);
        }
    }
#pragma unroll
    for (int o = 0; o < P; o++) {
        uint64_t *x = u + ((size_t)(z * P + o) * 2 * d.ext << d.log_n) + rw + pos;
        x[0] = A::to_raw(ar.red(s[o][0]));
        x[(size_t)d.ext << d.log_n] = A::to_raw(ar.red(s[o][1]));
    }
}

// rows q_l (blockIdx.x = 0) and P of each polynomial to centred coefficients times their factor, in place (a thread's
// words are in registers before the first block barrier and written after the last); grid (K + 1, polys)
template <int LOGN>
__global__ __launch_bounds__(blk::Shape<LOGN>::NT) void k_blk_wtop(uint64_t *u, Args a, Dims d, uint32_t pages, Quot qt,
                                                                   Tab tb)
{
    __shared__ double lds[blk::Shape<LOGN>::kLds];
    const uint32_t s = blockIdx.x, p = blockIdx.y, t = threadIdx.x;
    const bool rot = a.kind[a.ct[p / 2 / pages].kind].rotated;
    if (s && !rot) return;
    const uint32_t prime = d.prime(d.L - 1 + s);
    const A ar(tb.mods[prime]);
    A sc = ar;
    if (s) sc.ninv = ar.scaled_twiddle(qt.qhat_inv[s - 1]);
    else if (rot) sc.ninv = ar.scaled_twiddle((double)qt.pinv[d.L - 1].x);
    uint64_t *row = u + (((size_t)p * d.ext + d.L - 1 + s) << LOGN);
    const blk::ColTw<LOGN> cw(tb.itwf + ((size_t)prime << LOGN));
    const blk::RowTw<LOGN> rw(tb.itwf + ((size_t)prime << LOGN));
    double x[kE];
#pragma unroll
    for (int k = 0; k < kE; k++) x[k] = A::from_raw(row[blk::row_pos(t, k)]);
    blk::inverse<LOGN>(x, lds, cw, rw, ar, sc);
#pragma unroll
    for (int k = 0; k < kE; k++) row[blk::col_pos<LOGN>(t, k)] = A::to_raw(centre(ar, x[k]));
}

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

// row i of component k of output o: grid (level, 2, outs).  The K digits and the q_l row follow one another in u.
template <int LOGN>
__global__ __launch_bounds__(blk::Shape<LOGN>::NT) void k_blk_wfin(Args a, const uint64_t *u, Dims d, uint32_t pages,
                                                                   Quot qt, Tab tb)
{
    __shared__ double lds[blk::Shape<LOGN>::kLds];
    const uint32_t i = blockIdx.x, k = blockIdx.y, o = blockIdx.z, t = threadIdx.x;
    const Ct &ct = a.ct[o / pages];
    const bool rot = a.kind[ct.kind].rotated;
    const A ar(tb.mods[i]), top(tb.mods[d.L - 1]);
    const uint64_t *up = u + (((size_t)o * 2 + k) * d.ext << LOGN), *ur = up + ((size_t)i << LOGN),
                   *yr = up + ((size_t)(d.L - 1) << LOGN);
    const size_t row = ((size_t)k * (d.L - 1) + i) << LOGN;
    double x[kE], f = (double)qt.qlinv[i].x;
#pragma unroll
    for (int e = 0; e < kE; e++) x[e] = A::from_raw(yr[blk::col_pos<LOGN>(t, e)]);
    if (rot) {
        const double pq = (double)qt.pmodq[i].x;
        f = centre(ar, ar.mul(f, (double)qt.pinv[i].x));
        f = f < 0.0 ? f + ar.q : f;
        // the sums modulo q_l first, then those modulo q_i, eight points at a time: both at once would not fit the
        // registers
        double v[kE];
        digit_sums<LOGN>(v, yr, d, top, [&](int s) { return top_factor(qt, d, s, top); });
#pragma unroll
        for (int e = 0; e < kE; e++) x[e] = centre(top, x[e] - v[e]);
        digit_sums<LOGN>(v, yr, d, ar, [&](int s) { return qt.qhat_mod[s * (int)d.L + (int)i]; });
#pragma unroll
        for (int e = 0; e < kE; e++) x[e] = ar.red(v[e] + ar.mul(x[e], pq));
    } else {
#pragma unroll
        for (int e = 0; e < kE; e++) x[e] = ar.red(x[e]);
    }
    const blk::ColTw<LOGN> cw(tb.twf + ((size_t)i << LOGN));
    const blk::RowTw<LOGN> rw(tb.twf + ((size_t)i << LOGN));
    // the row's own words and the page's, ahead of the transform
    double uv[kE];
    uint64_t pv[kE];
#pragma unroll
    for (int e = 0; e < kE; e++) uv[e] = A::from_raw(ur[blk::row_pos(t, e)]);
    const uint64_t *prev = ct.prev[o % pages];
#pragma unroll
    for (int e = 0; e < kE; e++) pv[e] = prev ? prev[row + blk::row_pos(t, e)] : 0;
    blk::forward<LOGN>(x, lds, cw, rw, ar);
    const uint64_t q = tb.mods[i].q;
    uint64_t *out = ct.out[o % pages] + row;
#pragma unroll
    for (int e = 0; e < kE; e++) {
        const uint64_t v = quotient(ar, uv[e] - x[e], f);
        out[blk::row_pos(t, e)] = addmod(v, pv[e], q);
    }
}

}  // namespace

ckks_status wsum_blk_sums(ckks_ctx *ctx, const Args &a, uint32_t n, uint32_t pages, const Dims &d, uint64_t *u)
{
    const uint32_t level = d.L - 1, polys = 2 * n * pages;
    const double N = ctx->n;
    const ConvDev *cd;
    CK_TRY(ctx_conv(ctx, (int)level, -1, &cd));
    const Quot qt{cd->d_qhat_inv_f, cd->d_qhat_mod_f, ctx->d_pinv, ctx->d_qlinv + (size_t)level * ctx->n_q, ctx->d_pmodq};
    const Tab tb{ctx->d_mod, ctx->d_twf, ctx->d_itwf};
    prof_begin(ctx, K_KEYIP, 8.0 * N * d.ext * n * (d.nd + 1.0 + 2.0 * pages));
#define CK_GO(ND)                                                                                                  \
    do {                                                                                                           \
        const dim3 grid(ctx->n / 256, d.ext, n);                                                                   \
        if (pages == 1)                                                                                            \
            hipLaunchKernelGGL((k_blk_wsum<ND, 1>), grid, dim3(256), 0, ctx->stream, a, u, d, ctx->d_pmodq, ctx->d_mod); \
        else                                                                                                       \
            hipLaunchKernelGGL((k_blk_wsum<ND, 2>), grid, dim3(256), 0, ctx->stream, a, u, d, ctx->d_pmodq, ctx->d_mod); \
    } while (0)
    switch (d.nd) {
    case 1: CK_GO(1); break;
    case 2: CK_GO(2); break;
    case 3: CK_GO(3); break;
    case 4: CK_GO(4); break;
    default: CK_GO(5); break;
    }
#undef CK_GO
    prof_end(ctx, K_KEYIP);
    HIP_TRY(hipGetLastError());
    prof_begin(ctx, K_NTT_INV_ROW, 16.0 * polys * (d.K + 1) * N, polys * (d.K + 1) * N * kOpsButterflyF64 * d.log_n / 2);
#define CK_BLK(KERNEL, GRID, ...)                                                                                  \
    do {                                                                                                           \
        if (ctx->log_n == 12)                                                                                      \
            hipLaunchKernelGGL(KERNEL<12>, GRID, dim3(blk::Shape<12>::NT), 0, ctx->stream, __VA_ARGS__);             \
        else                                                                                                       \
            hipLaunchKernelGGL(KERNEL<13>, GRID, dim3(blk::Shape<13>::NT), 0, ctx->stream, __VA_ARGS__);             \
    } while (0)
    CK_BLK(k_blk_wtop, dim3(d.K + 1, polys), u, a, d, pages, qt, tb);
    prof_end(ctx, K_NTT_INV_ROW);
    HIP_TRY(hipGetLastError());
    prof_begin(ctx, K_MODDOWN, 8.0 * polys * N * (d.K + 1.0 + 3.0 * level), polys * level * N * kOpsButterflyF64 * d.log_n / 2);
    CK_BLK(k_blk_wfin, dim3(level, 2, n * pages), a, u, d, pages, qt, tb);
#undef CK_BLK
    prof_end(ctx, K_MODDOWN);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

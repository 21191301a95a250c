// Weighted sums of rotations (wsum.hip has the formulas) for any ring, primes and number of digits, in integers:
//   k_wsum     u on all rows of Q_l u P, in exact 128-bit sums;
//   the inverse transform of its rows q_l and P;
//   k_quot     x_t = sum_i y_i [P / p_i]_t + P w for every target q_t, t < l: the conversion of the centred P rows together
//              with the centred top coefficient w of the quotient by P (no P rows and w times 1: unrotated kinds);
//   the forward transform of x, whose row pass (fused_row.hip, N >= 2^12) writes out = (u - NTT(x)) (P q_l)^-1 + prev.
// One division by P q_l where a ModDown and a rescale are two: one forward transform, one pass over u.
#include <algorithm>

#include "ops.h"
#include "sum60.h"
#include "wsum_args.h"

namespace {

constexpr int kThreads = 256;
using namespace wsum;

// u[z P + o][k][row][n] of ciphertext z, output o of P.  Two positions a thread: sigma_g reads the pair (j, j + 1) at
// (j', j' ^ 1).  A digit's own rows are c1's.  Two ciphertexts of 37 limbs in five digits: 195 us, 0.67 GB at 3.4 TB/s,
// 79% of the issue slots, about 40% of the instructions in reduce128 (284 us with a ciphertext after the other, so that
// each reads the keys from HBM).  In the first passes of a process, where it takes 203 us, sums of 30-bit halves (sum60.h)
// measured 197 and loads a digit ahead 211: neither is used.
template <int P>
__global__ __launch_bounds__(kThreads) void k_wsum(Args a, uint64_t *u, Dims d, uint32_t n, uint32_t per_row,
                                                   const ulonglong2 *__restrict__ pmodq, const ModQ *__restrict__ mods)
{
    uint32_t z, tile;
    tile_of(n, z, tile);
    const uint32_t row = tile / per_row, col = 2 * (tile % per_row * kThreads + threadIdx.x);
    if (row >= d.ext || col >= (1u << d.log_n)) return;
    const uint32_t prime = d.prime(row);
    const ModQ m = mods[prime];
    const Ct &ct = a.ct[z];
    const WsumKind &w = a.kind[ct.kind];
    const uint64_t pq = row < d.L ? pmodq[row].x : 0;
    const uint64_t *c = ct.c + ((size_t)row << d.log_n), *c1 = c + ((size_t)d.L << d.log_n);
    const uint64_t *dig = ct.dig + ((size_t)row << d.log_n);
    const uint32_t own = row < d.L ? row / d.alpha : d.nd;
    acc128 acc[P][2][2] = {};
    for (uint32_t j = 0; j < w.n; j++) {
        acc128 t[2][2] = {};
        if (w.key[j]) {
            const uint32_t sc = auto_index(col, w.g[j], d.log_n), at = sc & ~1u, odd = sc & 1u;
            const uint64_t *key = w.key[j] + ((size_t)prime << d.log_n) + col;
            for (uint32_t i = 0; i < d.nd; i++) {
                const Pair v = ld2((i == own ? c1 : dig + ((size_t)i * d.ext << d.log_n)) + at);
                const Pair k0 = ld2(key + ((size_t)(2 * i) * d.key_rows << d.log_n));
                const Pair k1 = ld2(key + ((size_t)(2 * i + 1) * d.key_rows << d.log_n));
                const uint64_t x = odd ? v.y : v.x, y = odd ? v.x : v.y;
                mac(t[0][0], x, k0.x);
                mac(t[0][1], y, k0.y);
                mac(t[1][0], x, k1.x);
                mac(t[1][1], y, k1.y);
                // products are below 2^124: fold before the ninth
                if ((i & 7u) == 7u)
#pragma unroll
                    for (int k = 0; k < 4; k++) t[k >> 1][k & 1] = acc128{reduce128(t[k >> 1][k & 1], m), 0};
            }
            if (row < d.L) {
                const Pair v = ld2(c + at);
                mac(t[0][0], odd ? v.y : v.x, pq);
                mac(t[0][1], odd ? v.x : v.y, pq);
            }
        } else if (row < d.L) {
            const Pair v = ld2(c + col), v1 = ld2(c1 + col);
            mac(t[0][0], v.x, pq);
            mac(t[0][1], v.y, pq);
            mac(t[1][0], v1.x, pq);
            mac(t[1][1], v1.y, pq);
        }
        uint64_t r[2][2];
#pragma unroll
        for (int k = 0; k < 4; k++) r[k >> 1][k & 1] = reduce128(t[k >> 1][k & 1], m);
#pragma unroll
        for (int o = 0; o < P; o++) {
            const Pair pt = ld2(w.tab[o][j] + ((size_t)row << d.log_n) + col);
#pragma unroll
            for (int k = 0; k < 2; k++) {
                mac(acc[o][k][0], r[k][0], pt.x);
                mac(acc[o][k][1], r[k][1], pt.y);
            }
        }
    }
#pragma unroll
    for (int o = 0; o < P; o++)
#pragma unroll
        for (int k = 0; k < 2; k++)
            *(Pair *)(u + (((size_t)((z * P + o) * 2 + k) * d.ext + row) << d.log_n) + col) =
                Pair{reduce128(acc[o][k][0], m), reduce128(acc[o][k][1], m)};
}

// u[z P + o][k][row] = pt c_k: the outputs of unrotated kinds, with nothing to divide by P
__global__ __launch_bounds__(kThreads) void k_wmul(Args a, uint64_t *u, Dims d, uint32_t pages,
                                                   const ModQ *__restrict__ mods)
{
    const uint32_t col = blockIdx.x * kThreads + threadIdx.x, row = blockIdx.y, z = blockIdx.z;
    if (col >= (1u << d.log_n)) return;
    const ModQ m = mods[row];
    const size_t at = ((size_t)row << d.log_n) + col, half = (size_t)d.L << d.log_n;
    const Ct &ct = a.ct[z];
    const uint64_t c0 = ct.c[at], c1 = ct.c[half + at];
    for (uint32_t o = 0; o < pages; o++) {
        const uint64_t pt = a.kind[ct.kind].tab[o][0][at];
        uint64_t *x = u + (size_t)(z * pages + o) * 2 * half + at;
        x[0] = mulmod(c0, pt, m);
        x[half] = mulmod(c1, pt, m);
    }
}

// x[poly][t] for the targets [t0, t0 + t_per) of this block's group.  in: coefficients of polynomial p's row q_l at
// in + p ext N, the ns rows P after it.  A digit y_i > p_i / 2 stands for y_i - p_i: the sum of the canonical digits plus
// neg [-P]_t, neg the number of such digits; w > q_l / 2 likewise adds [-f q_l]_t, f what multiplies w (P or 1).
template <int NS_MAX>
__global__ __launch_bounds__(kThreads) void k_quot(uint64_t *x, const uint64_t *in, Dims d, int ns, uint32_t t_per,
                                                   const ulonglong2 *__restrict__ qhat_inv,
                                                   const ulonglong2 *__restrict__ qhat_mod,
                                                   const ulonglong2 *__restrict__ neg_q,
                                                   const ulonglong2 *__restrict__ pinv,
                                                   const ulonglong2 *__restrict__ pmodq, const ModQ *__restrict__ mods)
{
    __shared__ uint64_t s_mod[NS_MAX * kMaxPrimes];
    __shared__ uint64_t s_neg[kMaxPrimes], s_f[kMaxPrimes], s_negw[kMaxPrimes];
    __shared__ ModQ s_tm[kMaxPrimes];
    const uint32_t l = d.L - 1, t0 = blockIdx.y * t_per, t1 = min(l, t0 + t_per), poly = blockIdx.z;
    const uint64_t ql = mods[l].q;
    for (uint32_t k = threadIdx.x; k < (uint32_t)ns * d.L; k += kThreads) s_mod[k] = qhat_mod[k].x;
    for (uint32_t k = threadIdx.x; k < d.L; k += kThreads) {
        const ModQ m = mods[k];
        const uint64_t f = ns ? pmodq[k].x : 1;
        s_tm[k] = m;
        s_neg[k] = ns ? neg_q[k].x : 0;
        s_f[k] = f;
        s_negw[k] = submod(0, mulmod(f, ql, m), m.q);
    }
    __syncthreads();
    const uint32_t col = blockIdx.x * kThreads + threadIdx.x;
    if (col >= (1u << d.log_n)) return;
    const uint64_t *src = in + ((size_t)poly * d.ext << d.log_n) + col;
    uint64_t y[NS_MAX], neg = 0;
#pragma unroll
    for (int i = 0; i < NS_MAX; i++)
        if (i < ns) {
            const uint64_t q = mods[d.n_q + i].q;
            const ulonglong2 v = qhat_inv[i];
            y[i] = shoup(src[(size_t)(i + 1) << d.log_n], v.x, v.y, q);
            neg += y[i] > (q >> 1);
        }
    // sum_i y_i [P / p_i]_t, exact up to a fold every eight terms
    const auto sum = [&](uint32_t t, acc128 s) {
        mac(s, neg, s_neg[t]);
#pragma unroll
        for (int i = 0; i < NS_MAX; i++)
            if (i < ns) {
                mac(s, y[i], s_mod[i * d.L + t]);
                if ((i & 7) == 7 && i + 1 < ns) s = acc128{reduce128(s, s_tm[t]), 0};
            }
        return s;
    };
    uint64_t w = src[0];
    if (ns) w = shoup(submod(w, reduce128(sum(l, acc128{0, 0}), s_tm[l]), ql), pinv[l].x, pinv[l].y, ql);
    const uint64_t negw = w > (ql >> 1);
    for (uint32_t t = t0; t < t1; t++) {
        acc128 s = sum(t, acc128{0, 0});
        mac(s, w, s_f[t]);
        s.lo += negw ? s_negw[t] : 0;
        s.hi += s.lo < (negw ? s_negw[t] : 0);
        x[(((size_t)poly * l + t) << d.log_n) + col] = reduce128(s, s_tm[t]);
    }
}

// The same with at most 8 special primes and every prime below 2^60 (sum60.h).  The constants, 2^64 times theirs, are staged
// as halves, so the quotient's w takes its own sums (a ninth product would pass 64 bits in mid).
__global__ __launch_bounds__(kThreads) void k_quot60(uint64_t *x, const uint64_t *in, Dims d, int ns, uint32_t t_per,
                                                     const ulonglong2 *__restrict__ qhat_inv,
                                                     const ulonglong2 *__restrict__ qhat_mod,
                                                     const ulonglong2 *__restrict__ neg_q,
                                                     const ulonglong2 *__restrict__ pinv,
                                                     const ulonglong2 *__restrict__ pmodq, const ModQ *__restrict__ mods)
{
    // slot s of the constants: target t0 + s, and the last one, t1 - t0, q_l
    __shared__ uint2 s_mod[8 * kMaxPrimes], s_neg[kMaxPrimes], s_f[kMaxPrimes];
    __shared__ uint64_t s_negw[kMaxPrimes];
    __shared__ Mod60 s_tm[kMaxPrimes];
    const uint32_t l = d.L - 1, t0 = blockIdx.y * t_per, nt = min(l, t0 + t_per) - t0, poly = blockIdx.z;
    const uint64_t ql = mods[l].q;
    for (uint32_t k = threadIdx.x; k < (uint32_t)ns * (nt + 1); k += kThreads) {
        const uint32_t i = k / (nt + 1), s = k % (nt + 1), t = s < nt ? t0 + s : l;
        s_mod[i * kMaxPrimes + s] = halves(times_2_64(qhat_mod[i * d.L + t].x, mods[t]));
    }
    for (uint32_t s = threadIdx.x; s <= nt; s += kThreads) {
        const uint32_t t = s < nt ? t0 + s : l;
        const ModQ m = mods[t];
        const uint64_t f = times_2_64(ns ? pmodq[t].x : 1, m);
        s_tm[s] = mod60(m.q);
        s_neg[s] = halves(ns ? times_2_64(neg_q[t].x, m) : 0);
        s_f[s] = halves(f);
        s_negw[s] = submod(0, mulmod(f, ql, m), m.q);
    }
    __syncthreads();
    const uint32_t col = blockIdx.x * kThreads + threadIdx.x;
    if (col >= (1u << d.log_n)) return;
    const uint64_t *src = in + ((size_t)poly * d.ext << d.log_n) + col;
    uint2 y[8];
    uint32_t neg = 0;
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < ns) {
            const uint64_t q = mods[d.n_q + i].q;
            const ulonglong2 c = qhat_inv[i];
            const uint64_t v = shoup(src[(size_t)(i + 1) << d.log_n], c.x, c.y, q);
            neg += v > (q >> 1);
            y[i] = halves(v);
        }
    const auto sum = [&](uint32_t s) {
        Sum60 r;
        r.add(neg, s_neg[s]);
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < ns) r.add(y[i], s_mod[i * kMaxPrimes + s]);
        return r.value();
    };
    uint64_t w = src[0];
    if (ns) w = shoup(submod(w, redc(sum(nt), s_tm[nt]), ql), pinv[l].x, pinv[l].y, ql);
    const bool negw = w > (ql >> 1);
    const uint2 wh = halves(w);
    for (uint32_t s = 0; s < nt; s++) {
        Sum60 p;
        p.add(wh, s_f[s]);
        const acc128 a = sum(s), b = p.value();
        const unsigned __int128 r = ((unsigned __int128)a.hi << 64 | a.lo) + ((unsigned __int128)b.hi << 64 | b.lo) +
                                    (negw ? s_negw[s] : 0);
        x[(((size_t)poly * l + t0 + s) << d.log_n) + col] = redc(acc128{(uint64_t)r, (uint64_t)(r >> 64)}, s_tm[s]);
    }
}

// out = (u - x) f (+ prev) for rings below 2^12 points, x transformed
__global__ __launch_bounds__(kThreads) void k_finish(Args a, const uint64_t *u, const uint64_t *x, Dims d, uint32_t pages,
                                                     const ulonglong2 *__restrict__ f, const ModQ *__restrict__ mods)
{
    const uint32_t col = blockIdx.x * kThreads + threadIdx.x, l = d.L - 1, row = blockIdx.y % l, k = blockIdx.y / l,
                   z = blockIdx.z / pages, o = blockIdx.z % pages;
    if (col >= (1u << d.log_n)) return;
    const uint64_t q = mods[row].q;
    const size_t at = ((size_t)(k * l + row) << d.log_n) + col, p = 2 * blockIdx.z + k;
    uint64_t v = submod(u[((p * d.ext + row) << d.log_n) + col], x[((p * l + row) << d.log_n) + col], q);
    v = shoup(v, f[row].x, f[row].y, q);
    const uint64_t *prev = a.ct[z].prev[o];
    a.ct[z].out[o][at] = prev ? addmod(v, prev[at], q) : v;
}

// c1 of ciphertext z to out[z][L][N]
__global__ __launch_bounds__(kThreads) void k_gather_c1(uint64_t *out, Args a, uint32_t L, uint32_t log_n)
{
    const uint32_t col = 2 * (blockIdx.x * kThreads + threadIdx.x), row = blockIdx.y, z = blockIdx.z;
    if (col >= (1u << log_n)) return;
    *(Pair *)(out + (((size_t)z * L + row) << log_n) + col) = ld2(a.ct[z].c + (((size_t)L + row) << log_n) + col);
}

dim3 grid_of(const ckks_ctx *ctx, uint32_t rows, uint32_t z, uint32_t words)
{
    return dim3((ctx->n + words * kThreads - 1) / (words * kThreads), rows, z);
}

}  // namespace

ckks_status wsum_gather_c1(ckks_ctx *ctx, const Args &a, uint32_t n, uint32_t L, uint64_t *out)
{
    prof_begin(ctx, K_ELEM, 16.0 * ctx->n * L * n);
    hipLaunchKernelGGL(k_gather_c1, grid_of(ctx, L, n, 2), dim3(kThreads), 0, ctx->stream, out, a, L, ctx->log_n);
    prof_end(ctx, K_ELEM);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

ckks_status wsum_exact_sums(ckks_ctx *ctx, const Args &a, uint32_t n, uint32_t pages, const Dims &dims, bool rot,
                            uint64_t *u, uint64_t *x)
{
    Dims d = dims;
    if (!rot) {
        d.K = 0;
        d.ext = d.L;
    }
    const size_t N = ctx->n;
    const uint32_t level = d.L - 1, outs = n * pages, polys = 2 * outs;
    if (rot) {
        const uint32_t per_row = grid_of(ctx, 1, 1, 2).x, tiles = (d.ext * per_row + 7) / 8 * 8;
        prof_begin(ctx, K_KEYIP, 8.0 * N * d.ext * n * (d.nd + 1.0 + 2.0 * pages));
        if (pages == 1)
            hipLaunchKernelGGL(k_wsum<1>, dim3(tiles * n), dim3(kThreads), 0, ctx->stream, a, u, d, n, per_row,
                               ctx->d_pmodq, ctx->d_mod);
        else
            hipLaunchKernelGGL(k_wsum<2>, dim3(tiles * n), dim3(kThreads), 0, ctx->stream, a, u, d, n, per_row,
                               ctx->d_pmodq, ctx->d_mod);
        prof_end(ctx, K_KEYIP);
    } else {
        prof_begin(ctx, K_ELEM, 8.0 * N * d.L * n * (2.0 + 2.0 * pages));
        hipLaunchKernelGGL(k_wmul, grid_of(ctx, d.L, n, 1), dim3(kThreads), 0, ctx->stream, a, u, d, pages, ctx->d_mod);
        prof_end(ctx, K_ELEM);
    }
    HIP_TRY(hipGetLastError());

    LimbMap m = limb_range(level, 1);
    for (uint32_t i = 0; i < d.K; i++) m.prime[m.n++] = (uint8_t)(d.n_q + i);
    uint64_t *top = u + (size_t)level * N;
    CK_TRY(launch_ntt_strided(ctx, top, polys, d.ext, m, true));

    const ConvDev none{}, *cd = &none;
    if (rot) CK_TRY(ctx_conv(ctx, (int)level, -1, &cd));
    bool below60 = d.K <= 8;
    for (uint32_t i = 0; i < m.n; i++) below60 = below60 && ctx->primes[m.prime[i]] >> 60 == 0;
    for (uint32_t i = 0; i < level; i++) below60 = below60 && ctx->primes[i] >> 60 == 0;
    // groups of targets until the grid has eight waves a SIMD: 2048 blocks (four polynomials of 36 targets: 53 us undivided,
    // 48 in two groups, 55 in four, each of which forms the digits and w again).  us a call with none, groups to 1024, 2048,
    // 4096 and 8192 blocks: one ciphertext of 37 limbs at N = 2^16 488, 479, 478, 483, 490; four 1364, 1361, 1364, 1366,
    // 1380; one of 10 limbs 166, 164, 163, 167, 173; four at 2^14 154, 153, 153, 156, 159; one at 2^12 82, 78, 78, 78, 79
    const uint32_t blocks = grid_of(ctx, 1, 1, 1).x * polys, groups = std::min(level, std::max(1u, 2048u / blocks));
    const uint32_t t_per = (level + groups - 1) / groups;
    const dim3 grid(grid_of(ctx, 1, 1, 1).x, (level + t_per - 1) / t_per, polys);
    prof_begin(ctx, K_CONV, 8.0 * N * polys * (d.K + 1.0 + level));
#define CK_QUOT(KERN)                                                                                              \
    hipLaunchKernelGGL(KERN, grid, dim3(kThreads), 0, ctx->stream, x, top, d, (int)d.K, t_per, cd->d_qhat_inv,     \
                       cd->d_qhat_mod, cd->d_neg_q, ctx->d_pinv, ctx->d_pmodq, ctx->d_mod)
    if (below60) CK_QUOT(k_quot60);
    else if (d.K <= 8) CK_QUOT(k_quot<8>);
    else if (d.K <= 16) CK_QUOT(k_quot<16>);
    else CK_QUOT(k_quot<kMaxPrimes>);
#undef CK_QUOT
    prof_end(ctx, K_CONV);
    HIP_TRY(hipGetLastError());

    const ulonglong2 *f = (rot ? ctx->d_pqlinv : ctx->d_qlinv) + (size_t)level * ctx->n_q;
    if (fused_rows_ok(ctx)) {
        static_assert(kWsumCts * kWsumPages <= (uint32_t)kRotBatch, "a batch's outputs fit the list");
        RotArgs ra{};
        ra.count = outs;
        for (uint32_t i = 0; i < outs; i++) {
            const uint64_t *prev = a.ct[i / pages].prev[i % pages];
            ra.g[i] = 1;
            ra.out[i] = a.ct[i / pages].out[i % pages];
            ra.c0[i] = prev;
            ra.add1[i] = prev ? prev + (size_t)level * N : nullptr;
        }
        CK_TRY(launch_ntt_fwd_first_pass(ctx, x, polys, level, limb_range(0, level)));
        return fused_quotient(ctx, level, d.ext, ra, u, x, f);
    }
    CK_TRY(launch_ntt(ctx, x, polys * level, limb_range(0, level), false));
    prof_begin(ctx, K_ELEM, 8.0 * N * level * polys * 4.0);
    hipLaunchKernelGGL(k_finish, grid_of(ctx, 2 * level, outs, 1), dim3(kThreads), 0, ctx->stream, a, u, x, d, pages, f,
                       ctx->d_mod);
    prof_end(ctx, K_ELEM);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

// Steps (step.h) with fp64 arithmetic in two passes a transform (N >= 2^14, every prime of the level below 2^50), with one
// division by P q_l (wsum.hip) and nothing of a step in HBM but its digits and the rows that a transform's two passes
// exchange:
//   1. the ModUp of the products d2, formed where its row pass reads them (k_up_row of a PolyProd), up to the column pass
//      of the digits' forward transforms;
//   2. k_step_intt8   their row pass, u = P (d0, d1) + <digits, rlk> on the rows q_l and P, the row pass of u's inverse
//      transform;
//   3. wsum_convert   its column pass, the conversion, the column pass of the forward transform;
//   4. k_step_fin8    the row passes of that and of the digits, u on the rows below q_l, out = (u - NTT(x)) (P q_l)^-1.
// Steps without a product of ciphertexts have no digits and no rows P: u = (d0, d1), divided by q_l.
// SiLU of 8 ciphertexts of 13 limbs at N = 2^16: 4.93 ms from the separate stages, 3.60 with one division and digits that
// end their transforms in a launch of the ModUp, 2.9 so.  There, averages of 8 launches: k_step_intt8 65 us at 71% of the
// issue slots, k_step_fin8 113 us at 59% and 4.8 TB/s: the fp64 pipes and HBM bound them together.
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "step_args.h"
#include "wsum_pos.h"

namespace {

using namespace wsum;
using namespace steps;

// A half wave's row pass: forward twiddles of the row's prime and the transposes' memory.
struct RowPass {
    const double *tws;
    double *tr;
    uint32_t t;
};

// u at the 8 positions of a thread, both components, |u| <= q/2 + 1.  Q: the row is one of the q limbs (the P rows have
// no d0, d1).  The digits' rows come after their column pass and end their transforms here: a relinearisation reads each
// once, so they need not be written.  A digit's own row is d2 and is taken first.  In units of q: a digit below 2.6, its
// product with a key below 1.5, four of them and what is left of those before, below 7.
template <bool Q>
__device__ __forceinline__ void step8(const Operands &s, const uint64_t *dig, const uint64_t *key0, const Dims &d,
                                      uint32_t row, double pq, const A &ar, const A &top, const Positions &ps,
                                      const RowPass &rp, uint32_t h, double (&u)[2][kE8])
{
    const size_t rw = (size_t)row << d.log_n;
    const bool sw = s.switched();
    const uint32_t kind = Q ? s.kind() : kNone, own = Q ? row / d.alpha : ~0u;
    const size_t kstride = (size_t)d.key_rows << d.log_n;
    const uint64_t *key = key0 + ((size_t)d.prime(row) << d.log_n);
    double x[kE8], next[kE8];
    auto ask = [&](uint32_t i) {
        const uint64_t *p = dig + ((size_t)i * d.ext << d.log_n) + rw + (size_t)h * 256;
#pragma unroll
        for (int e = 0; e < kE8; e++) next[e] = A::from_raw(nttc::ld_stream(p + nttc::u8<0>(rp.t, e)));
    };
    const uint32_t first = own == 0 ? 1 : 0;
    if (sw && first < d.nd) ask(first);
#pragma unroll
    for (int e = 0; e < kE8; e++) u[0][e] = u[1][e] = 0.0;
    if constexpr (Q) {
        // linear terms: a product at most 0.875 q, reduced every four
        for (uint32_t i = 0; i < s.n(); i++) {
            const double k = int_mod(s.k[i], s.sh(i), ar);
            const uint64_t *z = s.z[i] + rw;
            Pair v[2][kE8 / 2];
            const bool two = s.two(i);
#pragma unroll
            for (int e = 0; e < kE8; e += 2) v[0][e / 2] = ld2(z + ps.pos(e));
            if (two) {
                const uint64_t *z1 = z + ((size_t)s.limbs(i) << d.log_n);
#pragma unroll
                for (int e = 0; e < kE8; e += 2) v[1][e / 2] = ld2(z1 + ps.pos(e));
            }
#pragma unroll
            for (int c = 0; c < 2; c++) {
                if (c && !two) break;
#pragma unroll
                for (int e = 0; e < kE8; e += 2) {
                    u[c][e] += ar.mul(A::from_u64(v[c][e / 2].x), k);
                    u[c][e + 1] += ar.mul(A::from_u64(v[c][e / 2].y), k);
                }
            }
            if ((i & 3) == 3) {
#pragma unroll
                for (int e = 0; e < kE8; e++) {
                    u[0][e] = ar.red(u[0][e]);
                    u[1][e] = ar.red(u[1][e]);
                }
            }
        }
        // the constant c as c q_l, which the division leaves as c
        if (s.k[kStepTerms]) {
            const double ql = ar.red(top.q);
            const double c = ar.mul(int_mod(s.k[kStepTerms], s.sh(kStepTerms), ar), ql < 0.0 ? ql + ar.q : ql);
#pragma unroll
            for (int e = 0; e < kE8; e++) u[0][e] += c;
        }
        // the product's operands (a0, a1, b0, b1; a0, a1, plaintext; d0, d1, d2), four positions at a time, and the key's
        // words for d2
        const double mult = s.mult;
        const uint64_t *kb = key + 2 * own * kstride, *ka = kb + kstride;
        auto finish = [&](auto is) {
            constexpr uint32_t KIND = decltype(is)::value;
            constexpr bool SW = KIND == kProduct || KIND == kGiven;
            const uint64_t *w0 = s.a + rw, *w1 = w0 + ((size_t)(KIND == kGiven ? d.L : s.a_limbs()) << d.log_n),
                           *w2 = KIND == kGiven ? w1 + ((size_t)d.L << d.log_n) : s.b + rw,
                           *w3 = w2 + ((size_t)s.b_limbs() << d.log_n);
#pragma unroll
            for (int e0 = 0; e0 < kE8; e0 += 4) {
                Pair w[4][2], b[2], a[2];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int p = 0; p < 2; p++) {
                    const uint32_t at = ps.pos(e0 + 2 * p);
                    if constexpr (KIND != kNone) {
                        w[0][p] = ld2(w0 + at);
                        w[1][p] = ld2(w1 + at);
                        w[2][p] = ld2(w2 + at);
                    }
                    if constexpr (KIND == kProduct) w[3][p] = ld2(w3 + at);
                    if constexpr (SW) {
                        b[p] = ld2(kb + at);
                        a[p] = ld2(ka + at);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int o = 0; o < 4; o++) {
                    const int e = e0 + o;
                    auto get = [&](const Pair &v) { return A::from_u64(o & 1 ? v.y : v.x); };
                    auto word = [&](int j) { return get(w[j][o / 2]); };
                    double d2 = 0.0;
                    if constexpr (KIND == kProduct) {
                        const double a0 = word(0), a1 = word(1), b0 = word(2), b1 = word(3);
                        ProductSum p1;
                        p1.add(a0, b1);
                        p1.add(a1, b0);
                        u[0][e] += mult * ar.mul(a0, b0);
                        u[1][e] += mult * p1.value(ar);
                        d2 = ar.red(mult * ar.mul(a1, b1));
                    } else if constexpr (KIND == kPlain) {
                        u[0][e] += ar.mul(word(0), word(2));
                        u[1][e] += ar.mul(word(1), word(2));
                    } else if constexpr (KIND == kGiven) {
                        u[0][e] += word(0);
                        u[1][e] += word(1);
                        d2 = word(2);
                    }
                    u[0][e] = ar.red(u[0][e]);
                    u[1][e] = ar.red(u[1][e]);
                    if constexpr (SW) {
                        u[0][e] = ar.red(ar.mul(u[0][e], pq) + ar.mul(d2, get(b[o / 2])));
                        u[1][e] = ar.red(ar.mul(u[1][e], pq) + ar.mul(d2, get(a[o / 2])));
                    }
                }
            }
        };
        if (kind == kProduct) finish(std::integral_constant<uint32_t, kProduct>());
        else if (kind == kNone) finish(std::integral_constant<uint32_t, kNone>());
        else if (kind == kPlain) finish(std::integral_constant<uint32_t, kPlain>());
        else finish(std::integral_constant<uint32_t, kGiven>());
    }
    if (!sw) return;
#pragma unroll 1
    for (uint32_t i = first, n = 0; i < d.nd; n++) {
        const uint32_t j = i + 1 == own ? i + 2 : i + 1;   // the next digit
        Pair kb[kE8 / 2], ka[kE8 / 2];
        uint32_t t = rp.t;
        asm volatile("" : "+v"(t));   // the twiddles' reads stay in the loop: held across it they cost a wave a SIMD
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < kE8; e += 2) {
            kb[e / 2] = ld2(key + 2 * i * kstride + ps.pos(e));
            ka[e / 2] = ld2(key + (2 * i + 1) * kstride + ps.pos(e));
        }
#pragma unroll
        for (int e = 0; e < kE8; e++) x[e] = next[e];
        if (j < d.nd) ask(j);
        __builtin_amdgcn_sched_barrier(0);
        nttc::fwd8_256<nttc::kRowMask8>(x, rp.tws, rp.tr, t, ar);
        swap_1_6(x);
#pragma unroll
        for (int e = 0; e < kE8; e++) {
            const Pair &b = kb[e / 2], &a = ka[e / 2];
            u[0][e] += ar.mul(x[e], A::from_u64(e & 1 ? b.y : b.x));
            u[1][e] += ar.mul(x[e], A::from_u64(e & 1 ? a.y : a.x));
        }
        if ((n & 3) == 3 || j >= d.nd) {
#pragma unroll
            for (int e = 0; e < kE8; e++) {
                u[0][e] = ar.red(u[0][e]);
                u[1][e] = ar.red(u[1][e]);
            }
        }
        i = j;
    }
}

// 2. rows q_l and P (s = 0: q_l, s > 0: p_{s-1}) of u: up[z][k][s], raw doubles below 2q after the row pass.  One wave, two
// rows of 256 points, 8 positions a thread.
__global__ __launch_bounds__(64) void k_step_intt8(Batch bt, const uint64_t *dig, const uint64_t *rlk, uint64_t *up,
                                                   Dims d, uint32_t n, const ulonglong2 *__restrict__ pmodq,
                                                   const ModQ *__restrict__ mods, const double *__restrict__ twf,
                                                   const double *__restrict__ itwf)
{
    __shared__ double tws[2][257];
    __shared__ double tr[2][nttc::kTr8];
    const uint32_t bpl = 1u << (d.log_n - 9);
    uint32_t z, tile;
    tile_of(n, z, tile);
    const uint32_t s = tile / bpl, blk = tile % bpl, row = d.L - 1 + s, prime = d.prime(row);
    const Operands &o = bt.s[z];
    if (s && !o.switched()) return;
    const A ar(mods[prime]);
    const uint32_t sub = threadIdx.x >> 5, t = threadIdx.x & 31, h = blk * 2 + sub;
    nttc::stage_twiddles8(tws[sub], twf + ((size_t)prime << d.log_n), (1u << (d.log_n - 8)) + h, t, 32);
    const Positions ps(h, t, d.log_n);
    const RowPass rp{tws[sub], tr[sub], t};
    __syncthreads();
    const uint64_t *mine = dig + ((size_t)z * d.nd * d.ext << d.log_n);
    double u[2][kE8];
    if (s) step8<false>(o, mine, rlk, d, row, 0.0, ar, ar, ps, rp, h, u);
    else step8<true>(o, mine, rlk, d, row, (double)pmodq[row].x, ar, ar, ps, rp, h, u);
    __syncthreads();
    nttc::stage_twiddles8(tws[sub], itwf + ((size_t)prime << d.log_n), (1u << (d.log_n - 8)) + h, t, 32);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; k++) {
        swap_1_6(u[k]);
        nttc::inv8_256(u[k], tws[sub], tr[sub], t, ar);
        uint64_t *out = up + ((((size_t)z * 2 + k) * (d.K + 1) + s) << d.log_n) + (size_t)h * 256;
#pragma unroll
        for (int e = 0; e < kE8; e++) nttc::st_stream(out + nttc::u8<0>(t, e), A::to_raw(u[k][e]));
    }
}

// 4. out = (u - NTT(x)) (P q_l)^-1 on the rows below q_l: cw[z][k][l] after the column pass.  In units of q: column-pass
// rows below 4.3, transformed below 2.6, u below 0.6: differences below 8.
__global__ __launch_bounds__(64) void k_step_fin8(Batch bt, const uint64_t *dig, const uint64_t *rlk,
                                                  const uint64_t *__restrict__ cw, Dims d, uint32_t n, Quot qt,
                                                  const ModQ *__restrict__ mods, const double *__restrict__ twf)
{
    __shared__ double tws[2][257];
    __shared__ double tr[2][nttc::kTr8];
    const uint32_t bpl = 1u << (d.log_n - 9), l = d.L - 1;
    uint32_t z, tile;
    tile_of(n, z, tile);
    const uint32_t row = tile / bpl, blk = tile % bpl;
    const Operands &o = bt.s[z];
    const A ar(mods[row]), top(mods[l]);
    const uint32_t sub = threadIdx.x >> 5, t = threadIdx.x & 31, h = blk * 2 + sub;
    nttc::stage_twiddles8(tws[sub], twf + ((size_t)row << d.log_n), (1u << (d.log_n - 8)) + h, t, 32);
    const Positions ps(h, t, d.log_n);
    double u[2][kE8], x[2][kE8];
    const RowPass rp{tws[sub], tr[sub], t};
    __syncthreads();
    step8<true>(o, dig + ((size_t)z * d.nd * d.ext << d.log_n), rlk, d, row, (double)qt.pmodq[row].x, ar, top, ps, rp, h,
                    u);
    const uint64_t *src = cw + (((size_t)z * 2 * l + row) << d.log_n) + (size_t)h * 256;
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
        for (int e = 0; e < kE8; e++)
            x[k][e] = A::from_raw(nttc::ld_stream(src + ((size_t)k * l << d.log_n) + nttc::u8<0>(t, e)));
    // (P q_l)^-1, or q_l^-1 where u has no factor P, canonical
    double f = (double)qt.qlinv[row].x;
    if (o.switched()) {
        f = centre(ar, ar.mul(f, (double)qt.pinv[row].x));
        f = f < 0.0 ? f + ar.q : f;
    }
#pragma unroll
    for (int k = 0; k < 2; k++) {
        nttc::fwd8_256<nttc::kRowMask8>(x[k], tws[sub], tr[sub], t, ar);
        swap_1_6(x[k]);
        uint64_t *out = o.out + ((size_t)(k * l + row) << d.log_n);
#pragma unroll
        for (int e = 0; e < kE8; e += 2)
            *(Pair *)(out + ps.pos(e)) =
                Pair{quotient(ar, u[k][e] - x[k][e], f), quotient(ar, u[k][e + 1] - x[k][e + 1], f)};
    }
}

}  // namespace

ckks_status step_f64(ckks_ctx *ctx, uint32_t L, const Batch &b, uint32_t n, uint32_t n_sw, const uint64_t *rlk,
                     uint64_t *mem)
{
    static_assert(kStepBatch <= (uint32_t)kPolyList && kStepBatch <= kWsumCts, "a batch fits the lists");
    Dims d = wsum_dims(ctx, L);
    const size_t N = ctx->n;
    const uint32_t level = L - 1, bpl = 1u << (d.log_n - 9);
    uint64_t *dig = mem, *up = dig + (size_t)n_sw * d.nd * d.ext * N;
    if (n_sw) {
        CK_TRY(up_modup_cols(ctx, step_sources(ctx, L, b, n_sw), n_sw, level, dig));
    } else {
        d.K = 0;
        d.ext = L;
    }
    uint64_t *cw = up + 2 * (size_t)n * (d.K + 1) * N;
    Args a{};
    a.kind[0].rotated = 1;
    for (uint32_t i = 0; i < n; i++) a.ct[i].kind = i < n_sw ? 0 : 1;
    const ConvDev *cd;
    CK_TRY(ctx_conv(ctx, (int)level, -1, &cd));
    const Quot qt{cd->d_qhat_inv_f, cd->d_qhat_mod_f, ctx->d_pinv, ctx->d_qlinv + (size_t)level * ctx->n_q, ctx->d_pmodq};
    double terms = 0;
    for (uint32_t i = 0; i < n; i++) terms += 2.0 * b.s[i].n() + (b.s[i].kind() == kProduct ? 4 : b.s[i].kind() ? 3 : 0);
    const double rows1 = (double)n_sw * d.K * N;
    prof_begin(ctx, K_KEYIP, 8.0 * (rows1 * (d.nd + 2.0) + N * (terms + n_sw * d.nd + 2.0 * n)),
               rows1 * (4.0 * d.nd * 4 + 2 * 4 * kOpsButterflyF64));
    hipLaunchKernelGGL(k_step_intt8, dim3((d.K + 1) * bpl * n), dim3(64), 0, ctx->stream, b, dig, rlk, up, d, n,
                       ctx->d_pmodq, ctx->d_mod, ctx->d_twf, ctx->d_itwf);
    prof_end(ctx, K_KEYIP);
    HIP_TRY(hipGetLastError());
    CK_TRY(wsum_convert(ctx, a, n, 1, d, up, cw));
    prof_begin(ctx, K_MODDOWN, 8.0 * N * level * (terms + n_sw * (d.nd - 1.0) + 4.0 * n),
               (double)N * level * n * (4.0 * d.nd * 4 + 2 * (4 * kOpsButterflyF64 + 14.0)));
    hipLaunchKernelGGL(k_step_fin8, dim3(level * bpl * n), dim3(64), 0, ctx->stream, b, dig, rlk, cw, d, n, qt, ctx->d_mod,
                       ctx->d_twf);
    prof_end(ctx, K_MODDOWN);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

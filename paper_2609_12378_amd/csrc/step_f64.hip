// Steps (step.h) with fp64 arithmetic in two passes a transform (N >= 2^14, every prime of the level below 2^50), with one
// division by P q_l (wsum.hip) and nothing of a step in HBM but its digits and the rows that a transform's two passes
// exchange:
//   1. the ModUp of the products d2, formed where its row pass reads them (k_up_row of a PolyProd);
//   2. k_step_intt8   u = P (d0, d1) + <digits, rlk> on the rows q_l and P, with the row pass of their inverse transform;
//   3. wsum_convert   their column pass, the conversion, the column pass of the forward transform;
//   4. k_step_fin8    its row pass, u on the rows below q_l, out = (u - NTT(x)) (P q_l)^-1.
// Steps without a product of ciphertexts have no digits and no rows P: u = (d0, d1), divided by q_l.
#include <algorithm>

#include "ops.h"
#include "step_args.h"
#include "wsum_pos.h"

namespace {

using namespace wsum;
using namespace steps;

// The words of a pair of positions: a product's operands (a0, a1, b0, b1; a0, a1, plaintext; d0, d1, d2), the digits and
// the key's two halves.  A unit's loads are issued together and the next unit's before its sums.
template <int ND>
struct Unit {
    Pair w[4], dig[ND], b[ND], a[ND];
};

// u at the 8 positions of a thread, both components, |u| <= q/2 + 1.  Q: the row is one of the q limbs (the P rows have
// no d0, d1).  A digit's own row is d2, formed again.
template <int ND, bool Q>
__device__ __forceinline__ void step8(const Operands &s, const uint64_t *dig, const uint64_t *key0, const Dims &d,
                                      uint32_t row, double pq, const A &ar, const A &top, const Positions &ps,
                                      double (&u)[2][kE8])
{
    const size_t rw = (size_t)row << d.log_n;
    const bool sw = s.switched();
#pragma unroll
    for (int e = 0; e < kE8; e++) u[0][e] = u[1][e] = 0.0;
    if constexpr (Q) {
        // linear terms: a product at most 0.875 q, reduced every four
        for (uint32_t i = 0; i < s.n; i++) {
            const double k = int_mod(s.k[i], s.sh[i], ar);
            const uint64_t *z = s.z[i] + rw;
            Pair v[2][kE8 / 2];
            const bool two = s.polys[i] == 2;
#pragma unroll
            for (int e = 0; e < kE8; e += 2) v[0][e / 2] = ld2(z + ps.pos(e));
            if (two) {
                const uint64_t *z1 = z + ((size_t)s.limbs[i] << d.log_n);
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
            const double c = ar.mul(int_mod(s.k[kStepTerms], s.sh[kStepTerms], ar), ql < 0.0 ? ql + ar.q : ql);
#pragma unroll
            for (int e = 0; e < kE8; e++) u[0][e] += c;
        }
    }
    const uint32_t kind = Q ? s.kind : kNone, own = Q ? row / d.alpha : ~0u;
    const size_t kstride = (size_t)d.key_rows << d.log_n, dstride = (size_t)d.ext << d.log_n;
    const uint64_t *key = key0 + ((size_t)d.prime(row) << d.log_n);
    const double mult = s.mult;
    const uint64_t *w0 = s.a + rw, *w1, *w2 = s.b + rw, *w3 = w2;
    if (kind == kGiven) {
        w1 = w0 + ((size_t)d.L << d.log_n);
        w2 = w1 + ((size_t)d.L << d.log_n);
    } else {
        w1 = w0 + ((size_t)s.a_limbs << d.log_n);
        if (kind == kProduct) w3 = w2 + ((size_t)s.b_limbs << d.log_n);
    }
    auto load = [&](Unit<ND> &x, int p) {
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t at = ps.pos(2 * p);
        if (kind != kNone) {
            x.w[0] = ld2(w0 + at);
            x.w[1] = ld2(w1 + at);
            x.w[2] = ld2(w2 + at);
            if (kind == kProduct) x.w[3] = ld2(w3 + at);
        }
        if (sw) {
#pragma unroll
            for (int i = 0; i < ND; i++) {
                if ((uint32_t)i != own) x.dig[i] = ld2(dig + i * dstride + rw + at);
                x.b[i] = ld2(key + 2 * i * kstride + at);
                x.a[i] = ld2(key + (2 * i + 1) * kstride + at);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto half = [&](const Unit<ND> &x, int e, auto word) {
        double d2 = 0.0;
        if constexpr (Q) {
            if (kind == kProduct) {
                const double a0 = A::from_u64(word(x.w[0])), a1 = A::from_u64(word(x.w[1])), b0 = A::from_u64(word(x.w[2])),
                             b1 = A::from_u64(word(x.w[3]));
                ProductSum p1;
                p1.add(a0, b1);
                p1.add(a1, b0);
                u[0][e] = ar.red(u[0][e] + mult * ar.mul(a0, b0));
                u[1][e] = ar.red(u[1][e] + mult * p1.value(ar));
                d2 = ar.red(mult * ar.mul(a1, b1));
            } else if (kind == kPlain) {
                const double p = A::from_u64(word(x.w[2]));
                u[0][e] = ar.red(u[0][e] + ar.mul(A::from_u64(word(x.w[0])), p));
                u[1][e] = ar.red(u[1][e] + ar.mul(A::from_u64(word(x.w[1])), p));
            } else if (kind == kGiven) {
                u[0][e] = ar.red(u[0][e] + A::from_u64(word(x.w[0])));
                u[1][e] = ar.red(u[1][e] + A::from_u64(word(x.w[1])));
                d2 = A::from_u64(word(x.w[2]));
            } else {
                u[0][e] = ar.red(u[0][e]);
                u[1][e] = ar.red(u[1][e]);
            }
        }
        if (!sw) return;
        ProductSum s0, s1;
        if constexpr (Q) {
            s0.add(u[0][e], pq);
            s1.add(u[1][e], pq);
        }
#pragma unroll
        for (int i = 0; i < ND; i++) {
            if (i && i % 3 == 0) {   // P d and three products
                s0.fold(ar);
                s1.fold(ar);
            }
            const double v = (uint32_t)i == own ? d2 : A::from_u64(word(x.dig[i]));
            s0.add(v, A::from_u64(word(x.b[i])));
            s1.add(v, A::from_u64(word(x.a[i])));
        }
        u[0][e] = s0.value(ar);
        u[1][e] = s1.value(ar);
    };
    auto use = [&](const Unit<ND> &x, int p) {
        half(x, 2 * p, [](const Pair &v) { return v.x; });
        half(x, 2 * p + 1, [](const Pair &v) { return v.y; });
        // ahead of the next unit's loads: the compiler would gather the sums behind the last load, with every word held
        asm volatile("" : "+v"(u[0][2 * p]), "+v"(u[1][2 * p]), "+v"(u[0][2 * p + 1]), "+v"(u[1][2 * p + 1]));
    };
    Unit<ND> x0, x1;
    load(x0, 0);
    load(x1, 1);
    use(x0, 0);
    load(x0, 2);
    use(x1, 1);
    load(x1, 3);
    use(x0, 2);
    use(x1, 3);
}

// 2. rows q_l and P (s = 0: q_l, s > 0: p_{s-1}) of u: up[z][k][s], raw doubles below 2q after the row pass.  One wave, two
// rows of 256 points, 8 positions a thread.
template <int ND>
__global__ __launch_bounds__(64) void k_step_intt8(Batch bt, const uint64_t *dig, const uint64_t *rlk, uint64_t *up,
                                                   Dims d, uint32_t n, const ulonglong2 *__restrict__ pmodq,
                                                   const ModQ *__restrict__ mods, const double *__restrict__ itwf)
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
    nttc::stage_twiddles8(tws[sub], itwf + ((size_t)prime << d.log_n), (1u << (d.log_n - 8)) + h, t, 32);
    const Positions ps(h, t, d.log_n);
    const uint64_t *mine = dig + ((size_t)z * d.nd * d.ext << d.log_n);
    double u[2][kE8];
    if (s) step8<ND, false>(o, mine, rlk, d, row, 0.0, ar, ar, ps, u);
    else step8<ND, true>(o, mine, rlk, d, row, (double)pmodq[row].x, ar, ar, ps, u);
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
template <int ND>
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
    step8<ND, true>(o, dig + ((size_t)z * d.nd * d.ext << d.log_n), rlk, d, row, (double)qt.pmodq[row].x, ar, top, ps, u);
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
    __syncthreads();
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

bool step_f64_ok(const ckks_ctx *ctx, uint32_t L)
{
    return L >= 2 && ctx->log_n >= 14 && f64_switch(ctx, L - 1) && n_digits(ctx, L - 1) <= 5;
}

// rows of N words: the digits, the rows q_l and P of u, the converted rows
size_t step_f64_rows(const ckks_ctx *ctx, uint32_t L, size_t n, bool switched)
{
    const size_t K = switched ? ctx->n_p : 0, dig = switched ? (size_t)n_digits(ctx, L - 1) * (L + K) : 0;
    return n * (dig + 2 * (K + 1) + 2 * (L - 1));
}

ckks_status step_f64(ckks_ctx *ctx, uint32_t L, const Batch &b, uint32_t n, uint32_t n_sw, const uint64_t *rlk,
                     uint64_t *mem)
{
    static_assert(kStepBatch <= (uint32_t)kPolyList && kStepBatch <= kWsumCts, "a batch fits the lists");
    Dims d = wsum_dims(ctx, L);
    const size_t N = ctx->n;
    const uint32_t level = L - 1, bpl = 1u << (d.log_n - 9);
    uint64_t *dig = mem, *up = dig + (size_t)n_sw * d.nd * d.ext * N;
    if (n_sw) {
        PolyProd src{};
        for (uint32_t i = 0; i < n_sw; i++) {
            const Operands &s = b.s[i];
            src.list[i] = s.a + (s.kind == kGiven ? 2 * (size_t)L : s.a_limbs) * N;
            src.mul[i] = s.kind == kGiven ? nullptr : s.b + (size_t)s.b_limbs * N;
            src.mult[i] = s.mult;
        }
        CK_TRY(up_modup(ctx, src, n_sw, level, dig));
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
    for (uint32_t i = 0; i < n; i++) terms += 2.0 * b.s[i].n + (b.s[i].kind == kProduct ? 4 : b.s[i].kind ? 3 : 0);
    const double rows1 = (double)n_sw * d.K * N;
    prof_begin(ctx, K_KEYIP, 8.0 * (rows1 * (d.nd + 2.0) + N * (terms + n_sw * d.nd + 2.0 * n)),
               rows1 * (4.0 * d.nd * 4 + 2 * 4 * kOpsButterflyF64));
#define CK_STEP(KERNEL, GRID, ...)                                                                                 \
    do {                                                                                                           \
        switch (d.nd) {                                                                                            \
        case 1: hipLaunchKernelGGL(KERNEL<1>, GRID, dim3(64), 0, ctx->stream, __VA_ARGS__); break;                 \
        case 2: hipLaunchKernelGGL(KERNEL<2>, GRID, dim3(64), 0, ctx->stream, __VA_ARGS__); break;                 \
        case 3: hipLaunchKernelGGL(KERNEL<3>, GRID, dim3(64), 0, ctx->stream, __VA_ARGS__); break;                 \
        case 4: hipLaunchKernelGGL(KERNEL<4>, GRID, dim3(64), 0, ctx->stream, __VA_ARGS__); break;                 \
        default: hipLaunchKernelGGL(KERNEL<5>, GRID, dim3(64), 0, ctx->stream, __VA_ARGS__); break;                \
        }                                                                                                          \
    } while (0)
    CK_STEP(k_step_intt8, dim3((d.K + 1) * bpl * n), b, dig, rlk, up, d, n, ctx->d_pmodq, ctx->d_mod, ctx->d_itwf);
    prof_end(ctx, K_KEYIP);
    HIP_TRY(hipGetLastError());
    CK_TRY(wsum_convert(ctx, a, n, 1, d, up, cw));
    prof_begin(ctx, K_MODDOWN, 8.0 * N * level * (terms + n_sw * (d.nd - 1.0) + 4.0 * n),
               (double)N * level * n * (4.0 * d.nd * 4 + 2 * (4 * kOpsButterflyF64 + 14.0)));
    CK_STEP(k_step_fin8, dim3(level * bpl * n), b, dig, rlk, cw, d, n, qt, ctx->d_mod, ctx->d_twf);
#undef CK_STEP
    prof_end(ctx, K_MODDOWN);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

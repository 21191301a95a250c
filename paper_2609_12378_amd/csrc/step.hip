// Steps on ciphertexts (step.h).
#include "step.h"

#include <algorithm>
#include <cmath>

#include "ks_args.h"
#include "ops.h"
#include "step_args.h"

namespace {

constexpr int kThreads = 256;

using namespace steps;
using namespace wsum;

// v times 1, 2 or -1 mod q
__device__ __forceinline__ uint64_t times(uint64_t v, int mult, uint64_t q)
{
    return mult == 2 ? csub(2 * v, q) : mult < 0 && v ? q - v : v;
}

// d2 of the steps that switch a key to out[z][L][N], two positions a thread
__global__ __launch_bounds__(kThreads) void k_step_d2(Batch bt, uint64_t *out, uint32_t L, uint32_t log_n,
                                                      const ModQ *__restrict__ mods)
{
    const Operands &s = bt.s[blockIdx.z];
    const uint32_t row = blockIdx.y, col = 2 * (blockIdx.x * kThreads + threadIdx.x);
    if (col >> log_n) return;
    const ModQ m = mods[row];
    const size_t at = ((size_t)row << log_n) + col;
    Pair v = ld2(s.a + at + ((size_t)(s.kind() == kGiven ? 2 * L : s.a_limbs()) << log_n));
    if (s.kind() == kProduct) {
        const Pair w = ld2(s.b + at + ((size_t)s.b_limbs() << log_n));
        v = Pair{times(mulmod(v.x, w.x, m), s.mult, m.q), times(mulmod(v.y, w.y, m), s.mult, m.q)};
    }
    *(Pair *)(out + ((size_t)blockIdx.z * L << log_n) + at) = v;
}

// u[z][k][row] (wsum.hip) of every step, all of which switch a key or none, in exact 128-bit sums: a step's linear part is
// at most 11 products below 2^124.  The constant goes in as c q_l: it vanishes modulo q_l and the division leaves c.  A
// digit's own row is d2, formed again.  Two positions a thread.  Bound by integer issue: two ciphertexts of 20 limbs of 59
// bits at N = 2^16, 62 us a launch at 82% of the issue slots and 4.3 TB/s.
__global__ __launch_bounds__(kThreads) void k_step_u(Batch bt, const uint64_t *dig, const uint64_t *rlk, uint64_t *u, Dims d,
                                                     uint32_t n, uint32_t per_row, const ulonglong2 *__restrict__ pmodq,
                                                     const ModQ *__restrict__ mods)
{
    __shared__ uint64_t ks[kStepTerms + 1];
    uint32_t z, tile;
    tile_of(n, z, tile);
    const uint32_t row = tile / per_row, col = 2 * (tile % per_row * kThreads + threadIdx.x);
    if (row >= d.ext) return;
    const Operands &s = bt.s[z];
    const uint32_t prime = d.prime(row);
    const ModQ m = mods[prime];
    const bool q_row = row < d.L;
    if (q_row && threadIdx.x <= s.n()) {
        const uint32_t i = threadIdx.x < s.n() ? threadIdx.x : kStepTerms;
        const uint64_t r = int_mod(s.k[i], s.sh(i), m.q);
        ks[threadIdx.x] = i < kStepTerms ? r : mulmod(r, mods[d.L - 1].q % m.q, m);
    }
    __syncthreads();
    if (col >> d.log_n) return;
    const size_t at = ((size_t)row << d.log_n) + col, half = (size_t)d.L << d.log_n;
    uint64_t r[2][2] = {}, d2[2] = {};   // [component][position]
    if (q_row) {
        acc128 x[2][2] = {{{ks[s.n()], 0}, {ks[s.n()], 0}}, {}};
        if (s.kind() == kGiven) {
            const Pair v0 = ld2(s.a + at), v1 = ld2(s.a + half + at), v2 = ld2(s.a + 2 * half + at);
            mac(x[0][0], v0.x, 1);
            mac(x[0][1], v0.y, 1);
            mac(x[1][0], v1.x, 1);
            mac(x[1][1], v1.y, 1);
            d2[0] = v2.x;
            d2[1] = v2.y;
        } else if (s.kind() != kNone) {
            const Pair a0 = ld2(s.a + at), a1 = ld2(s.a + at + ((size_t)s.a_limbs() << d.log_n)), b0 = ld2(s.b + at);
            const uint64_t c0 = times(b0.x, s.mult, m.q), c1 = times(b0.y, s.mult, m.q);
            mac(x[0][0], a0.x, c0);
            mac(x[0][1], a0.y, c1);
            mac(x[1][0], a1.x, c0);
            mac(x[1][1], a1.y, c1);
            if (s.kind() == kProduct) {
                const Pair b1 = ld2(s.b + at + ((size_t)s.b_limbs() << d.log_n));
                const uint64_t e0 = times(b1.x, s.mult, m.q), e1 = times(b1.y, s.mult, m.q);
                mac(x[1][0], a0.x, e0);
                mac(x[1][1], a0.y, e1);
                d2[0] = mulmod(a1.x, e0, m);
                d2[1] = mulmod(a1.y, e1, m);
            }
        }
        for (uint32_t i = 0; i < s.n(); i++) {
            const Pair v = ld2(s.z[i] + at);
            mac(x[0][0], v.x, ks[i]);
            mac(x[0][1], v.y, ks[i]);
            if (!s.two(i)) continue;
            const Pair w = ld2(s.z[i] + at + ((size_t)s.limbs(i) << d.log_n));
            mac(x[1][0], w.x, ks[i]);
            mac(x[1][1], w.y, ks[i]);
        }
#pragma unroll
        for (int k = 0; k < 4; k++) r[k >> 1][k & 1] = reduce128(x[k >> 1][k & 1], m);
    }
    if (s.switched()) {
        const uint64_t pq = q_row ? pmodq[row].x : 0;
        const uint32_t own = q_row ? row / d.alpha : d.nd;
        acc128 t[2][2] = {};
#pragma unroll
        for (int k = 0; k < 4; k++) mac(t[k >> 1][k & 1], r[k >> 1][k & 1], pq);
        dig += ((size_t)z * d.nd * d.ext << d.log_n) + at;
        const uint64_t *key = rlk + ((size_t)prime << d.log_n) + col;
        for (uint32_t i = 0; i < d.nd; i++) {
            Pair v{d2[0], d2[1]};
            if (i != own) v = ld2(dig + ((size_t)i * d.ext << d.log_n));
            const Pair k0 = ld2(key + ((size_t)(2 * i) * d.key_rows << d.log_n));
            const Pair k1 = ld2(key + ((size_t)(2 * i + 1) * d.key_rows << d.log_n));
            mac(t[0][0], v.x, k0.x);
            mac(t[0][1], v.y, k0.y);
            mac(t[1][0], v.x, k1.x);
            mac(t[1][1], v.y, k1.y);
            if ((i & 7u) == 7u)   // eight products and what is left of those before, below 2^128
#pragma unroll
                for (int k = 0; k < 4; k++) t[k >> 1][k & 1] = acc128{reduce128(t[k >> 1][k & 1], m), 0};
        }
#pragma unroll
        for (int k = 0; k < 4; k++) r[k >> 1][k & 1] = reduce128(t[k >> 1][k & 1], m);
    }
#pragma unroll
    for (int k = 0; k < 2; k++)
        *(Pair *)(u + (((size_t)(z * 2 + k) * d.ext + row) << d.log_n) + col) = Pair{r[k][0], r[k][1]};
}

struct Squares {
    const uint64_t *a[kStepBatch];
    uint32_t n, limbs;
};
// d (+)= sum_j (a0^2, 2 a0 a1, a1^2), two positions a thread.  F64 (primes below 2^50): four ciphertexts' products under
// one quotient, their loads issued together: 16 ciphertexts of 24 limbs at N = 2^16 94 us, 4.7 TB/s (in exact products 124).
template <bool F64>
__global__ __launch_bounds__(kThreads) void k_step_squares(Squares sq, uint64_t *d, bool accumulate, uint32_t L,
                                                           uint32_t log_n, const ModQ *__restrict__ mods)
{
    const uint32_t row = blockIdx.y, col = 2 * (blockIdx.x * kThreads + threadIdx.x);
    if (col >> log_n) return;
    const ModQ m = mods[row];
    const size_t at = ((size_t)row << log_n) + col, half = (size_t)L << log_n, next = (size_t)sq.limbs << log_n;
    Pair r[3] = {};
    if (accumulate)
#pragma unroll
        for (int k = 0; k < 3; k++) r[k] = ld2(d + k * half + at);
    if constexpr (F64) {
        const A ar(m);
        double t[3][2];
#pragma unroll
        for (int k = 0; k < 3; k++) {
            t[k][0] = A::from_u64(r[k].x);
            t[k][1] = A::from_u64(r[k].y);
        }
        for (uint32_t j0 = 0; j0 < sq.n; j0 += 4) {
            Pair a0[4], a1[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint64_t *p = sq.a[min(j0 + j, sq.n - 1)] + at;
                a0[j] = ld2(p);
                a1[j] = ld2(p + next);
            }
            ProductSum s[3][2];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (j0 + j >= sq.n) break;
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const double x = A::from_u64(e ? a0[j].y : a0[j].x), y = A::from_u64(e ? a1[j].y : a1[j].x);
                    s[0][e].add(x, x);
                    s[1][e].add(x, y);
                    s[2][e].add(y, y);
                }
            }
#pragma unroll
            for (int e = 0; e < 2; e++) {
                t[0][e] = ar.red(t[0][e] + s[0][e].value(ar));
                t[1][e] = ar.red(t[1][e] + 2.0 * s[1][e].value(ar));
                t[2][e] = ar.red(t[2][e] + s[2][e].value(ar));
            }
        }
#pragma unroll
        for (int k = 0; k < 3; k++) r[k] = Pair{ar.to_canon(t[k][0]), ar.to_canon(t[k][1])};
    } else {
        for (uint32_t j = 0; j < sq.n; j++) {
            const Pair a0 = ld2(sq.a[j] + at), a1 = ld2(sq.a[j] + at + next);
            r[0].x = addmod(r[0].x, mulmod(a0.x, a0.x, m), m.q);
            r[0].y = addmod(r[0].y, mulmod(a0.y, a0.y, m), m.q);
            r[1].x = addmod(r[1].x, mulmod(csub(2 * a0.x, m.q), a1.x, m), m.q);
            r[1].y = addmod(r[1].y, mulmod(csub(2 * a0.y, m.q), a1.y, m), m.q);
            r[2].x = addmod(r[2].x, mulmod(a1.x, a1.x, m), m.q);
            r[2].y = addmod(r[2].y, mulmod(a1.y, a1.y, m), m.q);
        }
    }
#pragma unroll
    for (int k = 0; k < 3; k++) *(Pair *)(d + k * half + at) = r[k];
}

Operands operands(const Step &s)
{
    Operands o{};
    const uint32_t kind = s.d ? kGiven : !s.a ? kNone : s.b_polys == 2 ? kProduct : kPlain;
    o.a = s.d ? s.d : s.a;
    o.b = s.b;
    o.out = s.out;
    o.info = s.n_terms | kind << 8 | s.a_limbs << 16 | s.b_limbs << 24;
    o.mult = s.mult;
    for (uint32_t i = 0; i < s.n_terms; i++) {
        o.z[i] = s.t[i].z;
        o.k[i] = s.t[i].k.m;
        o.term[i] = s.t[i].k.sh | s.t[i].limbs << 8 | s.t[i].polys << 16;
    }
    o.k[kStepTerms] = s.c.m;
    o.term[kStepTerms] = s.c.sh;
    return o;
}

// rows (of N words) of a batch of n steps, region by region: the digits, d2 for the ModUp, u, the converted rows.  One
// figure for both arithmetics: a workspace of it serves after ckks_ctx_set_ntt_arith as well.  The fp64 kernels take no
// more: of u they write the rows q_l and P alone.
struct Rows {
    size_t dig, stage, u, x, total;
};
Rows rows_of(const ckks_ctx *ctx, uint32_t L, size_t n, bool switched)
{
    const size_t ext = L + (switched ? ctx->n_p : 0);
    Rows r{};
    if (switched) {
        r.dig = n_digits(ctx, L - 1) * ext * n;
        r.stage = L * n;
    }
    r.u = 2 * ext * n;
    r.x = 2 * (L - 1) * n;
    r.total = r.dig + r.stage + r.u + r.x;
    return r;
}

// n steps that all switch a key, or none of them does, in any ring and primes (wsum_exact.hip divides)
ckks_status run_exact(ckks_ctx *ctx, uint32_t L, const Batch &b, uint32_t n, bool switched, const uint64_t *rlk,
                      uint64_t *mem)
{
    const size_t N = ctx->n;
    Dims d = wsum_dims(ctx, L);
    const Rows r = rows_of(ctx, L, n, switched);
    uint64_t *dig = mem, *stage = dig + r.dig * N, *u = stage + r.stage * N, *x = u + r.u * N;
    const uint32_t per_row = (ctx->n + 2 * kThreads - 1) / (2 * kThreads);
    Args a{};
    a.kind[0].rotated = switched;
    double words = 0;
    for (uint32_t i = 0; i < n; i++) {
        a.ct[i].out[0] = b.s[i].out;
        words += 2.0 * b.s[i].n() + (b.s[i].kind() == kProduct ? 4 : b.s[i].kind() ? 3 : 0);
    }
    if (switched) {
        prof_begin(ctx, K_ELEM, 24.0 * L * N * n);
        hipLaunchKernelGGL(k_step_d2, dim3(per_row, L, n), dim3(kThreads), 0, ctx->stream, b, stage, L, ctx->log_n, ctx->d_mod);
        prof_end(ctx, K_ELEM);
        HIP_TRY(hipGetLastError());
        CK_TRY(ks_modup_staged(ctx, stage, n, L - 1, dig));
    } else {
        d.K = 0;
        d.ext = L;
    }
    prof_begin(ctx, K_KEYIP, 8.0 * N * (words * L + n * d.ext * (switched ? d.nd + 2.0 : 2.0)));
    hipLaunchKernelGGL(k_step_u, dim3((d.ext * per_row + 7) / 8 * 8 * n), dim3(kThreads), 0, ctx->stream, b, dig, rlk, u, d, n,
                       per_row, ctx->d_pmodq, ctx->d_mod);
    prof_end(ctx, K_KEYIP);
    HIP_TRY(hipGetLastError());
    return wsum_exact_divide(ctx, a, n, 1, d, switched, u, x);
}

}  // namespace

PolyProd step_sources(const ckks_ctx *ctx, uint32_t L, const Batch &b, uint32_t n_sw)
{
    static_assert(kStepBatch <= (uint32_t)kPolyList && kStepBatch <= kWsumCts, "a batch fits the lists");
    PolyProd src{};
    for (uint32_t i = 0; i < n_sw; i++) {
        const Operands &s = b.s[i];
        src.list[i] = s.a + (s.kind() == kGiven ? 2 * (size_t)L : s.a_limbs()) * ctx->n;
        src.mul[i] = s.kind() == kGiven ? nullptr : s.b + (size_t)s.b_limbs() * ctx->n;
        src.mult[i] = s.mult;
    }
    return src;
}

bool step_int(double x, StepInt *out)
{
    if (!std::isfinite(x) || std::fabs(x) >= 0x1p120) return false;
    int e = 0;
    double r = std::nearbyint(x);
    if (std::fabs(r) >= 0x1p62) {   // an integer of 53 bits and a power of two
        r = std::frexp(r, &e) * 0x1p53;
        e -= 53;
    }
    *out = StepInt{(int64_t)r, (uint32_t)e};
    return true;
}

size_t step_scratch_words(const ckks_ctx *ctx, uint32_t L, uint32_t steps, bool switched)
{
    return rows_of(ctx, L, std::min(steps, kStepBatch), switched).total * ctx->n;
}

ckks_status step_run(ckks_ctx *ctx, uint32_t L, const std::vector<Step> &steps, const uint64_t *rlk, uint64_t *mem)
{
    // those that switch a key first; the fp64 kernels take both kinds in one batch
    std::vector<const Step *> list;
    size_t n_sw = 0;
    for (int sw = 1; sw >= 0; sw--) {
        for (const Step &s : steps) {
            CK_REQUIRE(!s.a || s.b_polys == 2 || s.mult == 1, CKKS_EINVAL, "a step's product with a plaintext times %d", s.mult);
            CK_REQUIRE(s.n_terms <= kStepTerms, CKKS_EINVAL, "a step of %u terms, at most %u", s.n_terms, kStepTerms);
            if (s.switched() == (sw != 0)) list.push_back(&s);
        }
        if (sw) n_sw = list.size();
    }
    const bool fast = f64_switch(ctx, L - 1);
    for (size_t at = 0; at < list.size();) {
        const size_t sw = at < n_sw ? n_sw - at : 0;
        const uint32_t n = (uint32_t)std::min<size_t>({kStepBatch, list.size() - at, !fast && sw ? sw : kStepBatch});
        Batch b{};
        for (uint32_t i = 0; i < n; i++) b.s[i] = operands(*list[at + i]);
        if (fast) CK_TRY((blk_switch(ctx, L - 1) ? step_blk : step_f64)(ctx, L, b, n, (uint32_t)std::min<size_t>(sw, n), rlk, mem));
        else CK_TRY(run_exact(ctx, L, b, n, sw != 0, rlk, mem));
        at += n;
    }
    return CKKS_OK;
}

ckks_status step_squares(ckks_ctx *ctx, uint32_t L, const std::vector<const uint64_t *> &a, uint32_t limbs, uint64_t *d)
{
    for (size_t j0 = 0; j0 < a.size(); j0 += kStepBatch) {
        Squares sq{};
        sq.n = (uint32_t)std::min<size_t>(kStepBatch, a.size() - j0);
        sq.limbs = limbs;
        for (uint32_t j = 0; j < sq.n; j++) sq.a[j] = a[j0 + j];
        prof_begin(ctx, K_ELEM, 8.0 * L * ctx->n * (2.0 * sq.n + (j0 ? 6 : 3)));
        const dim3 grid((ctx->n + 2 * kThreads - 1) / (2 * kThreads), L);
        if (ntt_uses_f64(ctx, L))
            hipLaunchKernelGGL(k_step_squares<true>, grid, dim3(kThreads), 0, ctx->stream, sq, d, j0 > 0, L, ctx->log_n,
                               ctx->d_mod);
        else
            hipLaunchKernelGGL(k_step_squares<false>, grid, dim3(kThreads), 0, ctx->stream, sq, d, j0 > 0, L, ctx->log_n,
                               ctx->d_mod);
        prof_end(ctx, K_ELEM);
        HIP_TRY(hipGetLastError());
    }
    return CKKS_OK;
}

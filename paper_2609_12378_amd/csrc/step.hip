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

// d of every step ([dp][L][N] each, dp 3 where the steps switch a key, else 2), one position a thread.  The constant goes
// in as c q_l: it vanishes modulo q_l and the rescale leaves c.  At most 11 products below 2^124 a sum.
__global__ __launch_bounds__(kThreads) void k_step_lin(Batch bt, uint64_t *d, uint32_t dp, uint32_t L, uint32_t log_n,
                                                       const ModQ *__restrict__ mods)
{
    __shared__ uint64_t ks[kStepTerms + 1];
    const Operands &s = bt.s[blockIdx.z];
    const uint32_t row = blockIdx.y, pos = blockIdx.x * kThreads + threadIdx.x;
    const ModQ m = mods[row];
    if (threadIdx.x <= s.n) {
        const uint32_t i = threadIdx.x < s.n ? threadIdx.x : kStepTerms;
        const uint64_t r = int_mod(s.k[i], s.sh[i], m.q);
        ks[threadIdx.x] = i < kStepTerms ? r : mulmod(r, mods[L - 1].q % m.q, m);
    }
    __syncthreads();
    if (pos >> log_n) return;
    const size_t at = ((size_t)row << log_n) + pos, half = (size_t)L << log_n;
    acc128 x0{ks[s.n], 0}, x1{0, 0};
    d += (size_t)blockIdx.z * dp * half;
    if (s.kind == kProduct || s.kind == kPlain) {
        const uint64_t *a = s.a + at, *b = s.b + at;
        const uint64_t a0 = a[0], a1 = a[(size_t)s.a_limbs << log_n];
        auto scaled = [&](uint64_t v) { return s.mult == 2 ? csub(2 * v, m.q) : s.mult < 0 && v ? m.q - v : v; };
        const uint64_t b0 = scaled(b[0]);
        mac(x0, a0, b0);
        mac(x1, a1, b0);
        if (s.kind == kProduct) {
            const uint64_t b1 = scaled(b[(size_t)s.b_limbs << log_n]);
            mac(x1, a0, b1);
            d[2 * half + at] = mulmod(a1, b1, m);
        }
    } else if (s.kind == kGiven) {
        mac(x0, s.a[at], 1);
        mac(x1, s.a[half + at], 1);
        d[2 * half + at] = s.a[2 * half + at];
    }
    for (uint32_t i = 0; i < s.n; i++) {
        mac(x0, s.z[i][at], ks[i]);
        if (s.polys[i] == 2) mac(x1, s.z[i][at + ((size_t)s.limbs[i] << log_n)], ks[i]);
    }
    d[at] = reduce128(x0, m);
    d[half + at] = reduce128(x1, m);
}

struct Squares {
    const uint64_t *a[kStepBatch];
    uint32_t n, limbs;
};
// d (+)= sum_j (a0^2, 2 a0 a1, a1^2)
__global__ __launch_bounds__(kThreads) void k_step_squares(Squares sq, uint64_t *d, bool accumulate, uint32_t L,
                                                           uint32_t log_n, const ModQ *__restrict__ mods)
{
    const uint32_t row = blockIdx.y, pos = blockIdx.x * kThreads + threadIdx.x;
    if (pos >> log_n) return;
    const ModQ m = mods[row];
    const size_t at = ((size_t)row << log_n) + pos, half = (size_t)L << log_n;
    uint64_t s0 = 0, s1 = 0, s2 = 0;
    if (accumulate) s0 = d[at], s1 = d[half + at], s2 = d[2 * half + at];
    for (uint32_t j = 0; j < sq.n; j++) {
        const uint64_t a0 = sq.a[j][at], a1 = sq.a[j][at + ((size_t)sq.limbs << log_n)];
        s0 = addmod(s0, mulmod(a0, a0, m), m.q);
        s1 = addmod(s1, mulmod(csub(2 * a0, m.q), a1, m), m.q);
        s2 = addmod(s2, mulmod(a1, a1, m), m.q);
    }
    d[at] = s0;
    d[half + at] = s1;
    d[2 * half + at] = s2;
}

dim3 grid_of(const ckks_ctx *ctx, uint32_t rows, uint32_t z) { return dim3((ctx->n + kThreads - 1) / kThreads, rows, z); }

Operands operands(const Step &s)
{
    Operands o{};
    o.kind = s.d ? kGiven : !s.a ? kNone : s.b_polys == 2 ? kProduct : kPlain;
    o.a = s.d ? s.d : s.a;
    o.b = s.b;
    o.out = s.out;
    o.a_limbs = (uint8_t)s.a_limbs;
    o.b_limbs = (uint8_t)s.b_limbs;
    o.mult = (int8_t)s.mult;
    o.n = (uint8_t)s.n_terms;
    for (uint32_t i = 0; i < s.n_terms; i++) {
        o.z[i] = s.t[i].z;
        o.k[i] = s.t[i].k.m;
        o.sh[i] = (uint8_t)s.t[i].k.sh;
        o.limbs[i] = (uint8_t)s.t[i].limbs;
        o.polys[i] = (uint8_t)s.t[i].polys;
    }
    o.k[kStepTerms] = s.c.m;
    o.sh[kStepTerms] = (uint8_t)s.c.sh;
    return o;
}

// rows (of N words) of a batch of n steps, region by region
struct Rows {
    size_t d, dig, stage, work, sum, top, total;
};
Rows rows_of(const ckks_ctx *ctx, uint32_t L, size_t n, bool switched)
{
    const size_t ext = L + ctx->n_p, nd = n_digits(ctx, L - 1);
    Rows r{};
    r.d = (switched ? 3 : 2) * L * n;
    r.top = 2 * L * n;
    if (switched) {
        r.dig = nd * ext * n;
        r.stage = std::max(L, ctx->alpha) * n;
        r.work = (2 * ext + 2 * L) * n;
        r.sum = 2 * L * n;
    }
    r.total = r.d + r.dig + r.stage + r.work + r.sum + r.top;
    return r;
}

// n steps that all switch a key, or none of them does, in any ring and arithmetic: d, ModUp, ModDown, rescale
ckks_status run_batch(ckks_ctx *ctx, uint32_t L, const Batch &b, uint32_t n, bool switched, const uint64_t *rlk,
                      uint64_t *mem)
{
    const size_t N = ctx->n;
    const uint32_t ext = L + ctx->n_p, nd = n_digits(ctx, L - 1), dp = switched ? 3 : 2;
    const Rows r = rows_of(ctx, L, n, switched);
    uint64_t *d = mem, *dig = d + r.d * N, *work = dig + (r.dig + r.stage) * N, *sum = work + r.work * N,
             *top = sum + r.sum * N;
    double words = 0;
    for (uint32_t i = 0; i < n; i++) words += dp + 2.0 * b.s[i].n + (b.s[i].kind == kProduct ? 4 : b.s[i].kind ? 3 : 0);
    prof_begin(ctx, K_ELEM, 8.0 * words * L * N);
    hipLaunchKernelGGL(k_step_lin, grid_of(ctx, L, n), dim3(kThreads), 0, ctx->stream, b, d, dp, L, ctx->log_n, ctx->d_mod);
    prof_end(ctx, K_ELEM);
    HIP_TRY(hipGetLastError());
    std::vector<uint64_t *> outs(n);
    for (uint32_t i = 0; i < n; i++) outs[i] = b.s[i].out;
    if (!switched) return rescale_each(ctx, d, n, L - 1, outs.data(), top);
    // a relinearisation is a rotation by the identity: (d0 + u0, d1 + u1), u the key switch of d2
    std::vector<const uint64_t *> c0(n), add1(n), digs(n), keys(n, rlk);
    std::vector<uint32_t> g(n, 1);
    std::vector<uint64_t *> sums(n);
    for (uint32_t i = 0; i < n; i++) {
        c0[i] = d + (size_t)i * 3 * L * N;
        add1[i] = c0[i] + L * N;
        digs[i] = dig + (size_t)i * nd * ext * N;
        sums[i] = sum + (size_t)i * 2 * L * N;
    }
    CK_TRY(ks_modup_batch(ctx, d + 2 * (size_t)L * N, 3 * (size_t)L * N, n, L - 1, dig, r.stage));
    CK_TRY(ks_rotate_batch(ctx, L - 1, n, c0.data(), digs.data(), g.data(), keys.data(), sums.data(), work, nullptr,
                           add1.data()));
    return rescale_each(ctx, sum, n, L - 1, outs.data(), top);
}

}  // namespace

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
    const uint32_t n = std::min(steps, kStepBatch);
    // one figure for both arithmetics: a workspace of it serves after ckks_ctx_set_ntt_arith as well
    return std::max(rows_of(ctx, L, n, switched).total, step_f64_rows(ctx, L, n, switched)) * ctx->n;
}

ckks_status step_run(ckks_ctx *ctx, uint32_t L, const std::vector<Step> &steps, const uint64_t *rlk, uint64_t *mem)
{
    // those that switch a key first; the fp64 kernels take both kinds in one batch
    std::vector<const Step *> list;
    size_t n_sw = 0;
    for (int sw = 1; sw >= 0; sw--) {
        for (const Step &s : steps)
            if (s.switched() == (sw != 0)) list.push_back(&s);
        if (sw) n_sw = list.size();
    }
    const bool fast = step_f64_ok(ctx, L);
    for (size_t at = 0; at < list.size();) {
        const size_t sw = at < n_sw ? n_sw - at : 0;
        const uint32_t n = (uint32_t)std::min<size_t>({kStepBatch, list.size() - at, !fast && sw ? sw : kStepBatch});
        Batch b{};
        for (uint32_t i = 0; i < n; i++) b.s[i] = operands(*list[at + i]);
        if (fast) CK_TRY(step_f64(ctx, L, b, n, (uint32_t)std::min<size_t>(sw, n), rlk, mem));
        else CK_TRY(run_batch(ctx, L, b, n, sw != 0, rlk, mem));
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
        hipLaunchKernelGGL(k_step_squares, grid_of(ctx, L, 1), dim3(kThreads), 0, ctx->stream, sq, d, j0 > 0, L, ctx->log_n,
                           ctx->d_mod);
        prof_end(ctx, K_ELEM);
        HIP_TRY(hipGetLastError());
    }
    return CKKS_OK;
}

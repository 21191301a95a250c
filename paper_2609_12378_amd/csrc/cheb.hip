// Sums of Chebyshev polynomials of ciphertexts, in the fewest levels: a sum of degree below 2^D takes D below T_1's.
//
// T_i = 2 T_(i - i/2) T_(i/2) - T_(i mod 2) is there ceil(log2 i) levels below T_1.  A sum of degree d that has to be there
// at depth D is one step of the terms k_i T_i where all T_i are there in time and among the first 2^b - 1; else, with
// m = 2^s the largest power of two up to d, c = q T_m + r (T_m T_i = (T_(m+i) + T_(m-i)) / 2): one product of q, at
// depth D - 1, and T_m, and in the same step r's terms (m < 2^b + 1) or r itself, at depth D - 1.  q's degree is below
// 2^(D-1), so no level is lost.  b = D - 2 in [1, 3]: near the fewest products for every degree (5 for 7, 9 for 15, 15
// for 31, 24 for 63).  Everything of one depth, for all ciphertexts, is one call of step_run.
#include <algorithm>
#include <cmath>
#include <map>

#include "step.h"

namespace {

uint32_t ceil_log2(uint32_t i)
{
    uint32_t d = 0;
    while ((1u << d) < i) d++;
    return d;
}

struct Builder {
    const ckks_ctx *ctx;
    ChebPlan &plan;
    double s1;
    uint32_t b;
    bool ok = true;
    std::map<uint32_t, uint32_t> powers;   // i -> object

    // prime that the step to `depth` divides by
    uint64_t prime(uint32_t depth) const { return ctx->primes[plan.L1 - depth]; }
    StepInt integer(double x)
    {
        StepInt v;
        ok = step_int(x, &v) && ok;
        return v;
    }

    uint32_t power(uint32_t i)
    {
        const auto it = powers.find(i);
        if (it != powers.end()) return it->second;
        const uint32_t x = power(i - i / 2), y = power(i / 2);
        ChebObj o;
        o.depth = ceil_log2(i);
        o.x = (int)x;
        o.y = (int)y;
        o.mult = 2;
        const double sx = plan.obj[x].scale, sy = plan.obj[y].scale;
        o.scale = sx * sy / (double)prime(o.depth);
        if (i % 2) o.t.push_back({0, integer(-(sx * sy / s1))});
        else o.c = integer(-o.scale);
        plan.obj.push_back(o);
        return powers[i] = (uint32_t)plan.obj.size() - 1;
    }

    ChebTerm term(uint32_t i, double c, double up)
    {
        const uint32_t o = power(i);
        return {o, integer(c * (up / plan.obj[o].scale))};
    }

    uint32_t node(const std::vector<double> &c, uint32_t depth, double target)
    {
        ChebObj o;
        o.depth = depth;
        o.scale = target;
        const double up = target * (double)prime(depth);
        const uint32_t d = (uint32_t)c.size() - 1;
        if (d < (1u << b) && ceil_log2(d) <= depth - 1) {
            for (uint32_t i = 1; i <= d; i++) o.t.push_back(term(i, c[i], up));
            o.c = integer(c[0] * target);
        } else {
            uint32_t m = 1;
            while (2 * m <= d) m *= 2;
            std::vector<double> q(c.begin() + m, c.end()), r(c.begin(), c.begin() + m);
            for (uint32_t i = 1; i < q.size(); i++) {
                q[i] *= 2;
                r[m - i] -= c[m + i];
            }
            if (q.size() == 1) {
                o.t.push_back(term(m, q[0], up));
            } else {
                o.y = (int)power(m);
                o.x = (int)node(q, depth - 1, up / plan.obj[o.y].scale);
            }
            if (m <= 1u << b) {
                for (uint32_t i = 1; i < m; i++) o.t.push_back(term(i, r[i], up));
                o.c = integer(r[0] * target);
            } else {
                o.t.push_back({node(r, depth - 1, target), StepInt{(int64_t)prime(depth), 0}});
            }
        }
        plan.obj.push_back(o);
        return (uint32_t)plan.obj.size() - 1;
    }
};

}  // namespace

ckks_status cheb_plan(const ckks_ctx *ctx, const double *coefs, uint32_t degree, uint32_t L1, double s1, double target,
                      const char *what, ChebPlan *out)
{
    out->L1 = L1;
    out->depth = cheb_depth(degree);
    out->obj.assign(1, ChebObj{});
    out->obj[0].depth = 0;
    out->obj[0].scale = s1;
    Builder bd{ctx, *out, s1, std::max(1u, std::min(3u, out->depth < 2 ? 0u : out->depth - 2))};
    bd.powers[1] = 0;
    std::vector<double> c(degree + 1, 0.0);
    if (coefs) c.assign(coefs, coefs + degree + 1);
    bd.node(c, out->depth, target);
    CK_REQUIRE(bd.ok || !coefs, CKKS_ESCALE, "%s: a coefficient times its scale is 2^120 or more (output scale %g)", what,
               target);
    return CKKS_OK;
}

size_t cheb_scratch_words(const ckks_ctx *ctx, const ChebPlan &plan, uint32_t cts)
{
    const uint32_t G = std::min(cts, kStepBatch);
    size_t rows = 0;
    for (size_t i = 1; i + 1 < plan.obj.size(); i++) rows += 2 * (size_t)(plan.L1 - plan.obj[i].depth);
    // the first steps have the most limbs, but not always the most steps
    size_t step = 0;
    for (uint32_t d = 1; d <= plan.depth; d++) {
        uint32_t n = 0;
        for (const ChebObj &o : plan.obj) n += o.depth == d;
        step = std::max(step, step_scratch_words(ctx, plan.L1 + 1 - d, n * G));
    }
    return G * rows * ctx->n + step;
}

ckks_status cheb_run(ckks_ctx *ctx, const ChebPlan &plan, const std::vector<const uint64_t *> &t1,
                     const std::vector<uint64_t *> &out, const std::vector<StepTerm> &extra, const uint64_t *rlk,
                     uint64_t *mem)
{
    const size_t N = ctx->n, last = plan.obj.size() - 1;
    for (size_t r0 = 0; r0 < t1.size(); r0 += kStepBatch) {
        const uint32_t G = (uint32_t)std::min<size_t>(kStepBatch, t1.size() - r0);
        std::vector<uint64_t *> base(plan.obj.size(), nullptr);
        uint64_t *at = mem;
        for (size_t i = 1; i < last; i++) {
            base[i] = at;
            at += (size_t)G * 2 * (plan.L1 - plan.obj[i].depth) * N;
        }
        auto limbs = [&](size_t i) { return plan.L1 - plan.obj[i].depth; };
        auto of = [&](size_t i, uint32_t r) -> const uint64_t * {
            return i ? base[i] + (size_t)r * 2 * limbs(i) * N : t1[r0 + r];
        };
        for (uint32_t d = 1; d <= plan.depth; d++) {
            std::vector<Step> steps;
            for (size_t i = 1; i <= last; i++) {
                const ChebObj &o = plan.obj[i];
                if (o.depth != d) continue;
                for (uint32_t r = 0; r < G; r++) {
                    Step s;
                    if (o.x >= 0) s.product(of(o.x, r), limbs(o.x), of(o.y, r), limbs(o.y), o.mult);
                    for (const ChebTerm &t : o.t) s.term(of(t.of, r), limbs(t.of), t.k);
                    if (i == last && !extra.empty()) s.term(extra[r0 + r]);
                    s.c = o.c;
                    s.out = i == last ? out[r0 + r] : base[i] + (size_t)r * 2 * limbs(i) * N;
                    steps.push_back(s);
                }
            }
            CK_TRY(step_run(ctx, plan.L1 + 1 - d, steps, rlk, at));
        }
    }
    return CKKS_OK;
}

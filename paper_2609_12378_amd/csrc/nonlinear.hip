// Polynomials of ciphertexts and root-mean-square norms: the calls, from steps (step.hip), sums of Chebyshev polynomials
// (cheb.hip) and lazily divided sums of rotations.
#include <cmath>

#include "api_args.h"
#include "nonlinear.h"
#include "ops.h"

ckks_status check_poly(const ckks_poly *p, const char *what)
{
    CK_REQUIRE(p && p->coefs, CKKS_EINVAL, "%s: null polynomial", what);
    CK_REQUIRE(p->degree >= 1 && p->degree <= kChebDegree, CKKS_EINVAL, "%s: degree %u outside [1, %u]", what, p->degree,
               kChebDegree);
    CK_REQUIRE(std::isfinite(p->lo) && std::isfinite(p->hi) && p->lo < p->hi && std::isfinite(p->hi - p->lo), CKKS_EINVAL,
               "%s: the interval [%g, %g] is empty or not finite", what, p->lo, p->hi);
    for (uint32_t i = 0; i <= p->degree; i++)
        CK_REQUIRE(std::isfinite(p->coefs[i]), CKKS_EINVAL, "%s: coefficient %u is not finite", what, i);
    return CKKS_OK;
}

ckks_status scaled_int(double x, StepInt *out, const char *what, const char *name)
{
    CK_REQUIRE(step_int(x, out), CKKS_ESCALE, "%s: %s becomes the factor %g, which is not below 2^120", what, name, x);
    return CKKS_OK;
}

ckks_status check_scale(double s, const char *what, const char *name)
{
    CK_REQUIRE(s > 0 && std::isfinite(s), CKKS_ESCALE, "%s: the %s's scale must be positive", what, name);
    return CKKS_OK;
}

ckks_status check_list(const ckks_ctx *ctx, const ckks_buf *b, uint32_t n, uint32_t polys, uint32_t least,
                       const char *what, const char *name)
{
    for (uint32_t i = 0; i < n; i++) {
        CK_REQUIRE(b[i].data && b[i].n_polys == polys, CKKS_EINVAL, "%s: %s %u is not a %s", what, name, i,
                   polys == 2 ? "ciphertext" : "plaintext");
        CK_REQUIRE(b[i].n_limbs >= least && b[i].n_limbs <= ctx->n_q, CKKS_ELEVEL, "%s: %s %u has %u limbs, needs %u to %u",
                   what, name, i, b[i].n_limbs, least, ctx->n_q);
    }
    CK_TRY(check_scales(b, n, what, name));
    return check_scale(b[0].scale, what, name);
}

ckks_status poly_map(const ckks_poly &p, double s1, double *by, StepInt *c, const char *what)
{
    *by = 2.0 / (p.hi - p.lo) * s1;
    return scaled_int(-(p.lo + p.hi) / (p.hi - p.lo) * s1, c, what, "the interval's middle");
}

namespace {

double prime_of(const ckks_ctx *ctx, uint32_t limbs) { return (double)ctx->primes[limbs - 1]; }

// Regions of a workspace one after another: with base null only counted.
struct Bump {
    uint64_t *base;
    size_t at = 0;
    uint64_t *take(size_t words)
    {
        uint64_t *p = base ? base + at : nullptr;
        at += words;
        return p;
    }
};

struct PolyMem {
    uint64_t *t1, *work;
};
size_t poly_mem(const ckks_ctx *ctx, uint32_t L, uint32_t count, const ChebPlan &plan, uint64_t *base, PolyMem *m)
{
    Bump b{base};
    m->t1 = b.take((size_t)count * 2 * (L - 1) * ctx->n);
    m->work = b.take(std::max(step_scratch_words(ctx, L, count, false), cheb_scratch_words(ctx, plan, count)));
    return b.at;
}

// Radixes of the rounds of a sum over 2^bits positions: at most 16, as even as they go.  A round of radix R reads R - 1
// keys for one ModUp and one ModDown.  Measured on both sides, us a norm with rounds of up to 16, 8 and 4: fewer rounds win
// wherever launches count (N = 2^12, one ciphertext 246, 275, 306; 2^13 590, 631, 680; 2^14 616, 656, 710, token-major 810,
// 889, 990; 2^15 787, 797, 842; 2^16 of 6 limbs 496, 527, 583), fewer keys at N = 2^16 from about 12 limbs on (13 limbs
// 1199, 1171, 1207; 24 limbs 2164, 2026, 2047; 16 ciphertexts of 24 limbs 3378, 3235, 3269).  One rule for all, since the
// radixes say which keys a program makes: it costs those 2 to 7%, and 13 keys more for 256 positions.
std::vector<uint32_t> sum_radixes(uint32_t count)
{
    uint32_t bits = 0;
    while ((1u << bits) < count) bits++;
    std::vector<uint32_t> r;
    for (uint32_t left = (bits + 3) / 4; left; left--) {
        const uint32_t b = (bits + left - 1) / left;
        r.push_back(1u << b);
        bits -= b;
    }
    return r;
}

// The steps of a round and their keys
struct Round {
    std::vector<uint32_t> g;
    std::vector<const uint64_t *> key;
};
ckks_status sum_rounds(const ckks_ctx *ctx, uint32_t count, int64_t stride, const int32_t *key_steps,
                       const uint64_t *const *keys, uint32_t n_keys, std::vector<Round> *out)
{
    const int64_t slots = ctx->n / 2;
    for (uint32_t radix : sum_radixes(count)) {
        Round r;
        for (uint32_t k = 1; k < radix; k++) {
            const int64_t st = ((k * stride) % slots + slots) % slots;
            const uint64_t *key = nullptr;
            bool exact = false;   // a key given for the step itself is taken before one for an equal rotation
            for (uint32_t i = 0; i < n_keys && !exact; i++) {
                exact = keys[i] && key_steps[i] == k * stride;
                if (exact || (!key && ((int64_t)key_steps[i] % slots + slots) % slots == st)) key = keys[i];
            }
            CK_REQUIRE(key, CKKS_ENOKEY, "rms_norm: no key for step %lld (modulo %lld)", (long long)st, (long long)slots);
            r.g.push_back(ckks_galois_elt(ctx, (int32_t)st));
            r.key.push_back(key);
        }
        out->push_back(r);
        stride *= radix;
    }
    return CKKS_OK;
}

// words of a round at L limbs: digits and their staging rows, u, the ModDown's rows
size_t round_words(const ckks_ctx *ctx, uint32_t L)
{
    const size_t ext = L + ctx->n_p, nd = n_digits(ctx, L - 1);
    return (nd * ext + std::max(L, ctx->alpha) + 2 * ext + 2 * L) * ctx->n;
}
// v = v + sum of its rotations, round by round, each with one ModUp and one ModDown; a, b: [2][L][N], the result in *v
ckks_status run_rounds(ckks_ctx *ctx, uint32_t L, const std::vector<Round> &rounds, uint64_t **v, uint64_t *other,
                       uint64_t *mem)
{
    const size_t N = ctx->n, ext = L + ctx->n_p, nd = n_digits(ctx, L - 1);
    uint64_t *dig = mem, *u = dig + (nd * ext + std::max(L, ctx->alpha)) * N, *work = u + 2 * ext * N;
    for (const Round &r : rounds) {
        const uint32_t n = (uint32_t)r.g.size();
        const std::vector<const uint64_t *> c0(n, *v), digs(n, dig);
        CK_TRY(ks_modup(ctx, *v + (size_t)L * N, L - 1, dig, std::max(L, ctx->alpha)));
        CK_TRY(ks_ip_accumulate(ctx, L - 1, n, c0.data(), digs.data(), r.g.data(), r.key.data(), &u, 1, false));
        CK_TRY(ks_moddown(ctx, u, 2, L - 1, *v, 1, *v + (size_t)L * N, other, work));
        std::swap(*v, other);
    }
    return CKKS_OK;
}

// The limbs along a norm and its workspace
struct Norm {
    uint32_t L, Lv, depth, m0, m;   // inputs, mean, polynomial's levels, its value's limbs, the inverse root's
    ChebPlan plan;
    uint64_t *d, *v, *v2, *t1, *means, *y, *y2, *ab, *xw, *work;
};
bool norm_limbs(const ckks_ctx *ctx, uint32_t L, uint32_t tm, uint32_t degree, uint32_t newton, Norm *n)
{
    if (L > ctx->n_q || degree < 1 || degree > kChebDegree || newton > 4) return false;
    n->L = L;
    n->depth = cheb_depth(degree);
    if (L < 1 + tm + 1 + n->depth + 2 * newton + 2) return false;
    n->Lv = L - 1 - tm;
    n->m0 = n->Lv - 1 - n->depth;
    n->m = n->m0 - 2 * newton;
    return true;
}
size_t norm_mem(const ckks_ctx *ctx, uint32_t count, uint32_t newton, uint64_t *base, Norm *n)
{
    const size_t N = ctx->n, ct = 2 * (size_t)n->L * N;
    Bump b{base};
    n->d = b.take(3 * (size_t)n->L * N);
    n->v = b.take(ct);
    n->v2 = b.take(ct);
    n->t1 = b.take(ct);
    n->means = b.take(newton * ct);
    n->y = b.take(ct);
    n->y2 = b.take(ct);
    n->ab = b.take(2 * ct);
    n->xw = b.take((size_t)count * 2 * n->m * N);
    size_t w = std::max(step_scratch_words(ctx, n->L, 1), step_scratch_words(ctx, n->Lv, 1 + newton, false));
    w = std::max({w, round_words(ctx, n->L - 1), cheb_scratch_words(ctx, n->plan, 1), step_scratch_words(ctx, n->m0, 2),
                  step_scratch_words(ctx, n->m + 1, count + 1)});
    n->work = b.take(w);
    return b.at;
}

}  // namespace

size_t poly_workspace_bytes(const ckks_ctx *ctx, uint32_t L, uint32_t count, uint32_t degree)
{
    if (L > ctx->n_q || !ctx->n_p || !count || degree < 1 || degree > kChebDegree || L < 2 + cheb_depth(degree))
        return SIZE_MAX;
    ChebPlan plan;
    PolyMem m;
    (void)cheb_plan(ctx, nullptr, degree, L - 1, 1.0, 1.0, "poly_eval", &plan);
    return poly_mem(ctx, L, count, plan, nullptr, &m) * 8;
}

size_t norm_workspace_bytes(const ckks_ctx *ctx, uint32_t L, uint32_t count, uint32_t tokens, uint32_t layout,
                            uint32_t degree, uint32_t newton)
{
    Norm n;
    if (!ctx->n_p || !count || tokens < 1 || tokens > ctx->n / 2 || (tokens & (tokens - 1)) ||
        (layout != CKKS_TOKEN_MAJOR && layout != CKKS_FEATURE_MAJOR) ||
        !norm_limbs(ctx, L, layout == CKKS_TOKEN_MAJOR, degree, newton, &n))
        return SIZE_MAX;
    (void)cheb_plan(ctx, nullptr, degree, n.Lv - 1, 1.0, 1.0, "rms_norm", &n.plan);
    return norm_mem(ctx, count, newton, nullptr, &n) * 8;
}

extern "C" {

ckks_status ckks_poly_eval(ckks_ctx *ctx, const ckks_buf *in, uint32_t count, const ckks_poly *poly, const uint64_t *rlk,
                           ckks_buf *out)
{
    clear_error();
    const DeviceScope dev(ctx);
    return guarded("poly_eval", [&]() -> ckks_status {
        CK_REQUIRE(ctx, CKKS_EINVAL, "poly_eval: null context");
        CK_TRY(check_poly(poly, "poly_eval"));
        if (!count) return CKKS_OK;
        CK_REQUIRE(in && out && rlk, CKKS_EINVAL, "poly_eval: null argument");
        CK_REQUIRE(ctx->n_p > 0, CKKS_EUNSUPPORTED, "poly_eval: the context has no special primes");
        const uint32_t L = in[0].n_limbs, depth = cheb_depth(poly->degree);
        CK_REQUIRE(L >= depth + 2 && L <= ctx->n_q, CKKS_ELEVEL, "poly_eval: degree %u needs %u to %u limbs, %u given",
                   poly->degree, depth + 2, ctx->n_q, L);
        CK_TRY(check_cts(in, count, L, "poly_eval", "input"));
        CK_TRY(check_scales(in, count, "poly_eval", "input"));
        CK_TRY(check_scale(in[0].scale, "poly_eval", "input"));
        CK_TRY(check_cts(out, count, L - 1 - depth, "poly_eval", "output"));
        std::vector<Range> ins, outs;
        add_ranges(ins, ctx, in, count);
        add_ranges(outs, ctx, out, count);
        CK_TRY(check_overlap(outs, ins, "poly_eval"));
        const double S = in[0].scale, s1 = prime_of(ctx, L - 1);
        double by;
        StepInt k, c;
        CK_TRY(poly_map(*poly, s1, &by, &c, "poly_eval"));
        CK_TRY(scaled_int(by * (prime_of(ctx, L) / S), &k, "poly_eval", "the interval's width"));
        ChebPlan plan;
        CK_TRY(cheb_plan(ctx, poly->coefs, poly->degree, L - 1, s1, S, "poly_eval", &plan));
        const uint32_t shp[3] = {L, count, poly->degree};
        void *mem;
        CK_TRY(ctx_scratch(ctx, op_workspace_bytes(ctx, CKKS_OP_POLY_EVAL, shp), &mem));
        PolyMem m;
        (void)poly_mem(ctx, L, count, plan, (uint64_t *)mem, &m);
        std::vector<Step> map(count);
        std::vector<const uint64_t *> t1(count);
        std::vector<uint64_t *> to(count);
        for (uint32_t r = 0; r < count; r++) {
            map[r].term(in[r].data, L, k);
            map[r].c = c;
            t1[r] = map[r].out = m.t1 + (size_t)r * 2 * (L - 1) * ctx->n;
            to[r] = out[r].data;
        }
        CK_TRY(step_run(ctx, L, map, nullptr, m.work));
        CK_TRY(cheb_run(ctx, plan, t1, to, {}, rlk, m.work));
        for (uint32_t r = 0; r < count; r++) out[r].scale = S;
        return CKKS_OK;
    });
}

ckks_status ckks_rms_norm(ckks_ctx *ctx, const ckks_buf *in, uint32_t count, const ckks_norm_shape *shape,
                          const ckks_poly *inv_root, const ckks_buf *weights, const ckks_buf *mask,
                          const ckks_buf *residual, double residual_scale, const uint64_t *rlk, const int32_t *key_steps,
                          const uint64_t *const *keys, uint32_t n_keys, ckks_buf *out)
{
    clear_error();
    const DeviceScope dev(ctx);
    return guarded("rms_norm", [&]() -> ckks_status {
        const char *what = "rms_norm";
        CK_REQUIRE(ctx && shape, CKKS_EINVAL, "rms_norm: null argument");
        CK_TRY(check_poly(inv_root, what));
        const uint32_t T = shape->tokens, slots = ctx->n / 2;
        CK_REQUIRE(T >= 1 && T <= slots && (T & (T - 1)) == 0, CKKS_EINVAL,
                   "rms_norm: %u tokens are not a power of two in [1, %u]", T, slots);
        CK_REQUIRE(shape->layout == CKKS_TOKEN_MAJOR || shape->layout == CKKS_FEATURE_MAJOR, CKKS_EINVAL,
                   "rms_norm: unknown layout %u", shape->layout);
        CK_REQUIRE(shape->newton <= 4, CKKS_EINVAL, "rms_norm: %u Newton steps, at most 4", shape->newton);
        CK_REQUIRE(std::isfinite(shape->eps) && shape->eps >= 0, CKKS_EINVAL, "rms_norm: eps %g", shape->eps);
        CK_REQUIRE(!residual || std::isfinite(residual_scale), CKKS_EINVAL, "rms_norm: residual scale %g", residual_scale);
        if (!count) return CKKS_OK;
        const uint32_t D = slots / T;
        const bool tm = shape->layout == CKKS_TOKEN_MAJOR;
        CK_REQUIRE(in && out && rlk && (!n_keys || (key_steps && keys)), CKKS_EINVAL, "rms_norm: null argument");
        CK_REQUIRE(tm == (mask != nullptr), CKKS_EINVAL, "rms_norm: a mask is for the token-major layout, which needs one");
        CK_REQUIRE(shape->features >= 1 && shape->features <= (uint64_t)count * D, CKKS_EINVAL,
                   "rms_norm: %u features outside [1, %llu]", shape->features, (unsigned long long)count * D);
        CK_REQUIRE(ctx->n_p > 0, CKKS_EUNSUPPORTED, "rms_norm: the context has no special primes");
        Norm n;
        const uint32_t L = in[0].n_limbs, newton = shape->newton;
        CK_REQUIRE(L <= ctx->n_q && norm_limbs(ctx, L, tm, inv_root->degree, newton, &n), CKKS_ELEVEL,
                   "rms_norm: degree %u and %u Newton steps need %u to %u limbs, %u given", inv_root->degree, newton,
                   4 + tm + cheb_depth(inv_root->degree) + 2 * newton, ctx->n_q, L);
        const uint32_t Lv = n.Lv, m = n.m;
        CK_TRY(check_cts(in, count, L, what, "input"));
        CK_TRY(check_scales(in, count, what, "input"));
        CK_TRY(check_scale(in[0].scale, what, "input"));
        CK_TRY(check_cts(out, count, m - 1, what, "output"));
        const uint32_t wp = weights ? weights[0].n_polys : 0;
        if (weights) {
            CK_REQUIRE(wp == 1 || wp == 2, CKKS_EINVAL, "rms_norm: weights are plaintexts or ciphertexts");
            CK_TRY(check_list(ctx, weights, count, wp, m + 1, what, "weight"));
        }
        if (tm) CK_TRY(check_list(ctx, mask, 1, 1, L - 1, what, "mask"));
        if (residual) CK_TRY(check_list(ctx, residual, count, 2, m, what, "residual"));
        std::vector<Range> ins, outs;
        add_ranges(ins, ctx, in, count);
        add_ranges(ins, ctx, weights, count);
        add_ranges(ins, ctx, mask, 1);
        add_ranges(ins, ctx, residual, count);
        add_ranges(outs, ctx, out, count);
        CK_TRY(check_overlap(outs, ins, what));
        std::vector<Round> sums, spread;
        CK_TRY(sum_rounds(ctx, D, tm ? 1 : T, key_steps, keys, n_keys, &sums));
        if (tm) CK_TRY(sum_rounds(ctx, D, -1, key_steps, keys, n_keys, &spread));

        // scales: of the sums, of the weighted inputs, of the inverse root that gives the outputs the inputs' scale
        auto top = [&](uint32_t limbs) { return prime_of(ctx, limbs); };
        const double S = in[0].scale, d = shape->features;
        double sv = S * S / top(L);
        if (tm) sv = sv * mask->scale / top(L - 1);
        const double sx = weights ? S * weights[0].scale / top(m + 1) : S;
        const double last = S * top(m) / sx;
        CK_TRY(check_scale(sv, what, "sum of squares"));
        CK_TRY(check_scale(sx, what, "weighted input"));
        CK_TRY(check_scale(last, what, "inverse root"));
        const double s1 = top(Lv - 1);
        double by;
        StepInt k, c, kr{};
        CK_TRY(poly_map(*inv_root, s1, &by, &c, what));
        CK_TRY(scaled_int(by / d * (top(Lv) / sv), &k, what, "the interval's width"));
        CK_TRY(cheb_plan(ctx, inv_root->coefs, inv_root->degree, Lv - 1, s1, newton ? top(n.m0) : last, what, &n.plan));
        struct Iter {
            StepInt mean, eps, y;
        } it[4];
        double sy = newton ? top(n.m0) : last;
        for (uint32_t j = 0; j < newton; j++) {
            const uint32_t limbs = n.m0 - 2 * j;
            const double qa = top(limbs), qb = top(limbs - 1), to = j + 1 < newton ? top(limbs - 2) : last;
            const double s2 = sy * sy / qa, sn = to / 2 * qb / s2 * qa / sy, sp = sn * sy / qa * s2 / qb;
            CK_TRY(scaled_int(sn / d * (top(Lv) / sv), &it[j].mean, what, "the mean"));
            CK_TRY(scaled_int(shape->eps * sn, &it[j].eps, what, "eps"));
            CK_TRY(scaled_int(3.0 * (sp * qb / sy), &it[j].y, what, "a Newton step's value"));
            sy = to;
        }
        if (residual) CK_TRY(scaled_int(residual_scale * (S * top(m) / residual[0].scale), &kr, what, "the residual"));

        const uint32_t shp[6] = {L, count, T, shape->layout, inv_root->degree, newton};
        void *mem;
        CK_TRY(ctx_scratch(ctx, op_workspace_bytes(ctx, CKKS_OP_RMS_NORM, shp), &mem));
        (void)norm_mem(ctx, count, newton, (uint64_t *)mem, &n);
        const size_t N = ctx->n;

        // the sum of squares, over the ciphertexts and then over their features
        std::vector<const uint64_t *> x(count);
        for (uint32_t r = 0; r < count; r++) x[r] = in[r].data;
        CK_TRY(step_squares(ctx, L, x, L, n.d));
        std::vector<Step> st(1);
        st[0].d = n.d;
        st[0].out = n.v;
        CK_TRY(step_run(ctx, L, st, rlk, n.work));
        uint64_t *v = n.v, *v2 = n.v2;
        CK_TRY(run_rounds(ctx, L - 1, sums, &v, v == n.v ? n.v2 : n.v, n.work));
        if (tm) {
            v2 = v == n.v ? n.v2 : n.v;
            st[0] = Step{};
            st[0].product(v, L - 1, mask->data, mask->n_limbs, 1, 1);
            st[0].out = v2;
            CK_TRY(step_run(ctx, L - 1, st, nullptr, n.work));
            v = v2;
            CK_TRY(run_rounds(ctx, L - 2, spread, &v, v == n.v ? n.v2 : n.v, n.work));
        }

        // the mean on the polynomial's interval, and for each Newton step; its inverse root
        st.assign(1 + newton, Step{});
        st[0].term(v, Lv, k);
        st[0].c = c;
        st[0].out = n.t1;
        for (uint32_t j = 0; j < newton; j++) {
            st[1 + j].term(v, Lv, it[j].mean);
            st[1 + j].c = it[j].eps;
            st[1 + j].out = n.means + j * 2 * (size_t)L * N;
        }
        CK_TRY(step_run(ctx, Lv, st, nullptr, n.work));
        CK_TRY(cheb_run(ctx, n.plan, {n.t1}, {n.y}, {}, rlk, n.work));
        uint64_t *y = n.y, *y2 = n.y2;
        st.clear();
        for (uint32_t j = 0; j < newton; j++) {   // y (3 - (mean + eps) y^2) / 2
            const uint32_t limbs = n.m0 - 2 * j;
            uint64_t *b = n.ab + 2 * (size_t)L * N;
            st.assign(2, Step{});
            st[0].product(n.means + j * 2 * (size_t)L * N, Lv - 1, y, limbs);
            st[0].out = n.ab;
            st[1].product(y, limbs, y, limbs);
            st[1].out = b;
            CK_TRY(step_run(ctx, limbs, st, rlk, n.work));
            st.assign(1, Step{});
            st[0].product(n.ab, limbs - 1, b, limbs - 1, -1);
            st[0].term(y, limbs, it[j].y);
            st[0].out = y2;
            if (j + 1 < newton || !weights || count % kStepBatch == 0) {
                CK_TRY(step_run(ctx, limbs - 1, st, rlk, n.work));
                st.clear();
            }
            std::swap(y, y2);
        }

        // the inputs by their weights, a level above the inverse root: in one batch with its last Newton step (one
        // ciphertext of 24 limbs at N = 2^16 1281 -> 1229 us), unless that step would need a batch of its own (16
        // ciphertexts 3445 -> 3477 us); the products
        if (weights)
            for (uint32_t r = 0; r < count; r++) {
                Step w;
                w.product(in[r].data, L, weights[r].data, weights[r].n_limbs, 1, wp);
                w.out = n.xw + (size_t)r * 2 * m * N;
                x[r] = w.out;
                st.push_back(w);
            }
        CK_TRY(step_run(ctx, m + 1, st, rlk, n.work));
        st.assign(count, Step{});
        for (uint32_t r = 0; r < count; r++) {
            st[r].product(x[r], weights ? m : L, y, m);
            if (residual) st[r].term(residual[r].data, residual[r].n_limbs, kr);
            st[r].out = out[r].data;
        }
        CK_TRY(step_run(ctx, m, st, rlk, n.work));
        for (uint32_t r = 0; r < count; r++) out[r].scale = S;
        return CKKS_OK;
    });
}

}  // extern "C"

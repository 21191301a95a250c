// The packed projection with an epilogue, out_j = gate_j act((X W)_j + bias_j) + r residual_j.  Bias and, where nothing
// follows, residual go into the projection's sums before their rescale; the weights are encoded at the scale at which that
// rescale leaves what comes next: T_1 of the activation, the gate's factor or the output.  So an activation costs the
// levels of its sum alone, and the map of its interval no step.
#include <cmath>

#include "nonlinear.h"
#include "ops.h"

namespace {

// limbs along the way and the workspace: what the projection leaves (kept), then one region that the projection and
// what follows it use in turn
struct Epi {
    uint32_t L, n_out, depth, m;   // inputs, outputs, the activation's levels, limbs before the gate
    ChebPlan plan;
    size_t mid, steps, acts, after, kept, least;   // words: T_1, the tiles' steps, activated; bytes: see ProjHook
};
bool epi_limbs(const ckks_ctx *ctx, uint32_t L, uint32_t degree, bool gate, Epi *e)
{
    if (L < 2 || L > ctx->n_q || degree > kChebDegree) return false;
    e->L = L;
    e->depth = degree ? cheb_depth(degree) : 0;
    if (L < 2 + e->depth + gate) return false;
    e->m = L - 1 - e->depth;
    return true;
}
void epi_mem(const ckks_ctx *ctx, bool act, bool gate, Epi *e)
{
    const size_t N = ctx->n;
    e->mid = act || gate ? (size_t)e->n_out * 2 * (e->L - 1) * N : 0;
    e->steps = step_scratch_words(ctx, e->L, e->n_out, false);
    e->acts = act && gate ? (size_t)e->n_out * 2 * e->m * N : 0;
    e->after = e->acts + std::max(act ? cheb_scratch_words(ctx, e->plan, e->n_out) : 0,
                                  gate ? step_scratch_words(ctx, e->m, e->n_out) : 0);
    e->kept = ((e->mid + e->steps) * 8 + 255) & ~(size_t)255;
    e->least = (e->mid + e->after) * 8;
}

}  // namespace

// shape: {limbs, tokens, d_in, d_out, n1, layout, degree (0: no activation), gate (0 or 1)}
size_t epilogue_workspace_bytes(const ckks_ctx *ctx, const uint32_t *s)
{
    const bool tm = s[5] == CKKS_TOKEN_MAJOR;
    if (!ctx->n_p || s[5] > CKKS_FEATURE_MAJOR || s[7] > 1) return SIZE_MAX;
    const size_t proj = tm ? proj_tm_workspace_bytes(ctx, s[0], s[1], s[2], s[3], s[4])
                           : proj_workspace_bytes(ctx, s[0], s[1], s[2], s[3], s[4]);
    Epi e;
    if (proj == SIZE_MAX || !epi_limbs(ctx, s[0], s[6], s[7], &e)) return SIZE_MAX;
    e.n_out = s[3] / (ctx->n / 2 / s[1]);
    if (s[6]) (void)cheb_plan(ctx, nullptr, s[6], s[0] - 1, 1.0, 1.0, "", &e.plan);
    epi_mem(ctx, s[6] != 0, s[7] != 0, &e);
    return std::max(e.kept + proj, e.least);
}

extern "C" ckks_status ckks_linear_project_epilogue(ckks_ctx *ctx, const ckks_buf *in, const double *W,
                                                    const ckks_proj_shape *shape, uint32_t layout,
                                                    const ckks_epilogue *epi, const int32_t *key_steps,
                                                    const uint64_t *const *keys, uint32_t n_keys, ckks_buf *out)
{
    clear_error();
    const DeviceScope dev(ctx);
    return guarded("linear_project_epilogue", [&]() -> ckks_status {
        const char *what = "linear_project_epilogue";
        CK_REQUIRE(ctx && in && W && shape && epi && out && (!n_keys || (key_steps && keys)), CKKS_EINVAL,
                   "linear_project_epilogue: null argument");
        CK_REQUIRE(layout == CKKS_TOKEN_MAJOR || layout == CKKS_FEATURE_MAJOR, CKKS_EINVAL,
                   "linear_project_epilogue: unknown layout %u", layout);
        CK_REQUIRE(ctx->n_p > 0, CKKS_EUNSUPPORTED, "linear_project_epilogue: the context has no special primes");
        const uint32_t T = shape->tokens, slots = ctx->n / 2;
        CK_REQUIRE(T >= 1 && slots % T == 0, CKKS_EINVAL, "linear_project_epilogue: %u tokens do not divide %u slots", T,
                   slots);
        const uint32_t D = slots / T;
        CK_REQUIRE(shape->d_in && shape->d_out && shape->d_in % D == 0 && shape->d_out % D == 0, CKKS_EINVAL,
                   "linear_project_epilogue: d_in %u and d_out %u must be positive multiples of %u", shape->d_in,
                   shape->d_out, D);
        const ckks_poly *act = epi->act;
        if (act) CK_TRY(check_poly(act, what));
        const bool gate = epi->gate != nullptr;
        CK_REQUIRE(!(act || gate) || epi->dev_rlk, CKKS_EINVAL, "linear_project_epilogue: no relinearisation key");
        CK_REQUIRE(!epi->residual || std::isfinite(epi->residual_scale), CKKS_EINVAL,
                   "linear_project_epilogue: residual scale %g", epi->residual_scale);
        Epi e;
        const uint32_t L = in[0].n_limbs, n_in = shape->d_in / D, n_out = e.n_out = shape->d_out / D;
        CK_REQUIRE(epi_limbs(ctx, L, act ? act->degree : 0, gate, &e), CKKS_ELEVEL,
                   "linear_project_epilogue: inputs need %u to %u limbs, %u given",
                   2 + (act ? cheb_depth(act->degree) : 0) + gate, ctx->n_q, L);
        const uint32_t m = e.m, done = m - gate;
        CK_TRY(check_cts(in, n_in, L, what, "input"));
        CK_TRY(check_scales(in, n_in, what, "input"));
        CK_TRY(check_scale(in[0].scale, what, "input"));
        CK_TRY(check_cts(out, n_out, done, what, "output"));
        if (epi->bias) CK_TRY(check_list(ctx, epi->bias, n_out, 1, L, what, "bias"));
        if (gate) CK_TRY(check_list(ctx, epi->gate, n_out, 2, m, what, "gate"));
        if (epi->residual) CK_TRY(check_list(ctx, epi->residual, n_out, 2, done + 1, what, "residual"));
        std::vector<Range> ins, outs;
        add_ranges(ins, ctx, in, n_in);
        add_ranges(ins, ctx, epi->bias, n_out);
        add_ranges(ins, ctx, epi->gate, n_out);
        add_ranges(ins, ctx, epi->residual, n_out);
        ins.push_back({(const uint64_t *)W, (size_t)shape->d_in * shape->d_out});
        add_ranges(outs, ctx, out, n_out);
        CK_TRY(check_overlap(outs, ins, what));

        // scales: what the projection's rescale leaves, the factor that the gate takes
        auto top = [&](uint32_t limbs) { return (double)ctx->primes[limbs - 1]; };
        const double S = in[0].scale, to = gate ? S * top(m) / epi->gate[0].scale : S;
        StepInt c{}, kb{}, kr{};
        ProjHook hook{};
        double left = to;
        CK_TRY(check_scale(to, what, "gate's factor"));
        if (act) {
            double by;
            CK_TRY(poly_map(*act, top(L - 1), &by, &c, what));
            CK_TRY(cheb_plan(ctx, act->coefs, act->degree, L - 1, top(L - 1), to, what, &e.plan));
            left = by;
        }
        hook.w_scale = top(L) * (left / S);
        CK_REQUIRE(hook.w_scale <= 0x1p62, CKKS_ESCALE,
                   "linear_project_epilogue: weights would be encoded at scale %g, above 2^62", hook.w_scale);
        if (epi->bias)
            CK_TRY(scaled_int(act ? left * (top(L) / epi->bias[0].scale) : left * top(L) / epi->bias[0].scale, &kb, what,
                              "the bias"));
        if (epi->residual)
            CK_TRY(scaled_int(epi->residual_scale * (S * top(done + 1) / epi->residual[0].scale), &kr, what,
                              "the residual"));
        epi_mem(ctx, act != nullptr, gate, &e);
        const size_t N = ctx->n;
        hook.kept = e.kept;
        hook.least = e.least;
        auto residual = [&](uint32_t j) { return StepTerm{epi->residual[j].data, epi->residual[j].n_limbs, 2, kr}; };
        auto mid = [&](uint32_t j) { return (uint64_t *)hook.mem + (size_t)j * 2 * (L - 1) * N; };
        hook.finish = [&](const uint64_t *tot, uint32_t j0, uint32_t jc) {
            std::vector<Step> st(jc);
            for (uint32_t j = 0; j < jc; j++) {
                Step &s = st[j];
                s.term(tot + (size_t)j * 2 * L * N, L, StepInt{1, 0});
                if (epi->bias) s.term(epi->bias[j0 + j].data, epi->bias[j0 + j].n_limbs, kb, 1);
                if (epi->residual && !act && !gate) s.term(residual(j0 + j));
                s.c = c;
                s.out = act || gate ? mid(j0 + j) : out[j0 + j].data;
            }
            return step_run(ctx, L, st, nullptr, (uint64_t *)hook.mem + e.mid);
        };
        CK_TRY((layout == CKKS_TOKEN_MAJOR ? project_tm : project_fm)(ctx, in, W, shape, key_steps, keys, n_keys, nullptr,
                                                                      &hook));
        uint64_t *acts = (uint64_t *)hook.mem + e.mid, *work = acts + e.acts;
        std::vector<const uint64_t *> x(n_out);
        for (uint32_t j = 0; j < n_out; j++) x[j] = mid(j);
        if (act) {
            std::vector<uint64_t *> y(n_out);
            std::vector<StepTerm> extra;
            for (uint32_t j = 0; j < n_out; j++) {
                y[j] = gate ? acts + (size_t)j * 2 * m * N : out[j].data;
                if (epi->residual && !gate) extra.push_back(residual(j));
            }
            CK_TRY(cheb_run(ctx, e.plan, x, y, extra, epi->dev_rlk, work));
            for (uint32_t j = 0; j < n_out; j++) x[j] = y[j];
        }
        if (gate) {
            std::vector<Step> st(n_out);
            for (uint32_t j = 0; j < n_out; j++) {
                st[j].product(x[j], m, epi->gate[j].data, epi->gate[j].n_limbs);
                if (epi->residual) st[j].term(residual(j));
                st[j].out = out[j].data;
            }
            CK_TRY(step_run(ctx, m, st, epi->dev_rlk, work));
        }
        for (uint32_t j = 0; j < n_out; j++) out[j].scale = S;
        return CKKS_OK;
    });
}

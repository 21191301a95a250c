"""Steps (csrc/step.h) and sums of Chebyshev polynomials (csrc/cheb.hip) on the host: what a step may not be is refused before
anything is launched; the library's own plan of a sum is evaluated in plain arithmetic, for every degree."""
import host_program as hp

RING = r"""
#include "step.h"

static void ring(ckks_ctx &c)   // no device memory: enough for what is decided on the host
{
    c.log_n = 8;
    c.n = 256;
    c.n_q = 10;
    c.n_p = 1;
    c.dnum = 10;
    for (uint32_t i = 0; i <= c.n_q; i++) c.primes.push_back((1ull << 50) - (1ull << 20) * i - 1);
}
"""


def test_a_plaintext_product_has_no_factor(tmp_path):
    """The factor 2 or -1 belongs to products of ciphertexts; of a plaintext product every ring's kernels would have to
    apply it alike, and nothing asks for it."""
    hp.run(tmp_path, RING + r"""
int main()
{
    ckks_ctx c;
    ring(c);
    for (int mult : {2, -1}) {
        std::vector<Step> s(3);
        s[1].product(nullptr + 1, 4, nullptr + 1, 4, mult, 1);
        clear_error();
        CHECK(step_run(&c, 4, s, nullptr, nullptr) == CKKS_EINVAL);
        CHECK(std::strstr(ckks_last_error(), "plaintext"));
    }
    return 0;
}
""".replace("nullptr + 1", "(const uint64_t *)64"))


def test_more_terms_than_a_step_holds(tmp_path):
    """They are counted, not written behind the list, and the step is refused."""
    hp.run(tmp_path, RING + r"""
int main()
{
    ckks_ctx c;
    ring(c);
    std::vector<Step> s(2);
    uint64_t *const out = (uint64_t *)128;
    s[1].out = out;
    s[1].c = StepInt{5, 3};
    for (uint32_t i = 0; i < kStepTerms; i++) s[1].term((const uint64_t *)64, 4, StepInt{(int64_t)i, 0});
    CHECK(s[1].n_terms == kStepTerms && s[1].t[kStepTerms - 1].k.m == kStepTerms - 1);
    for (int more = 0; more < 4; more++) s[1].term((const uint64_t *)(64 + more), 7, StepInt{-1, 77}, 1);
    CHECK(s[1].out == out && s[1].c.m == 5 && s[1].c.sh == 3 && s[1].t[kStepTerms - 1].k.m == kStepTerms - 1);
    clear_error();
    CHECK(step_run(&c, 4, s, nullptr, nullptr) == CKKS_EINVAL);
    CHECK(std::strstr(ckks_last_error(), "terms"));
    return 0;
}
""")


def test_the_plan_of_every_degree(tmp_path):
    """The plan with real numbers for ciphertexts gives the sum; every object is there when it is read, the sum in as many
    levels as the degree has bits, and a residual's term fits beside the last step's own (kStepTerms = 9 in all).

    The bound, of values in units of their scales: an object adds at most 2^-50 by its integers (each off by 1/2 of about
    2^50) and 2^-50 by roundings of doubles.  T_2i is off by four times T_i's error and its own 2^-49, so T_i, i <= 64, by
    2^-49 (1 + 4 + .. + 4^6) < 2^-36.  A split's q has at most twice its sum's coefficients in all and r as many, so the
    coefficients of all sums of four splits are at most 1 + 3 + 9 + 27 + 81 = 121 times the first's; each is off by at most
    2^-36 of its coefficients and 2^-49 a term: 2^-29 of sum |c| + 1 in all."""
    out = hp.run(tmp_path, RING + r"""
static double value(const StepInt &k) { return std::ldexp((double)k.m, (int)k.sh); }

int main()
{
    ckks_ctx c;
    ring(c);
    uint64_t seed = 1;
    auto random = [&] { return (double)((seed = seed * 6364136223846793005ull + 1442695040888963407ull) >> 33) * 0x1p-30 - 1; };
    for (uint32_t degree = 1; degree <= kChebDegree; degree++) {
        std::vector<double> coef(degree + 1);
        for (double &x : coef) x = 4 * random() / 3;
        ChebPlan plan;
        const uint32_t L1 = 9;
        const double s1 = (double)c.primes[L1 - 1], target = 1.01 * 0x1p49;
        CHECK(cheb_plan(&c, coef.data(), degree, L1, s1, target, "test", &plan) == CKKS_OK);
        uint32_t bits = 0;
        while (degree >> bits) bits++;
        CHECK(plan.depth == bits && plan.L1 == L1 && plan.obj[0].depth == 0 && plan.obj.back().depth == bits);
        CHECK(plan.obj.back().scale == target);
        for (size_t i = 1; i < plan.obj.size(); i++) {
            const ChebObj &o = plan.obj[i];
            CHECK(o.depth >= 1 && o.depth <= bits && o.t.size() <= 8 && o.t.size() < kStepTerms);
            CHECK((o.x < 0) == (o.y < 0) && o.x < (int)i && o.y < (int)i);
            if (o.x >= 0) CHECK(plan.obj[o.x].depth < o.depth && plan.obj[o.y].depth < o.depth);
            for (const ChebTerm &t : o.t) CHECK(t.of < i && plan.obj[t.of].depth < o.depth);
        }
        double sum = 0;
        for (double x : coef) sum += std::fabs(x);
        for (double t : {-1.0, -0.3, 0.0, 0.77, 1.0}) {
            std::vector<double> v(plan.obj.size());
            v[0] = t * s1;
            for (size_t i = 1; i < plan.obj.size(); i++) {
                const ChebObj &o = plan.obj[i];
                double s = o.x < 0 ? 0.0 : o.mult * v[o.x] * v[o.y];
                for (const ChebTerm &z : o.t) s += value(z.k) * v[z.of];
                v[i] = s / (double)c.primes[L1 - o.depth] + value(o.c);
            }
            double want = 0, b0 = 1, b1 = t;   // T_i by their recurrence
            for (uint32_t i = 0; i <= degree; i++) {
                want += coef[i] * b0;
                const double b2 = 2 * t * b1 - b0;
                b0 = b1;
                b1 = b2;
            }
            CHECK(std::fabs(v.back() / target - want) < 0x1p-29 * (sum + 1));
        }
    }
    std::printf("%u degrees", kChebDegree);
    return 0;
}
""")
    assert out == "127 degrees"


def test_more_products_than_a_list_holds(tmp_path):
    """ModUps of products take their operands from lists of kPolyList: a longer batch is refused on the host.  Those of
    polynomials alone take no second factor (one for every entry of a batch, it was used for the first)."""
    hp.run(tmp_path, RING + r"""
#include "ks_args.h"
#include "ops.h"

int main()
{
    ckks_ctx c;
    ring(c);
    PolyProd p[2] = {};
    ckks_status (*const polys)(ckks_ctx *, const PolySrc &, uint32_t, uint32_t, uint64_t *, uint64_t *) = blk_modup;
    CHECK(polys);
    for (uint32_t count : {(uint32_t)kPolyList + 1, 70000u}) {
        clear_error();
        CHECK(blk_modup(&c, p[0], count, 3, nullptr, nullptr) == CKKS_EINVAL);
        CHECK(std::strstr(ckks_last_error(), "products"));
        clear_error();
        CHECK(up_modup_cols(&c, p[0], count, 3, nullptr) == CKKS_EINVAL);
        CHECK(std::strstr(ckks_last_error(), "products"));
    }
    return 0;
}
""")

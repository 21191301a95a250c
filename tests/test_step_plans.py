"""Steps (csrc/step.h) on the host: what a step may not be is refused before anything is launched."""
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

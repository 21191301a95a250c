// What the calls over lists of ciphertexts check alike, and the guard around their host side.
#pragma once
#include <algorithm>
#include <new>
#include <vector>

#include "ckks_internal.h"

namespace {

ckks_status check_cts(const ckks_buf *b, uint32_t n, uint32_t L, const char *what, const char *name)
{
    for (uint32_t i = 0; i < n; i++) {
        CK_REQUIRE(b[i].data && b[i].n_polys == 2, CKKS_EINVAL, "%s: %s %u is not a ciphertext", what, name, i);
        CK_REQUIRE(b[i].n_limbs == L, CKKS_ELEVEL, "%s: %s %u has %u limbs, expected %u", what, name, i, b[i].n_limbs, L);
    }
    return CKKS_OK;
}
ckks_status check_scales(const ckks_buf *b, uint32_t n, const char *what, const char *name)
{
    for (uint32_t i = 0; i < n; i++)
        CK_REQUIRE(b[i].scale == b[0].scale, CKKS_ESCALE, "%s: %s scales differ", what, name);
    return CKKS_OK;
}

struct Range {
    const uint64_t *p;
    size_t n;
};
// outs overlap neither one another nor any of ins
ckks_status check_overlap(std::vector<Range> outs, const std::vector<Range> &ins, const char *what)
{
    std::sort(outs.begin(), outs.end(), [](const Range &a, const Range &b) { return a.p < b.p; });
    for (size_t i = 1; i < outs.size(); i++)
        CK_REQUIRE(outs[i - 1].p + outs[i - 1].n <= outs[i].p, CKKS_EINVAL, "%s: two outputs overlap", what);
    for (const Range &r : ins) {
        auto it = std::upper_bound(outs.begin(), outs.end(), r.p + (r.n - 1),
                                   [](const uint64_t *p, const Range &b) { return p < b.p; });
        if (it == outs.begin()) continue;
        --it;
        CK_REQUIRE(it->p + it->n <= r.p, CKKS_EINVAL, "%s: an output overlaps an input", what);
    }
    return CKKS_OK;
}

void add_ranges(std::vector<Range> &to, const ckks_ctx *ctx, const ckks_buf *b, uint32_t n)
{
    for (uint32_t i = 0; b && i < n; i++) to.push_back({b[i].data, (size_t)b[i].n_polys * b[i].n_limbs * ctx->n});
}

// no C++ exception crosses the C boundary: the argument lists are the only host memory a call takes
template <typename Body>
ckks_status guarded(const char *what, Body body)
{
    try {
        return body();
    } catch (const std::bad_alloc &) {
        return set_error(CKKS_ENOMEM, "%s: out of host memory", what);
    } catch (...) {
        return set_error(CKKS_ENOMEM, "%s: argument lists too long", what);
    }
}

// launches go to the context's stream, on its device whichever is current
struct DeviceScope {
    int before = -1;
    explicit DeviceScope(const ckks_ctx *ctx)
    {
        int d;
        if (ctx && hipGetDevice(&d) == hipSuccess && d != ctx->device && hipSetDevice(ctx->device) == hipSuccess) before = d;
    }
    ~DeviceScope()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

}  // namespace

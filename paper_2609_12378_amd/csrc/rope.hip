// Rotary positions on ciphertexts and the encrypted key/value cache: the tables, and the calls.  Both are weighted sums
// of rotations (wsum.hip):
//   rope     cos at the slot itself, -sin and sin at the slots of its pair, half the rotated part away or next to it;
//   append   the same, every rotation lowered by the token slots that the new tokens move up, the weights zero
//            outside the new tokens' slots of the page; values take one term with a 0/1 weight.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ckks_internal.h"
#include "ntt_core.h"
#include "ops.h"
#include "wsum.h"

namespace {

constexpr int kThreads = 256;
// Tables are made once for a position and serve every layer and head, so they are plain element-wise kernels around the
// encoder's transforms.
// cos and sin of positions[i] * inv_freq[k], times factor.  The product is taken with its rounding error e (an FMA) and
// the angles added, so a far position's angle is as exact as a near one's.
__global__ __launch_bounds__(kThreads) void k_cos_sin(const int64_t *positions, const double *inv_freq, uint32_t half,
                                                      size_t total, double factor, double *cs, double *sn)
{
    const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= total) return;
    const double p = (double)positions[i / half], f = inv_freq[i % half];
    const double ang = p * f, e = fma(p, f, -ang);
    double s, c, se, ce;
    sincos(ang, &s, &c);
    sincos(e, &se, &ce);
    cs[i] = factor * fma(c, ce, -s * se);
    sn[i] = factor * fma(s, ce, c * se);
}

struct Shape {
    uint32_t tokens, feats, head_dim, rot_dim;
    bool fm, interleaved;
};
// Slot vectors of the tables: out[b][N/2], b < n_tab the rotary terms (cos; -sin of the lower feature of a pair, which
// reads the upper one; sin of the upper feature), table n_tab - with `mask` - 1 on the live tokens.  Live are the
// tokens first .. first + count - 1, token first + i with row i of cos and sin ([count][rot_dim / 2]).
__global__ __launch_bounds__(kThreads) void k_slots(double *out, Shape s, uint32_t first, uint32_t count, uint32_t n_tab,
                                                    const double *cs, const double *sn, uint32_t slots)
{
    const uint32_t x = blockIdx.x * kThreads + threadIdx.x, b = blockIdx.y;
    if (x >= slots) return;
    const uint32_t t = s.fm ? x % s.tokens : x / s.feats, f = s.fm ? x / s.tokens : x % s.feats;
    double v = 0.0;
    if (t >= first && t - first < count) {
        const uint32_t d = f % s.head_dim, half = s.rot_dim / 2;
        const bool turned = d < s.rot_dim && f < s.feats - s.feats % s.head_dim;
        const bool upper = s.interleaved ? d & 1u : d >= half;
        const size_t at = (size_t)(t - first) * half + (s.interleaved ? d >> 1 : upper ? d - half : d);
        if (b == n_tab) v = 1.0;
        else if (b == 0) v = turned ? cs[at] : 1.0;
        else if (turned && upper == (b == 2)) v = b == 1 ? -sn[at] : sn[at];
    }
    out[(size_t)b * slots + x] = v;
}

// residues of m[b][N] modulo the primes of the map, out[b][map.n][N]
__global__ __launch_bounds__(kThreads) void k_rns(uint64_t *out, const int64_t *m, LimbMap map,
                                                  const ModQ *__restrict__ mods, uint32_t log_n)
{
    const uint32_t col = blockIdx.x * kThreads + threadIdx.x, row = blockIdx.y, b = blockIdx.z;
    if (col >= (1u << log_n)) return;
    const ModQ q = mods[map.prime[row]];
    const nttc::Ar<false> ar(q);
    out[(((size_t)b * map.n + row) << log_n) + col] = ar.from_i64(m[((size_t)b << log_n) + col], q);
}

LimbMap ext_map(const ckks_ctx *ctx, uint32_t L)
{
    LimbMap m{};
    m.n = L + ctx->n_p;
    for (uint32_t r = 0; r < m.n; r++) m.prime[r] = (uint8_t)(r < L ? r : ctx->n_q + (r - L));
    return m;
}

dim3 grid_of(const ckks_ctx *ctx, uint32_t rows, uint32_t z) { return dim3((ctx->n + kThreads - 1) / kThreads, rows, z); }

// ------------------------------------------------------------------------------------------- arguments --------------
ckks_status check_shape(const ckks_ctx *ctx, const ckks_rope_shape *s, const char *what, bool rotary, Shape *out)
{
    CK_REQUIRE(s, CKKS_EINVAL, "%s: null shape", what);
    const uint32_t slots = ctx->n / 2, T = s->tokens;
    CK_REQUIRE(T >= 1 && T <= slots && (T & (T - 1)) == 0, CKKS_EINVAL, "%s: %u tokens are not a power of two in [1, %u]",
               what, T, slots);
    const uint32_t D = slots / T;
    CK_REQUIRE(s->head_dim >= 1 && s->head_dim <= D, CKKS_EINVAL, "%s: heads of %u features outside [1, %u]", what,
               s->head_dim, D);
    CK_REQUIRE(s->rot_dim % 2 == 0 && s->rot_dim <= s->head_dim, CKKS_EINVAL,
               "%s: a rotated part of %u features is odd or larger than a head of %u", what, s->rot_dim, s->head_dim);
    CK_REQUIRE(!rotary || s->rot_dim >= 2, CKKS_EINVAL, "%s: no features to rotate", what);
    CK_REQUIRE(s->layout == CKKS_TOKEN_MAJOR || s->layout == CKKS_FEATURE_MAJOR, CKKS_EINVAL, "%s: unknown layout %u", what,
               s->layout);
    CK_REQUIRE(s->pairing == CKKS_ROPE_HALF || s->pairing == CKKS_ROPE_INTERLEAVED, CKKS_EINVAL, "%s: unknown pairing %u",
               what, s->pairing);
    *out = Shape{T, D, s->head_dim, s->rot_dim, s->layout == CKKS_FEATURE_MAJOR, s->pairing == CKKS_ROPE_INTERLEAVED};
    return CKKS_OK;
}

// left rotation of the pair above, in slots
int64_t pair_step(const Shape &s) { return (int64_t)(s.interleaved ? 1 : s.rot_dim / 2) * (s.fm ? s.tokens : 1); }

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

// the terms' automorphisms and keys: left rotations by base, base + h, base - h
ckks_status find_keys(const ckks_ctx *ctx, WsumKind *w, uint32_t n, int64_t base, int64_t h, const int32_t *key_steps,
                      const uint64_t *const *keys, uint32_t n_keys, const char *what)
{
    const int64_t slots = ctx->n / 2;
    w->n = n;
    for (uint32_t j = 0; j < n; j++) {
        const int64_t st = ((base + (j == 0 ? 0 : j == 1 ? h : -h)) % slots + slots) % slots;
        w->g[j] = ckks_galois_elt(ctx, (int32_t)st);
        w->key[j] = nullptr;
        if (!st) continue;
        w->rotated = 1;
        for (uint32_t r = 0; r < n_keys && !w->key[j]; r++)
            if ((((int64_t)key_steps[r] % slots) + slots) % slots == st) w->key[j] = keys[r];
        CK_REQUIRE(w->key[j], CKKS_ENOKEY, "%s: no key for step %lld (modulo %lld)", what, (long long)st, (long long)slots);
    }
    return CKKS_OK;
}

// tables of one page: the rotary ones (n_rot) and, with `mask`, one of 0 and 1
ckks_status make_tables(ckks_ctx *ctx, const Shape &s, uint32_t first, uint32_t count, uint32_t n_rot, bool mask,
                        const double *cs, const double *sn, uint32_t L, uint64_t *out, void *mem)
{
    const uint32_t slots = ctx->n / 2, nb = n_rot + (mask ? 1 : 0);
    double *z = (double *)mem;
    double2 *work = (double2 *)(z + (size_t)nb * slots);
    int64_t *m = (int64_t *)((char *)work + enc_work_bytes(ctx, nb));
    prof_begin(ctx, K_ELEM, 8.0 * nb * slots);
    hipLaunchKernelGGL(k_slots, dim3((slots + kThreads - 1) / kThreads, nb), dim3(kThreads), 0, ctx->stream, z, s, first,
                       count, n_rot, cs, sn, slots);
    prof_end(ctx, K_ELEM);
    HIP_TRY(hipGetLastError());
    SlotSource src;
    src.re = z;
    CK_TRY(enc_coeffs(ctx, src, nb, (double)ctx->primes[L - 1], work, m));
    const LimbMap map = ext_map(ctx, L);
    prof_begin(ctx, K_TO_RNS, 8.0 * nb * ctx->n * (1 + map.n));
    hipLaunchKernelGGL(k_rns, grid_of(ctx, map.n, nb), dim3(kThreads), 0, ctx->stream, out, m, map, ctx->d_mod, ctx->log_n);
    prof_end(ctx, K_TO_RNS);
    HIP_TRY(hipGetLastError());
    return launch_ntt(ctx, out, nb * map.n, map, false);
}
size_t tables_bytes(const ckks_ctx *ctx, uint32_t nb)
{
    return (size_t)nb * ctx->n / 2 * sizeof(double) + enc_work_bytes(ctx, nb) + (size_t)nb * ctx->n * sizeof(int64_t);
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

size_t rope_workspace_bytes(const ckks_ctx *ctx, uint32_t L, uint32_t count)
{
    if (L < 2 || L > ctx->n_q || !ctx->n_p || !count) return SIZE_MAX;
    return wsum_scratch_words(ctx, L, count, 1) * 8;
}
size_t append_workspace_bytes(const ckks_ctx *ctx, uint32_t L, uint32_t heads)
{
    if (L < 2 || L > ctx->n_q || !ctx->n_p || !heads) return SIZE_MAX;
    return wsum_scratch_words(ctx, L, (uint32_t)std::min<uint64_t>(2 * (uint64_t)heads, UINT32_MAX), kWsumPages) * 8;
}
size_t rope_tables_workspace_bytes(const ckks_ctx *ctx) { return tables_bytes(ctx, kWsumTerms + 1); }

extern "C" {

ckks_status ckks_rope_cos_sin(ckks_ctx *ctx, const int64_t *positions, uint32_t count, const double *inv_freq,
                              uint32_t half, double factor, double *cs, double *sn)
{
    clear_error();
    const DeviceScope dev(ctx);
    CK_REQUIRE(ctx, CKKS_EINVAL, "rope_cos_sin: null context");
    if (!count || !half) return CKKS_OK;
    CK_REQUIRE(positions && inv_freq && cs && sn, CKKS_EINVAL, "rope_cos_sin: null argument");
    CK_REQUIRE(std::isfinite(factor), CKKS_EINVAL, "rope_cos_sin: the factor must be finite");
    const size_t total = (size_t)count * half;
    const size_t blocks = (total + kThreads - 1) / kThreads;
    CK_REQUIRE(blocks <= 0x7fffffffu, CKKS_EINVAL, "rope_cos_sin: %u positions of %u frequencies", count, half);
    prof_begin(ctx, K_ELEM, 16.0 * total);
    hipLaunchKernelGGL(k_cos_sin, dim3((uint32_t)blocks), dim3(kThreads), 0, ctx->stream, positions, inv_freq, half, total,
                       factor, cs, sn);
    prof_end(ctx, K_ELEM);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

ckks_status ckks_rope_tables(ckks_ctx *ctx, const ckks_rope_shape *shape, uint32_t first, uint32_t count, const double *cs,
                             const double *sn, uint32_t n_limbs, uint64_t *tables)
{
    clear_error();
    const DeviceScope dev(ctx);
    CK_REQUIRE(ctx && tables, CKKS_EINVAL, "rope_tables: null argument");
    Shape s;
    CK_TRY(check_shape(ctx, shape, "rope_tables", true, &s));
    CK_REQUIRE(n_limbs >= 2 && n_limbs <= ctx->n_q, CKKS_ELEVEL, "rope_tables: %u limbs outside [2, %u]", n_limbs, ctx->n_q);
    CK_REQUIRE(ctx->n_p > 0, CKKS_EUNSUPPORTED, "rope_tables: the context has no special primes");
    CK_REQUIRE(first <= s.tokens && count <= s.tokens - first, CKKS_EINVAL, "rope_tables: tokens %u .. %llu of %u", first,
               (unsigned long long)first + count, s.tokens);
    CK_REQUIRE(!count || (cs && sn), CKKS_EINVAL, "rope_tables: null argument");
    void *w;
    CK_TRY(ctx_scratch(ctx, op_workspace_bytes(ctx, CKKS_OP_ROPE_TABLES, nullptr), &w));
    return make_tables(ctx, s, first, count, kWsumTerms, false, cs, sn, n_limbs, tables, w);
}

ckks_status ckks_cache_tables(ckks_ctx *ctx, const ckks_rope_shape *shape, uint32_t length, uint32_t count, const double *cs,
                              const double *sn, uint32_t n_limbs, uint64_t *tables)
{
    clear_error();
    const DeviceScope dev(ctx);
    CK_REQUIRE(ctx, CKKS_EINVAL, "cache_tables: null context");
    Shape s;
    CK_TRY(check_shape(ctx, shape, "cache_tables", false, &s));
    CK_REQUIRE(!s.fm, CKKS_EUNSUPPORTED, "cache_tables: pages are token-major");
    CK_REQUIRE(n_limbs >= 2 && n_limbs <= ctx->n_q, CKKS_ELEVEL, "cache_tables: %u limbs outside [2, %u]", n_limbs, ctx->n_q);
    CK_REQUIRE(ctx->n_p > 0, CKKS_EUNSUPPORTED, "cache_tables: the context has no special primes");
    CK_REQUIRE(count <= s.tokens, CKKS_EINVAL, "cache_tables: %u tokens at once, a ciphertext holds %u", count, s.tokens);
    if (!count) return CKKS_OK;
    CK_REQUIRE(tables && (!s.rot_dim || (cs && sn)), CKKS_EINVAL, "cache_tables: null argument");
    void *w;
    CK_TRY(ctx_scratch(ctx, op_workspace_bytes(ctx, CKKS_OP_ROPE_TABLES, nullptr), &w));
    const uint32_t off = length % s.tokens, n0 = std::min(count, s.tokens - off), n_rot = s.rot_dim ? kWsumTerms : 0;
    CK_TRY(make_tables(ctx, s, off, n0, n_rot, true, cs, sn, n_limbs, tables, w));
    if (n0 == count) return CKKS_OK;
    const size_t done = (size_t)n0 * (s.rot_dim / 2), page = (size_t)(n_rot + 1) * (n_limbs + ctx->n_p) * ctx->n;
    return make_tables(ctx, s, 0, count - n0, n_rot, true, s.rot_dim ? cs + done : nullptr, s.rot_dim ? sn + done : nullptr,
                       n_limbs, tables + page, w);
}

ckks_status ckks_rope(ckks_ctx *ctx, const ckks_buf *in, uint32_t count, const ckks_rope_shape *shape,
                      const uint64_t *tables, const int32_t *key_steps, const uint64_t *const *keys, uint32_t n_keys,
                      ckks_buf *out)
{
    clear_error();
    const DeviceScope dev(ctx);
    return guarded("rope", [&]() -> ckks_status {
        CK_REQUIRE(ctx, CKKS_EINVAL, "rope: null context");
        Shape s;
        CK_TRY(check_shape(ctx, shape, "rope", true, &s));
        if (!count) return CKKS_OK;
        CK_REQUIRE(in && out && tables && (!n_keys || (key_steps && keys)), CKKS_EINVAL, "rope: null argument");
        CK_REQUIRE(ctx->n_p > 0, CKKS_EUNSUPPORTED, "rope: the context has no special primes");
        const uint32_t L = in[0].n_limbs;
        CK_REQUIRE(L >= 2 && L <= ctx->n_q, CKKS_ELEVEL, "rope: inputs need 2 to %u limbs, %u given", ctx->n_q, L);
        CK_TRY(check_cts(in, count, L, "rope", "input"));
        CK_TRY(check_cts(out, count, L - 1, "rope", "output"));
        const size_t N = ctx->n, row_words = (size_t)(L + ctx->n_p) * N;
        std::vector<Range> ins(count), outs(count);
        std::vector<WsumCt> cts(count);
        for (uint32_t r = 0; r < count; r++) {
            ins[r] = {in[r].data, 2 * (size_t)L * N};
            outs[r] = {out[r].data, 2 * (size_t)(L - 1) * N};
            cts[r] = {in[r].data, 0, {out[r].data}, {}};
        }
        CK_TRY(check_overlap(outs, ins, "rope"));
        WsumKind kinds[kWsumKinds] = {};
        CK_TRY(find_keys(ctx, &kinds[0], kWsumTerms, 0, pair_step(s), key_steps, keys, n_keys, "rope"));
        for (uint32_t j = 0; j < kWsumTerms; j++) kinds[0].tab[0][j] = tables + j * row_words;
        const uint32_t shp[2] = {L, count};
        void *mem;
        CK_TRY(ctx_scratch(ctx, op_workspace_bytes(ctx, CKKS_OP_ROPE, shp), &mem));
        CK_TRY(wsum_run(ctx, L, 1, kinds, cts, (uint64_t *)mem));
        for (uint32_t r = 0; r < count; r++) out[r].scale = in[r].scale;
        return CKKS_OK;
    });
}

ckks_status ckks_cache_append(ckks_ctx *ctx, const ckks_buf *k, const ckks_buf *v, uint32_t n_heads,
                              const ckks_rope_shape *shape, uint32_t src, uint32_t length, uint32_t count,
                              const uint64_t *tables, const int32_t *key_steps, const uint64_t *const *keys,
                              uint32_t n_keys, const ckks_cache *cache, const uint32_t *fork)
{
    clear_error();
    const DeviceScope dev(ctx);
    return guarded("cache_append", [&]() -> ckks_status {
        CK_REQUIRE(ctx, CKKS_EINVAL, "cache_append: null context");
        Shape s;
        CK_TRY(check_shape(ctx, shape, "cache_append", false, &s));
        CK_REQUIRE(!s.fm, CKKS_EUNSUPPORTED, "cache_append: pages are token-major");
        CK_REQUIRE(src <= s.tokens && count <= s.tokens - src, CKKS_EINVAL, "cache_append: tokens %u .. %llu of %u", src,
                   (unsigned long long)src + count, s.tokens);
        CK_REQUIRE((uint64_t)length + count <= UINT32_MAX, CKKS_EINVAL, "cache_append: %u tokens after %u", count, length);
        if (!n_heads || !count) return CKKS_OK;
        CK_REQUIRE(k && v && tables && cache && cache->k_pages && cache->v_pages && cache->table &&
                       (!n_keys || (key_steps && keys)), CKKS_EINVAL, "cache_append: null argument");
        CK_REQUIRE(ctx->n_p > 0, CKKS_EUNSUPPORTED, "cache_append: the context has no special primes");
        const uint32_t L = k[0].n_limbs, T = s.tokens;
        CK_REQUIRE(L >= 2 && L <= ctx->n_q, CKKS_ELEVEL, "cache_append: inputs need 2 to %u limbs, %u given", ctx->n_q, L);
        CK_TRY(check_cts(k, n_heads, L, "cache_append", "key"));
        CK_TRY(check_cts(v, n_heads, L, "cache_append", "value"));
        CK_TRY(check_scales(k, n_heads, "cache_append", "key"));
        CK_TRY(check_scales(v, n_heads, "cache_append", "value"));
        const uint32_t b0 = length / T, blocks = (length + count - 1) / T - b0 + 1, off = length % T;
        CK_REQUIRE(cache->n_blocks >= b0 + blocks, CKKS_EINVAL, "cache_append: token %u needs block %u, the table has %u",
                   length + count - 1, b0 + blocks - 1, cache->n_blocks);
        const size_t N = ctx->n, ctw = 2 * (size_t)(L - 1) * N;
        std::vector<Range> ins, outs;
        std::vector<WsumCt> cts;
        for (uint32_t kv = 0; kv < 2; kv++) {
            ckks_buf *pages = kv ? cache->v_pages : cache->k_pages;
            const ckks_buf *x = kv ? v : k;
            const char *name = kv ? "value page" : "key page";
            for (uint32_t h = 0; h < n_heads; h++) {
                ins.push_back({x[h].data, 2 * (size_t)L * N});
                WsumCt ct{x[h].data, kv, {}, {}};
                for (uint32_t b = 0; b < blocks; b++) {
                    const uint32_t p = cache->table[(size_t)h * cache->n_blocks + b0 + b];
                    CK_REQUIRE(p < cache->n_pages, CKKS_EINVAL, "cache_append: head %u, block %u: page %u of %u", h, b0 + b,
                               p, cache->n_pages);
                    CK_TRY(check_cts(&pages[p], 1, L - 1, "cache_append", name));
                    ct.out[b] = pages[p].data;
                    outs.push_back({pages[p].data, ctw});
                    if (b || !off) continue;
                    // a started page goes on, itself or the one it is forked from
                    const uint32_t f = fork ? fork[h] : p;
                    CK_REQUIRE(f < cache->n_pages, CKKS_EINVAL, "cache_append: head %u takes over page %u of %u", h, f,
                               cache->n_pages);
                    CK_TRY(check_cts(&pages[f], 1, L - 1, "cache_append", name));
                    CK_REQUIRE(pages[f].scale == x[h].scale, CKKS_ESCALE,
                               "cache_append: page %u has scale %g, the new tokens %g", f, pages[f].scale, x[h].scale);
                    ct.prev[b] = pages[f].data;
                    if (pages[f].data != pages[p].data) ins.push_back({pages[f].data, ctw});
                }
                cts.push_back(ct);
            }
        }
        CK_TRY(check_overlap(outs, ins, "cache_append"));
        // the keys' weights, then the values': either page's tables
        const size_t row_words = (size_t)(L + ctx->n_p) * N;
        const uint32_t n_rot = s.rot_dim ? kWsumTerms : 0;
        const int64_t base = -(int64_t)((off + T - src) % T) * s.feats;
        WsumKind kinds[kWsumKinds] = {};
        CK_TRY(find_keys(ctx, &kinds[0], n_rot ? n_rot : 1, base, n_rot ? pair_step(s) : 0, key_steps, keys, n_keys,
                         "cache_append"));
        CK_TRY(find_keys(ctx, &kinds[1], 1, base, 0, key_steps, keys, n_keys, "cache_append"));
        for (uint32_t b = 0; b < blocks; b++) {
            const uint64_t *t = tables + (size_t)b * (n_rot + 1) * row_words;
            for (uint32_t j = 0; j < kinds[0].n; j++) kinds[0].tab[b][j] = t + j * row_words;
            kinds[1].tab[b][0] = t + n_rot * row_words;
        }
        const uint32_t shp[2] = {L, n_heads};
        void *mem;
        CK_TRY(ctx_scratch(ctx, op_workspace_bytes(ctx, CKKS_OP_CACHE_APPEND, shp), &mem));
        CK_TRY(wsum_run(ctx, L, blocks, kinds, cts, (uint64_t *)mem));
        for (uint32_t h = 0; h < n_heads; h++)
            for (uint32_t b = 0; b < blocks; b++) {
                const uint32_t p = cache->table[(size_t)h * cache->n_blocks + b0 + b];
                cache->k_pages[p].scale = k[h].scale;
                cache->v_pages[p].scale = v[h].scale;
            }
        return CKKS_OK;
    });
}

}  // extern "C"

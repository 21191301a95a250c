// Weighted sums of rotations of a ciphertext (c0, c1) at level l, divided by P q_l:
//
//   t_j,k = sum_d sigma_gj(D_d) key_j,d,k + [k = 0] P sigma_gj(c0)     over Q_l u P (D the ModUp digits of c1)
//   t_0,k = P c_k                                                       (a term that is not rotated)
//   u_k   = sum_j pt_j t_j,k,            out = Rescale(ModDown(u))  (+ prev)
//
// The weights multiply before the division by P (they are encoded over Q_l u P), so a sum of rotations takes one ModUp
// and one division where rotate, multiply and add take a ModDown per rotation: the double hoisting of Bossuat et al.
// 2021.  ModDown(P x) = x exactly, so the unrotated term is what a plaintext product gives, and an output of that term
// alone needs no ModUp and no P rows.
//
// Two passes a transform with fp64 arithmetic (N >= 2^14, every prime of the level below 2^50): after the ModUp
//   1. k_wsum_intt8   u on the rows modulo q_l and P, with the row pass of their inverse transform;
//   2. k_quot_col     its column pass: centred digits y_i of the P rows, U P^-1 of the q_l row;
//   3. k_quot_col8    x_t = sum_i y_i [P / p_i]_t + P w for every target q_t, t < l, with the forward column pass
//      (elsewhere k_quot_col16, or for many reads k_quot_conv and a column pass), w the centred top coefficient of the
//      quotient by P: w = [(U - sum_i y_i [P / p_i]) P^-1]_{q_l}.  ModDown and rescale subtract Conv(y) P^-1 and then
//      w, so out = (u - NTT(x)) (P q_l)^-1 holds for both together and the q_l row never leaves the coefficient domain;
//   4. k_wsum_fin8    the forward row pass, u on the rows below q_l (in registers, never in HBM), the quotient, prev.
// Rings of 2^12 and 2^13 points do the same in whole rows (wsum_block.hip), other primes and rings in exact 128-bit
// sums (wsum_exact.hip).
#include <algorithm>

#include "conv_col.h"
#include "ops.h"
#include "wsum_args.h"
#include "wsum_pos.h"

namespace {

constexpr int kThreads = 256;
using namespace wsum;
using nttc::kE;
using nttc::kE8;

// ------------------------------------------------------------------------- two passes, fp64 ----------------------------

// the words of sigma_g(p) at an even position and the next, j' = source of the even one
__device__ __forceinline__ Pair ld2_auto(const uint64_t *p, uint32_t src)
{
    const Pair v = ld2(p + (src & ~1u));
    return src & 1u ? Pair{v.y, v.x} : v;
}

// The words that one term takes at PU pairs of positions: c0 (and, unrotated, c1 in place of the first digit), the
// digits, the key's two halves, the tables.  A unit's loads are issued together, and the next unit's before its own
// sums: what bounds these kernels otherwise is the wait on one row after another with two or three waves a SIMD.
template <int ND, int PU, int NOUT>
struct Unit {
    Pair c[PU], dig[ND][PU], b[ND][PU], a[ND][PU], tab[NOUT][PU];
    uint32_t flip[PU];
};

// u of output o at the 8 positions of a thread, both components, as doubles: |u| <= 2.6 q (a term of at most 0.7 q
// after the reduction of t, or 0.83 q unrotated).  Unrotated kinds: pt c without the factor P.  A digit's own rows are
// the ciphertext's (the ModUp leaves them out).  Q: the row is one of the q limbs (the P rows have no c terms).
template <int ND, int NOUT, bool Q>
__device__ __forceinline__ void wsum8(const WsumKind &w, const Ct &ct, const Dims &d, uint32_t row, double pq, const A &ar,
                                      const Positions &ps, double (&u)[NOUT][2][kE8])
{
    constexpr int PU = 1, kUnits = 4 / PU;   // two pairs a unit hold more words than the registers
    using U = Unit<ND, PU, NOUT>;
    const size_t rw = (size_t)row << d.log_n, half = (size_t)d.L << d.log_n;
    const size_t kstride = (size_t)d.key_rows << d.log_n, dstride = (size_t)d.ext << d.log_n;
    const size_t krow = (size_t)d.prime(row) << d.log_n;
    const uint64_t *c0 = ct.c + rw;
    const uint32_t own = Q ? row / d.alpha : ~0u;
    auto load = [&](U &x, uint32_t j, int p0) {
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t g = w.g[j], kg = ps.start(g);
        const uint64_t *key = w.key[j] + krow;
#pragma unroll
        for (int e = 0; e < PU; e++) {
            const uint32_t sc = ps.source(kg, g, 2 * (p0 + e)), at = sc & ~1u;
            x.flip[e] = sc & 1u;
            if constexpr (Q) x.c[e] = ld2(c0 + at);
#pragma unroll
            for (int i = 0; i < ND; i++)
                x.dig[i][e] = ld2((Q && (uint32_t)i == own ? ct.c + half : ct.dig + i * dstride) + rw + at);
        }
#pragma unroll
        for (int e = 0; e < PU; e++) {
            const uint32_t at = ps.pos(2 * (p0 + e));
#pragma unroll
            for (int i = 0; i < ND; i++) {
                x.b[i][e] = ld2(key + 2 * i * kstride + at);
                x.a[i][e] = ld2(key + (2 * i + 1) * kstride + at);
            }
#pragma unroll
            for (int o = 0; o < NOUT; o++) x.tab[o][e] = ld2(w.tab[o][j] + rw + at);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto weigh = [&](const Pair &tab, int o, int e, double t0, double t1, double s0, double s1) {
        const double p0 = A::from_u64(tab.x), p1 = A::from_u64(tab.y);
        u[o][0][e] += ar.mul(t0, p0);
        u[o][1][e] += ar.mul(t1, p0);
        u[o][0][e + 1] += ar.mul(s0, p1);
        u[o][1][e + 1] += ar.mul(s1, p1);
    };
    // keeps the sums of one unit ahead of the next unit's loads: the compiler would gather them all behind the last
    // load, with every unit's words in registers
    auto done = [&] {
#pragma unroll
        for (int o = 0; o < NOUT; o++)
#pragma unroll
            for (int e = 0; e < kE8; e++) asm volatile("" : "+v"(u[o][0][e]), "+v"(u[o][1][e]));
    };
    auto use = [&](const U &x, int p0) {
#pragma unroll
        for (int e = 0; e < PU; e++) {
            const bool f = x.flip[e];
            ProductSum s0, s1, r0, r1;   // both components at the even position, then at the odd one
            if constexpr (Q) {
                s0.add(A::from_u64(f ? x.c[e].y : x.c[e].x), pq);
                r0.add(A::from_u64(f ? x.c[e].x : x.c[e].y), pq);
            }
#pragma unroll
            for (int i = 0; i < ND; i++) {
                if (i && i % 3 == 0) {   // s0 and r0 hold the c0 term and three products
                    s0.fold(ar);
                    s1.fold(ar);
                    r0.fold(ar);
                    r1.fold(ar);
                }
                const double v0 = A::from_u64(f ? x.dig[i][e].y : x.dig[i][e].x),
                             v1 = A::from_u64(f ? x.dig[i][e].x : x.dig[i][e].y);
                s0.add(v0, A::from_u64(x.b[i][e].x));
                s1.add(v0, A::from_u64(x.a[i][e].x));
                r0.add(v1, A::from_u64(x.b[i][e].y));
                r1.add(v1, A::from_u64(x.a[i][e].y));
            }
            const double t0 = s0.value(ar), t1 = s1.value(ar), t2 = r0.value(ar), t3 = r1.value(ar);
#pragma unroll
            for (int o = 0; o < NOUT; o++) weigh(x.tab[o][e], o, 2 * (p0 + e), t0, t1, t2, t3);
        }
        done();
    };
#pragma unroll
    for (int o = 0; o < NOUT; o++)
#pragma unroll
        for (int e = 0; e < kE8; e++) u[o][0][e] = u[o][1][e] = 0.0;
    const uint32_t first = w.key[0] ? 0 : 1, n = w.n;
    U x0, x1;
    if (first < n) load(x0, first, 0);
    if (Q && first) {
        // the unrotated term: two pairs at a time
#pragma unroll
        for (int p0 = 0; p0 < 4; p0 += 2) {
            Pair v0[2], v1[2], tab[NOUT][2];
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const uint32_t at = ps.pos(2 * (p0 + e));
                v0[e] = ld2(c0 + at);
                v1[e] = ld2(c0 + half + at);
#pragma unroll
                for (int o = 0; o < NOUT; o++) tab[o][e] = ld2(w.tab[o][0] + rw + at);
            }
#pragma unroll
            for (int e = 0; e < 2; e++) {
                double t0 = A::from_u64(v0[e].x), t1 = A::from_u64(v1[e].x), t2 = A::from_u64(v0[e].y),
                       t3 = A::from_u64(v1[e].y);
                if (w.rotated) {
                    t0 = ar.mul(t0, pq);
                    t1 = ar.mul(t1, pq);
                    t2 = ar.mul(t2, pq);
                    t3 = ar.mul(t3, pq);
                }
#pragma unroll
                for (int o = 0; o < NOUT; o++) weigh(tab[o][e], o, 2 * (p0 + e), t0, t1, t2, t3);
            }
            done();
        }
    }
    for (uint32_t j = first; j < n; j++) {
        // two register sets in turn; the last unit's successor is the term after it
#pragma unroll
        for (int k = 0; k < kUnits; k += 2) {
            load(x1, j, (k + 1) * PU);
            use(x0, k * PU);
            if (k + 2 < kUnits) load(x0, j, (k + 2) * PU);
            else if (j + 1 < n) load(x0, j + 1, 0);
            use(x1, (k + 1) * PU);
        }
    }
}

// 1. rows q_l and P (s = 0: q_l, s > 0: p_{s-1}) of u: up[z P + o][k][s], raw doubles below 2q after the row pass.  One
// wave, two rows of 256 points, 8 positions a thread.  16 ciphertexts of 13 limbs in two digits, three terms: 122 us,
// 63% of the issue slots, 0.26 GB at 2.2 TB/s: the products, their conversions from words and the transform.
template <int ND, int NOUT>
__global__ __launch_bounds__(64) void k_wsum_intt8(Args a, uint64_t *up, Dims d, uint32_t n,
                                                   const ulonglong2 *__restrict__ pmodq, const ModQ *__restrict__ mods,
                                                   const double *__restrict__ itwf)
{
    __shared__ double tws[2][257];
    __shared__ double tr[2][nttc::kTr8];
    const uint32_t bpl = 1u << (d.log_n - 9);
    uint32_t z, tile;
    tile_of(n, z, tile);
    const uint32_t s = tile / bpl, blk = tile % bpl, row = d.L - 1 + s, prime = d.prime(row);
    const Ct &ct = a.ct[z];
    const WsumKind &w = a.kind[ct.kind];
    if (s && !w.rotated) return;
    const A ar(mods[prime]);
    const uint32_t sub = threadIdx.x >> 5, t = threadIdx.x & 31, h = blk * 2 + sub;
    nttc::stage_twiddles8(tws[sub], itwf + ((size_t)prime << d.log_n), (1u << (d.log_n - 8)) + h, t, 32);
    const Positions ps(h, t, d.log_n);
    double u[NOUT][2][kE8];
    if (s) wsum8<ND, NOUT, false>(w, ct, d, row, 0.0, ar, ps, u);
    else wsum8<ND, NOUT, true>(w, ct, d, row, (double)pmodq[row].x, ar, ps, u);
    __syncthreads();
#pragma unroll
    for (int o = 0; o < NOUT; o++)
#pragma unroll
        for (int k = 0; k < 2; k++) {
            double x[kE8];
#pragma unroll
            for (int e = 0; e < kE8; e++) x[e] = ar.red(u[o][k][e]);
            swap_1_6(x);
            nttc::inv8_256(x, tws[sub], tr[sub], t, ar);
            uint64_t *out = up + ((((size_t)(z * NOUT + o) * 2 + k) * (d.K + 1) + s) << d.log_n) + (size_t)h * 256;
#pragma unroll
            for (int e = 0; e < kE8; e++) nttc::st_stream(out + nttc::u8<0>(t, e), A::to_raw(x[e]));
        }
}

// 2. column pass of those rows, in place: centred digits as doubles
template <int LOGS>
__global__ __launch_bounds__(256) void k_quot_col(uint64_t *up, Args a, Dims d, uint32_t pages, Quot qt,
                                                  const ModQ *__restrict__ mods, const double *__restrict__ itwf)
{
    constexpr uint32_t TS = (1u << LOGS) / 16, kCols = 4096u >> LOGS, kBpr = 256 / kCols;
    __shared__ double lds[LOGS > 4 ? kCols * ((1u << LOGS) + (1u << LOGS) / 16 + 1) : 1];
    const uint32_t rr = blockIdx.x / kBpr, s = rr % (d.K + 1), p = rr / (d.K + 1);
    const bool rot = a.kind[a.ct[p / 2 / pages].kind].rotated;
    if (s && !rot) return;
    const uint32_t prime = d.prime(d.L - 1 + s);
    const A ar(mods[prime]);
    A sc = ar;
    if (s) sc.ninv = ar.scaled_twiddle(qt.qhat_inv[s - 1]);
    else if (rot) sc.ninv = ar.scaled_twiddle((double)qt.pinv[d.L - 1].x);
    const double *tw = itwf + ((size_t)prime << d.log_n);
    const uint32_t col = threadIdx.x % kCols, t = threadIdx.x / kCols;
    uint64_t *base = up + ((size_t)rr << d.log_n) + (blockIdx.x % kBpr) * kCols + col;
    double x[kE];
#pragma unroll
    for (int k = 0; k < kE; k++) x[k] = A::from_raw(base[(size_t)(LOGS > 4 ? 16 * t + k : k) * 256]);
    if (LOGS > 4) {
        nttc::inv_low<LOGS, true>(x, tw, 1, t, ar);
        nttc::transpose<LOGS, false>(x, lds, col, t);
    }
    nttc::inv_top<true, true>(x, tw, 1, sc);
#pragma unroll
    for (int k = 0; k < kE; k++) base[(size_t)(t + TS * k) * 256] = A::to_raw(centre(ar, x[k]));
}

// 3. The conversion fused with the forward column pass, N = 2^16 and at most 8 special primes (k_conv_col8's shape:
// block (poly; 16 adjacent columns; group of t_per targets), 512 threads, 8 points of a 256-point column each, the
// digits of the block's 4096 coefficients and w in registers for every target).  EXACT: K = 8.  COLS: `up` holds the
// rows after the row pass of their inverse transforms, whose column passes run here as well (step 2 is not a launch of
// its own). 32 polynomials, 8 special primes, 12 targets: 152 us, 63% of the issue slots with the two waves a SIMD that
// the digits' registers allow.
template <bool EXACT, bool COLS>
__global__ __launch_bounds__(512) void k_quot_col8(uint64_t *out, const uint64_t *up, Args a, Dims d, uint32_t pages,
                                                   uint32_t t_per, Quot qt, const ModQ *__restrict__ mods,
                                                   const double *__restrict__ twf, const double *__restrict__ itwf)
{
    __shared__ double s_mod[9 * kMaxPrimes];   // [K][targets], then [P]_t
    __shared__ double s_top[8];
    __shared__ double tws[2][256];
    __shared__ double tr[16][nttc::kTr8], trb[16][nttc::kTr8];
    __shared__ nttc::LimbConst s_tgt[kMaxPrimes];
    __shared__ nttc::InvConst s_src[9];
    constexpr uint32_t log_n = 16, n2 = 256;
    const uint32_t p = blockIdx.x >> 4, blk = blockIdx.x & 15u;
    const int K = EXACT ? 8 : (int)d.K, nt = (int)d.L - 1;
    const int t0 = (int)(blockIdx.y * t_per), t1 = min(nt, t0 + (int)t_per);
    if (t0 >= nt) return;
    const bool rot = a.kind[a.ct[p / 2 / pages].kind].rotated;
    const A top(mods[d.L - 1]);
    if (rot) {
        for (int k = threadIdx.x; k < K * nt; k += 512) s_mod[k] = qt.qhat_mod[(k / nt) * (int)d.L + k % nt];
        for (int k = threadIdx.x; k < nt; k += 512) s_mod[8 * kMaxPrimes + k] = (double)qt.pmodq[k].x;
        if (threadIdx.x < (uint32_t)K) s_top[threadIdx.x] = top_factor(qt, d, (int)threadIdx.x, top);
    }
    for (int k = threadIdx.x; k < nt; k += 512) s_tgt[k].set(A(mods[k]));
    const uint32_t col = threadIdx.x & 15, t = threadIdx.x >> 4;
    const uint32_t coff = blk * 16 + col;
    const uint64_t *src = up + ((size_t)p * (d.K + 1) << log_n) + coff;
    uint64_t *dst0 = out + ((size_t)p * nt << log_n) + coff;
    const bool stages = threadIdx.x < 255;
    const double *first = twf + ((size_t)t0 << log_n) + threadIdx.x + 1;
    double y[8][kE8], w[kE8];
    int turn = 0;   // target tt's twiddles are in half (tt - t0 + turn) & 1 of the table
    if constexpr (COLS) {
        // rows P, then q_l, each asked for while the one before is transformed
        double next[kE8];
        const int rows = rot ? K + 1 : 1;
        auto slot = [&](int i) { return rot && i < K ? i + 1 : 0; };
        // row i's twiddles, asked for two rows ahead
        auto itw = [&](int i) {
            return stages && i < rows ? itwf[((size_t)d.prime(d.L - 1 + slot(i)) << log_n) + threadIdx.x + 1] : 0.0;
        };
        if (threadIdx.x < (uint32_t)rows) {
            const int s = slot((int)threadIdx.x);
            const uint32_t prime = d.prime(d.L - 1 + s);
            const double f = s ? qt.qhat_inv[s - 1] : rot ? (double)qt.pinv[d.L - 1].x : 1.0;
            s_src[threadIdx.x].set(A(mods[prime]), f, itwf[((size_t)prime << log_n) + 1]);
        }
        if (stages) tws[0][threadIdx.x + 1] = itw(0);
        double tw1 = itw(1);
        auto ask = [&](int i) {
#pragma unroll
            for (int k = 0; k < kE8; k++)
                next[k] = A::from_raw(src[((size_t)slot(i) << log_n) + (size_t)nttc::u8<2>(t, k) * n2]);
        };
        auto column = [&](double (&x)[kE8], int i) {
            const A ar = s_src[i].m.get();
            const nttc::StageNext nx{tws[(i + 1) & 1], tw1, stages && i + 1 < rows};
#pragma unroll
            for (int k = 0; k < kE8; k++) x[k] = next[k];
            if (i + 1 < rows) ask(i + 1);
            tw1 = itw(i + 2);
            nttc::inv8_256_loop(x, tws[i & 1], tr[col], trb[col], t, ar, nttc::uniform(s_src[i].ninv),
                                nttc::uniform(s_src[i].wn), nx);
#pragma unroll
            for (int k = 0; k < kE8; k++) {
                x[k] = centre(ar, x[k]);
                asm volatile("" : "+v"(x[k]));   // here, not where it is used: the transform's words are free again
            }
        };
        ask(0);
        __syncthreads();
        if (rot) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (EXACT || i < K) column(y[i], i);
        }
        column(w, rows - 1);
        turn = rows;
        if (stages) tws[turn & 1][threadIdx.x + 1] = *first;
    } else {
        if (stages) tws[0][threadIdx.x + 1] = *first;
#pragma unroll
        for (int k = 0; k < kE8; k++) w[k] = A::from_raw(src[(size_t)nttc::u8<0>(t, k) * n2]);
        if (rot) {
#pragma unroll
            for (int i = 0; i < 8; i++)
#pragma unroll
                for (int k = 0; k < kE8; k++)
                    if (EXACT || i < K)
                        y[i][k] = A::from_raw(src[((size_t)(i + 1) << log_n) + (size_t)nttc::u8<0>(t, k) * n2]);
        }
    }
    __syncthreads();
    if (rot) {
#pragma unroll
        for (int k = 0; k < kE8; k++) {
            nttc::GridSum acc;
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (EXACT || i < K) acc.add(y[i][k], s_top[i]);
            w[k] = centre(top, w[k] - top.red(acc.value(top)));
        }
    }
    for (int tt = t0; tt < t1; tt++) {
        const A ar = s_tgt[tt].get();
        const double *tw = tws[(tt - t0 + turn) & 1];
        nttc::StageNext next{tws[(tt - t0 + turn + 1) & 1], 0.0, tt + 1 < t1 && stages};
        if (next.on) next.v = twf[((size_t)(tt + 1) << log_n) + threadIdx.x + 1];
        double x[kE8];
        if (rot) {
            const double pt = s_mod[8 * kMaxPrimes + tt];
            nttc::GridSum acc[kE8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (EXACT || i < K) {
                    const double m = s_mod[i * nt + tt];
#pragma unroll
                    for (int k = 0; k < kE8; k++) acc[k].add(y[i][k], m);
                }
#pragma unroll
            for (int k = 0; k < kE8; k++) x[k] = ar.red(acc[k].value(ar) + ar.mul(w[k], pt));
        } else {
#pragma unroll
            for (int k = 0; k < kE8; k++) x[k] = ar.red(w[k]);
        }
        nttc::fwd8_256_loop<nttc::kColMask8>(x, tw, tr[col], trb[col], t, ar, next);
        uint64_t *dst = dst0 + ((size_t)tt << log_n);
#pragma unroll
        for (int k = 0; k < kE8; k++) nttc::st_stream(dst + (size_t)nttc::u8<2>(t, k) * n2, A::to_raw(x[k]));
    }
}

// 3. The conversion alone (N < 2^16, or more than 8 special primes): thread = one coefficient, blockIdx.y a group of
// t_per targets, blockIdx.z the polynomial; canonical residues out.
template <int NS>
__global__ __launch_bounds__(256) void k_quot_conv(uint64_t *out, const uint64_t *up, Args a, Dims d, uint32_t pages,
                                                   uint32_t t_per, Quot qt, const ModQ *__restrict__ mods)
{
    __shared__ double s_mod[NS * kMaxPrimes], s_top[NS], s_p[kMaxPrimes];
    __shared__ double2 s_tq[kMaxPrimes];
    const uint32_t p = blockIdx.z;
    const int K = (int)d.K, nt = (int)d.L - 1;
    const int t0 = (int)(blockIdx.y * t_per), t1 = min(nt, t0 + (int)t_per), n = t1 - t0;
    if (t0 >= nt) return;
    const bool rot = a.kind[a.ct[p / 2 / pages].kind].rotated;
    const A top(mods[d.L - 1]);
    if (rot) {
        for (int k = threadIdx.x; k < K * n; k += 256) s_mod[k] = qt.qhat_mod[(k / n) * (int)d.L + t0 + k % n];
        if (threadIdx.x < (uint32_t)K) s_top[threadIdx.x] = top_factor(qt, d, (int)threadIdx.x, top);
    }
    for (int k = threadIdx.x; k < n; k += 256) {
        s_tq[k] = make_double2(mods[t0 + k].qd, mods[t0 + k].qinvd);
        s_p[k] = (double)qt.pmodq[t0 + k].x;
    }
    const uint32_t col = blockIdx.x * 256 + threadIdx.x;
    const uint64_t *src = up + ((size_t)p * (d.K + 1) << d.log_n) + col;
    double y[NS], w = A::from_raw(src[0]);
    if (rot) {
#pragma unroll
        for (int i = 0; i < NS; i++) y[i] = A::from_raw(src[(size_t)(min(i, K - 1) + 1) << d.log_n]);
    }
    __syncthreads();
    if (rot) {
        nttc::GridSum acc;
#pragma unroll
        for (int i = 0; i < NS; i++) {
            if (i < K) {
                acc.add(y[i], s_top[i]);
                if ((i & 7) == 7 && i + 1 < K) acc.fold(top);
            }
        }
        w = centre(top, w - top.red(acc.value(top)));
    }
    uint64_t *dst = out + ((size_t)p * nt << d.log_n) + col;
    for (int t = 0; t < n; t++) {
        A ar;
        ar.q = s_tq[t].x;
        ar.qinv = s_tq[t].y;
        double x = w;
        if (rot) {
            nttc::GridSum acc;
#pragma unroll
            for (int i = 0; i < NS; i++) {
                if (i < K) {
                    acc.add(y[i], s_mod[i * n + t]);
                    if ((i & 7) == 7 && i + 1 < K) acc.fold(ar);
                }
            }
            x = acc.value(ar) + ar.mul(w, s_p[t]);
        }
        dst[(size_t)(t0 + t) << d.log_n] = ar.to_canon(x);
    }
}

// forward stages that reduce, column output below 2 q
constexpr unsigned quot_col_mask(int logs)
{
    return logs == 6 ? 0x34 : logs == 7 ? 0x74 : 0xd4;
}

// 3. The conversion with the forward column pass for N < 2^16 or more than 8 special primes (conv_col.h): block
// (target; polynomial and tile of columns).  Every target forms w again, from the reads of its own sum.
template <int LOGS>
__global__ __launch_bounds__(256) void k_quot_col16(uint64_t *out, const uint64_t *up, Args a, Dims d, uint32_t pages,
                                                    uint32_t tiles, Quot qt, const ModQ *__restrict__ mods,
                                                    const double *__restrict__ twf)
{
    using Tile = nttc::ColTile<LOGS>;
    __shared__ double lds[Tile::kLds], s_top[kMaxPrimes];
    const uint32_t nt = d.L - 1;
    uint32_t tile, tt;
    nttc::target_of(nt, tile, tt);
    if (tile >= tiles) return;
    const uint32_t p = tile / Tile::kTiles;
    const bool rot = a.kind[a.ct[p / 2 / pages].kind].rotated;
    const A top(mods[nt]), ar(mods[tt]);
    const uint64_t *src = up + ((size_t)p * (d.K + 1) << d.log_n), *rows = src + (1u << d.log_n);
    const Tile ct(tile % Tile::kTiles);
    double w[kE], x[kE];
    if (rot) {
        if (threadIdx.x < d.K) s_top[threadIdx.x] = top_factor(qt, d, (int)threadIdx.x, top);
        __syncthreads();
        double s[2][kE];
        ct.sum(s, rows, d.log_n, d.K, {s_top, qt.qhat_mod + tt}, {1, d.L}, {top, ar});
        ct.load(w, src);
        const double pt = (double)qt.pmodq[tt].x;
#pragma unroll
        for (int k = 0; k < kE; k++)
            x[k] = ar.red(s[1][k] + ar.mul(centre(top, w[k] - top.red(s[0][k])), pt));
    } else {
        ct.load(x, src);
#pragma unroll
        for (int k = 0; k < kE; k++) x[k] = ar.red(x[k]);
    }
    ct.template forward<quot_col_mask(LOGS)>(x, out + (((size_t)p * nt + tt) << d.log_n), twf + ((size_t)tt << d.log_n), lds, ar);
}

// 4. out = (u - NTT(x)) (P q_l)^-1 (+ prev) on the rows below q_l: cw[z P + o][k][l] after the column pass.  Magnitudes
// in units of q: column-pass rows below 4.3, transformed below 2.6, u below 2.6, products below 2.5: all below 8 q =
// 2^53. 16 ciphertexts of 13 limbs: 198 us, 64% of the issue slots, 0.53 GB at 2.7 TB/s; 8 rotated and 8 unrotated
// added to their pages: 194 us, 51%, 0.61 GB at 3.2 TB/s.
template <int ND, int NOUT>
__global__ __launch_bounds__(64) void k_wsum_fin8(Args a, const uint64_t *__restrict__ cw, Dims d, uint32_t n, Quot qt,
                                                  const ModQ *__restrict__ mods, const double *__restrict__ twf)
{
    __shared__ double tws[2][257];
    __shared__ double tr[2][nttc::kTr8];
    const uint32_t bpl = 1u << (d.log_n - 9), l = d.L - 1;
    uint32_t z, tile;
    tile_of(n, z, tile);
    const uint32_t row = tile / bpl, blk = tile % bpl;
    const Ct &ct = a.ct[z];
    const WsumKind &w = a.kind[ct.kind];
    const A ar(mods[row]);
    const uint64_t q = mods[row].q;
    const uint32_t sub = threadIdx.x >> 5, t = threadIdx.x & 31, h = blk * 2 + sub;
    nttc::stage_twiddles8(tws[sub], twf + ((size_t)row << d.log_n), (1u << (d.log_n - 8)) + h, t, 32);
    const Positions ps(h, t, d.log_n);
    // an output's transform rows, both components: the first one's asked for ahead of the last sums
    double x[2][kE8];
    auto ask = [&](int o) {
        __builtin_amdgcn_sched_barrier(0);
        const uint64_t *src = cw + (((size_t)(z * NOUT + o) * 2 * l + row) << d.log_n) + (size_t)h * 256;
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int e = 0; e < kE8; e++)
                x[k][e] = A::from_raw(nttc::ld_stream(src + ((size_t)k * l << d.log_n) + nttc::u8<0>(t, e)));
        __builtin_amdgcn_sched_barrier(0);
    };
    double u[NOUT][2][kE8];
    wsum8<ND, NOUT, true>(w, ct, d, row, (double)qt.pmodq[row].x, ar, ps, u);
    // (P q_l)^-1, or q_l^-1 where u has no factor P, canonical
    double f = (double)qt.qlinv[row].x;
    if (w.rotated) {
        f = centre(ar, ar.mul(f, (double)qt.pinv[row].x));
        f = f < 0.0 ? f + ar.q : f;
    }
    __syncthreads();
#pragma unroll
    for (int o = 0; o < NOUT; o++) {
        ask(o);
        const uint64_t *prev = ct.prev[o];
        Pair pv[2][kE8 / 2];
        if (prev) {
#pragma unroll
            for (int k = 0; k < 2; k++)
#pragma unroll
                for (int e = 0; e < kE8; e += 2)
                    pv[k][e / 2] = ld2(prev + ((size_t)(k * l + row) << d.log_n) + ps.pos(e));
        }
#pragma unroll
        for (int k = 0; k < 2; k++) {
            nttc::fwd8_256<nttc::kRowMask8>(x[k], tws[sub], tr[sub], t, ar);
            swap_1_6(x[k]);
#pragma unroll
            for (int e = 0; e < kE8; e += 2) {
                Pair v;
                v.x = quotient(ar, u[o][k][e] - x[k][e], f);
                v.y = quotient(ar, u[o][k][e + 1] - x[k][e + 1], f);
                if (prev) {
                    v.x = addmod(v.x, pv[k][e / 2].x, q);
                    v.y = addmod(v.y, pv[k][e / 2].y, q);
                }
                *(Pair *)(ct.out[o] + ((size_t)(k * l + row) << d.log_n) + ps.pos(e)) = v;
            }
        }
    }
}

dim3 grid_of(const ckks_ctx *ctx, uint32_t rows, uint32_t z) { return dim3((ctx->n + kThreads - 1) / kThreads, rows, z); }

// the fp64 kernels run: in two passes, or (N = 2^12 and 2^13, blk_switch) in whole rows
bool fp64_sums(const ckks_ctx *ctx, uint32_t level)
{
    return f64_switch(ctx, level) && n_digits(ctx, level) <= 5;
}

// Words of a batch: the digits, the staging rows of the ModUps that take any, u and the converted rows.  The figure is
// what the sums in integers write; the fp64 kernels leave a part of it alone (u's rows below q_l and the staging rows
// in two passes, the converted rows in whole ones: 16 ciphertexts of 13 + 8 limbs at N = 2^16 touch 0.70 GB of 1.02).
// It is one figure for both arithmetics, since a workspace of it has to serve after ckks_ctx_set_ntt_arith as well, and
// one for all calls of as many ciphertexts, so that no later one - a moved token, a page border - makes the arena grow
// inside a graph.
struct Scratch {
    size_t dig, stage, u, x, total;
};
Scratch scratch_of(const ckks_ctx *ctx, uint32_t L, uint32_t cts, uint32_t pages)
{
    const size_t N = ctx->n, ext = L + ctx->n_p, nd = n_digits(ctx, L - 1), outs = (size_t)cts * pages;
    Scratch s{};
    s.dig = cts * nd * ext * N;
    s.stage = (size_t)cts * L * N;
    s.u = outs * 2 * ext * N;
    s.x = outs * 2 * (L - 1) * N;
    s.total = s.dig + s.stage + s.u + s.x;
    return s;
}

// The digits of the first n_rot ciphertexts, without their own rows (blk_modup writes those too).  With fp64 primes the
// ModUps read c1 where it is; else it is gathered to `stage` and taken to coefficient form there.
ckks_status modup_cts(ckks_ctx *ctx, uint32_t L, const Args &a, uint32_t n_rot, uint64_t *dig, uint64_t *stage)
{
    if (f64_switch(ctx, L - 1)) {
        static_assert(kWsumCts <= (uint32_t)kPolyList, "a batch's polynomials fit the list");
        PolySrc src{};
        for (uint32_t i = 0; i < n_rot; i++) src.list[i] = a.ct[i].c + (size_t)L * ctx->n;
        return blk_switch(ctx, L - 1) ? blk_modup(ctx, src, n_rot, L - 1, dig, stage)
                                      : up_modup(ctx, src, n_rot, L - 1, dig, false);
    }
    CK_TRY(wsum_gather_c1(ctx, a, n_rot, L, stage));
    return ks_modup_staged(ctx, stage, n_rot, L - 1, dig);
}

#define CK_ND(nd, GO)                                                                                              \
    do {                                                                                                           \
        switch (nd) {                                                                                              \
        case 1: GO(1); break;                                                                                      \
        case 2: GO(2); break;                                                                                      \
        case 3: GO(3); break;                                                                                      \
        case 4: GO(4); break;                                                                                      \
        default: GO(5); break;                                                                                     \
        }                                                                                                          \
    } while (0)

// steps 1 to 4 for n ciphertexts whose digits are formed
ckks_status two_pass_sums(ckks_ctx *ctx, const Args &a, uint32_t n, uint32_t pages, const Dims &d, uint64_t *up,
                          uint64_t *cw)
{
    const size_t N = ctx->n;
    const uint32_t level = d.L - 1, bpl = 1u << (d.log_n - 9);
    const ConvDev *cd;
    CK_TRY(ctx_conv(ctx, (int)level, -1, &cd));
    const Quot qt{cd->d_qhat_inv_f, cd->d_qhat_mod_f, ctx->d_pinv, ctx->d_qlinv + (size_t)level * ctx->n_q, ctx->d_pmodq};
    // products of a row position: the digits' and the weights'
    const double prods = 2.0 * 2 * d.nd + 2.0 * 3 * pages;
    const double rows1 = (double)n * (d.K + 1) * N;
    prof_begin(ctx, K_KEYIP, 8.0 * rows1 * (d.nd + 2.0 * pages), rows1 * (prods * 7.0 + 2 * pages * 4 * kOpsButterflyF64));
#define CK_GO(ND)                                                                                                  \
    do {                                                                                                           \
        const dim3 grid((d.K + 1) * bpl * n);                                                                      \
        if (pages == 1)                                                                                            \
            hipLaunchKernelGGL((k_wsum_intt8<ND, 1>), grid, dim3(64), 0, ctx->stream, a, up, d, n,                 \
                               ctx->d_pmodq, ctx->d_mod, ctx->d_itwf);                                             \
        else                                                                                                       \
            hipLaunchKernelGGL((k_wsum_intt8<ND, 2>), grid, dim3(64), 0, ctx->stream, a, up, d, n,                 \
                               ctx->d_pmodq, ctx->d_mod, ctx->d_itwf);                                             \
    } while (0)
    CK_ND(d.nd, CK_GO);
#undef CK_GO
    prof_end(ctx, K_KEYIP);
    HIP_TRY(hipGetLastError());

    CK_TRY(wsum_convert(ctx, a, n, pages, d, up, cw));

    const double rows4 = (double)n * level * N;
    prof_begin(ctx, K_MODDOWN, 8.0 * rows4 * (d.nd + 2.0 + 4.0 * pages),
               rows4 * (prods * 7.0 + 2 * pages * (4 * kOpsButterflyF64 + 14.0)));
#define CK_GO(ND)                                                                                                  \
    do {                                                                                                           \
        const dim3 grid(level * bpl * n);                                                                          \
        if (pages == 1)                                                                                            \
            hipLaunchKernelGGL((k_wsum_fin8<ND, 1>), grid, dim3(64), 0, ctx->stream, a, cw, d, n, qt,              \
                               ctx->d_mod, ctx->d_twf);                                                            \
        else                                                                                                       \
            hipLaunchKernelGGL((k_wsum_fin8<ND, 2>), grid, dim3(64), 0, ctx->stream, a, cw, d, n, qt,              \
                               ctx->d_mod, ctx->d_twf);                                                            \
    } while (0)
    CK_ND(d.nd, CK_GO);
#undef CK_GO
    prof_end(ctx, K_MODDOWN);
    HIP_TRY(hipGetLastError());
    return CKKS_OK;
}

}  // namespace

// steps 2 and 3: the rows q_l and P of u ([2 n pages][K + 1][N], after the row pass of their inverse transforms) to the
// converted rows cw ([2 n pages][l][N], after the column pass of their forward ones)
ckks_status wsum_convert(ckks_ctx *ctx, const Args &a, uint32_t n, uint32_t pages, const Dims &d, uint64_t *up,
                         uint64_t *cw)
{
    const size_t N = ctx->n;
    const uint32_t level = d.L - 1, polys = 2 * n * pages;
    const ConvDev *cd;
    CK_TRY(ctx_conv(ctx, (int)level, -1, &cd));
    const Quot qt{cd->d_qhat_inv_f, cd->d_qhat_mod_f, ctx->d_pinv, ctx->d_qlinv + (size_t)level * ctx->n_q, ctx->d_pmodq};
    const bool fused = d.log_n == 16 && d.K <= 8;
    // above half a block a CU no block's targets are split and its columns are transformed where they are converted (us
    // a call with the pass apart and along, by blocks: 13 limbs 150.4 and 160.4 (64), 251.9 and 253.7 (128), 363 and 356
    // (192), 433 and 415 (256), 812 and 783 (512); 4 limbs 73.0 and 75.6 (64), 124.3 and 119.3 (192))
    const bool cols = fused && polys * 16 > 128;
    // k_quot_col16 forms w for every target, a second sum over its reads: worth it for a quarter of what the other
    // conversions take (us a call in two launches and in one: 2^14, 5 ciphertexts of 9 limbs 97.2 and 94.5, 1280 reads;
    // 16 of them 189 and 186, 4096; 2^15, 8 of 6 limbs 137 and 132, 1280; 4 of 16 limbs 172.5 and 174.3, 7680; 8 of
    // them 293 and 311, 15360; 2^16, 4 of 10 limbs and 10 special primes 211 and 221, 11520)
    const bool col16 = !fused && conv_col_few(ctx, polys, d.K, level, kConvColReads / 4);
    const double rows2 = (double)polys * (d.K + 1) * N;
    if (!cols) {
        prof_begin(ctx, K_NTT_INV_COL, 16.0 * rows2, rows2 * kOpsButterflyF64 * (d.log_n - 8) / 2);
#define CK_COL(S)                                                                                                  \
    hipLaunchKernelGGL(k_quot_col<S>, dim3(polys * (d.K + 1) * (256 / (4096u >> S))), dim3(256), 0, ctx->stream, up, \
                       a, d, pages, qt, ctx->d_mod, ctx->d_itwf)
        switch (d.log_n) {
        case 14: CK_COL(6); break;
        case 15: CK_COL(7); break;
        default: CK_COL(8); break;
        }
#undef CK_COL
        prof_end(ctx, K_NTT_INV_COL);
        HIP_TRY(hipGetLastError());
    }

    prof_begin(ctx, K_CONV, 8.0 * N * polys * (d.K + 1.0 + level),
               (double)N * polys * level * (d.K * 4.0 + 14.0 + (fused ? kOpsButterflyF64 * 4 : 0.0)));
    if (fused) {
        // one block a CU; fewer blocks than CUs: the targets split over blockIdx.y
        const uint32_t blocks = polys * 16, groups = std::min(level, std::max(1u, 256u / blocks));
        const uint32_t t_per = (level + groups - 1) / groups;
        const dim3 grid(blocks, (level + t_per - 1) / t_per);
#define CK_QC(EXACT, COLS)                                                                                         \
    hipLaunchKernelGGL((k_quot_col8<EXACT, COLS>), grid, dim3(512), 0, ctx->stream, cw, up, a, d, pages, t_per, qt,  \
                       ctx->d_mod, ctx->d_twf, ctx->d_itwf)
        if (d.K == 8 && cols) CK_QC(true, true);
        else if (d.K == 8) CK_QC(true, false);
        else if (cols) CK_QC(false, true);
        else CK_QC(false, false);
#undef CK_QC
    } else if (col16) {
        const uint32_t tiles = polys << (d.log_n - 12);
        const dim3 grid((tiles + 7) / 8 * 8 * level);
#define CK_QC(S)                                                                                                   \
    hipLaunchKernelGGL(k_quot_col16<S>, grid, dim3(256), 0, ctx->stream, cw, up, a, d, pages, tiles, qt, ctx->d_mod, \
                       ctx->d_twf)
        switch (d.log_n) {
        case 14: CK_QC(6); break;
        case 15: CK_QC(7); break;
        default: CK_QC(8); break;
        }
#undef CK_QC
    } else {
        // groups of targets until the grid has 2048 blocks of four waves
        const uint32_t blocks = polys * (ctx->n / 256), groups = std::min(level, std::max(1u, 2048u / blocks));
        const uint32_t t_per = (level + groups - 1) / groups;
        const dim3 grid(ctx->n / 256, (level + t_per - 1) / t_per, polys);
        if (d.K <= 8)
            hipLaunchKernelGGL(k_quot_conv<8>, grid, dim3(256), 0, ctx->stream, cw, up, a, d, pages, t_per, qt, ctx->d_mod);
        else
            hipLaunchKernelGGL(k_quot_conv<16>, grid, dim3(256), 0, ctx->stream, cw, up, a, d, pages, t_per, qt, ctx->d_mod);
    }
    prof_end(ctx, K_CONV);
    HIP_TRY(hipGetLastError());
    if (!fused && !col16) CK_TRY(launch_ntt_fwd_first_pass(ctx, cw, polys, level, limb_range(0, level)));
    return CKKS_OK;
}

size_t wsum_scratch_words(const ckks_ctx *ctx, uint32_t L, uint32_t cts, uint32_t pages)
{
    return scratch_of(ctx, L, std::min(cts, kWsumCts), pages).total;
}

ckks_status wsum_run(ckks_ctx *ctx, uint32_t L, uint32_t pages, const WsumKind *kinds, const std::vector<WsumCt> &cts,
                     uint64_t *mem)
{
    const Dims d = wsum_dims(ctx, L);
    const bool fast = fp64_sums(ctx, L - 1), rows = fast && blk_switch(ctx, L - 1);
    for (size_t r0 = 0; r0 < cts.size();) {
        // a batch: rotated and unrotated ciphertexts together where the kernels take both
        Args a{};
        for (uint32_t i = 0; i < kWsumKinds; i++) a.kind[i] = kinds[i];
        const bool first = kinds[cts[r0].kind].rotated;
        uint32_t n = 0, n_rot = 0;
        for (; n < kWsumCts && r0 + n < cts.size(); n++) {
            const WsumCt &c = cts[r0 + n];
            const bool rot = kinds[c.kind].rotated;
            if (!fast && rot != first) break;
            Ct &x = a.ct[n];
            x.c = c.c;
            x.kind = c.kind;
            if (rot) x.dig = mem + (size_t)n_rot++ * d.nd * d.ext * ctx->n;
            for (uint32_t o = 0; o < pages; o++) {
                x.out[o] = c.out[o];
                x.prev[o] = c.prev[o];
            }
        }
        const Scratch s = scratch_of(ctx, L, n, pages);
        uint64_t *stage = mem + s.dig, *u = stage + s.stage, *x = u + s.u;
        if (n_rot) CK_TRY(modup_cts(ctx, L, a, n_rot, mem, stage));
        if (rows)
            CK_TRY(wsum_blk_sums(ctx, a, n, pages, d, u));
        else if (fast)
            CK_TRY(two_pass_sums(ctx, a, n, pages, d, u, x));
        else
            CK_TRY(wsum_exact_sums(ctx, a, n, pages, d, first, u, x));
        r0 += n;
    }
    return CKKS_OK;
}

// Weighted sums of rotations of a ciphertext, divided by P q_l (wsum.hip).
#pragma once
#include <vector>

#include "ckks_internal.h"

constexpr uint32_t kWsumTerms = 3;   // weighted terms of an output: the slot itself and its pair on either side
constexpr uint32_t kWsumPages = 2;   // outputs of one ciphertext: the same rotations, other weights
constexpr uint32_t kWsumKinds = 2;   // ways of weighting in one call: keys and values
constexpr uint32_t kWsumCts = 16;    // ciphertexts a batch

// One way of weighting: term j reads through the automorphism g[j] with key[j] (null: the unrotated term) and, for
// output o, the table tab[o][j] ([level+1+n_p][N], plaintexts over Q_level u P).  rotated: any key is set; without one
// the kind has one term.
struct WsumKind {
    uint32_t n;
    uint32_t rotated;
    uint32_t g[kWsumTerms];
    const uint64_t *key[kWsumTerms];
    const uint64_t *tab[kWsumPages][kWsumTerms];
};
// A ciphertext c ([2][level+1][N]) and its outputs out[o] ([2][level][N]), prev[o] ([2][level][N]; null: nothing)
// added; prev[o] may be out[o], no output overlaps another or a ciphertext.
struct WsumCt {
    const uint64_t *c;
    uint32_t kind;
    uint64_t *out[kWsumPages];
    const uint64_t *prev[kWsumPages];
};

// words of scratch for `cts` ciphertexts of L limbs with `pages` outputs each
size_t wsum_scratch_words(const ckks_ctx *ctx, uint32_t L, uint32_t cts, uint32_t pages);
// every ciphertext's outputs; mem: the words above.  Ciphertexts of rotated kinds come first.
ckks_status wsum_run(ckks_ctx *ctx, uint32_t L, uint32_t pages, const WsumKind *kinds, const std::vector<WsumCt> &cts,
                     uint64_t *mem);

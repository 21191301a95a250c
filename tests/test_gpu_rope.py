"""Rotary positions on ciphertexts and the encrypted key/value cache on the GPU.

Tables, rotations and appends agree bit for bit with the same sums put together from the oracle's stages, in every ring
size, either arithmetic, both layouts and pairings; cosines and sines agree with a 50-digit evaluation; decrypted
results agree with the plain rotation; a run of them (chunks of a prompt, single tokens, a fork, scores over the
cached pages) agrees with plain attention.  Refused calls leave their outputs as they were.
"""
import decimal
import math

import numpy as np
import pytest

from gpu_common import require_gpu, say, to_dev, to_host
from oracle import Ckks
from rope_common import (encode_ext, pack, plain_rope, random_cts, random_keys, slot_vectors, term_steps, weighted)
from workloads import attention_steps, gaussian_error, rng, ternary_secret, uniform_residues

pytestmark = pytest.mark.gpu

_RINGS = {}


def ring(log_n, n_q, n_p, dnum, bits):
    """(context, oracle) of a ring; bits 0: a 60-bit first prime and special primes around 45-bit ones."""
    require_gpu()
    from paper_2609_12378_amd import Context
    key = (log_n, n_q, n_p, dnum, bits)
    if key not in _RINGS:
        _RINGS.clear()
        if bits:
            ctx = Context(log_n, n_q, n_p, dnum, q_bits=bits, p_bits=60 if bits == 59 else bits)
        else:
            from oracle.ckks import gen_primes
            wide, narrow = gen_primes(60, 2 << log_n, 1 + n_p), gen_primes(45, 2 << log_n, n_q - 1)
            ctx = Context(log_n, n_q, n_p, dnum, q=[wide[0]] + list(narrow), p=list(wide[1:]))
        _RINGS[key] = ctx, Ckks(log_n, ctx.q, ctx.p, dnum)
    return _RINGS[key]


def bufs(arrays, scale=2.0 ** 40):
    from paper_2609_12378_amd import Buf
    return [Buf(to_dev(a), scale) for a in arrays]


def dev_keys(keys):
    return {s: to_dev(k) for s, k in keys.items()}


def angles(count, half, seed):
    a = rng(seed, 1).uniform(-40, 40, (count, max(1, half)))[:, :half]
    return np.cos(a), np.sin(a)


def same(got, want, what):
    bad = np.argwhere(to_host(got) != want)
    assert bad.size == 0, "%s: %d residues differ, first at %s" % (what, len(bad), bad[:4].tolist())


# ---- cosines and sines ------------------------------------------------------------------------------------------

def test_cos_sin_of_near_and_far_positions():
    """Against the exact angle reduced with 60 digits.  sincos is within 2 units in the last place (2^-52 of 1) of each
    of its two angles' values, the two products and their sum round three times by 2^-53 at most: 8 2^-53 covers it;
    the factor rounds once more, relatively."""
    import torch
    ctx, _ = ring(12, 4, 2, 2, 36)
    pos = np.array([0, 1, -1, 2, 127, 128, 131071, 10 ** 6 + 1, 2 ** 31 + 7, 2 ** 40 + 12345, 2 ** 53 - 1], dtype=np.int64)
    freq = np.array([1.0, 0.7310585786300049, 1e-3 / 3, 500000.0 ** -0.984375, 1e-300, 0.0])
    decimal.getcontext().prec = 80
    tau = 2 * decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803")
    for factor in (1.0, 1.3862943611198906):
        c, s = ctx.rope_cos_sin(to_dev(pos), to_dev(freq), factor)
        c, s = to_host(c), to_host(s)
        assert c.shape == (len(pos), len(freq))
        for i, p in enumerate(pos):
            for k, f in enumerate(freq):
                r = float((decimal.Decimal(int(p)) * decimal.Decimal(float(f))) % tau)
                tol = 8 * 2.0 ** -53 * factor + 2.0 ** -52 * 2 * math.pi * factor   # r itself is rounded, below 2 pi
                assert abs(c[i, k] - factor * math.cos(r)) <= tol, (p, f, c[i, k])
                assert abs(s[i, k] - factor * math.sin(r)) <= tol, (p, f, s[i, k])
    empty = ctx.rope_cos_sin(torch.empty(0, dtype=torch.int64, device="cuda"), to_dev(freq))
    assert empty[0].shape == (0, len(freq))


# ---- tables -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("log_n,n_q,n_p,dnum,bits,limbs,tokens,hd,rot,layout,pairing,first,count", [
    (4, 3, 1, 2, 36, 3, 1, 8, 8, "tm", "half", 0, 1),
    (5, 3, 1, 2, 36, 2, 4, 3, 2, "fm", "interleaved", 1, 2),
    (10, 4, 2, 2, 50, 4, 16, 32, 32, "tm", "half", 0, 16),
    (12, 4, 2, 2, 36, 4, 16, 128, 128, "tm", "half", 3, 1),
    (12, 4, 2, 2, 36, 3, 16, 48, 26, "fm", "half", 0, 16),
    (13, 4, 2, 2, 59, 4, 32, 20, 14, "tm", "interleaved", 31, 1),
    (14, 6, 2, 3, 0, 5, 64, 128, 96, "tm", "half", 5, 40),
    (16, 3, 2, 2, 50, 2, 128, 128, 128, "tm", "interleaved", 0, 128),
    (12, 4, 2, 2, 36, 4, 2048, 1, 0, "tm", "half", 0, 0),
])
def test_tables_are_the_encoded_cosines(log_n, n_q, n_p, dnum, bits, limbs, tokens, hd, rot, layout, pairing, first, count):
    import torch
    ctx, ck = ring(log_n, n_q, n_p, dnum, bits)
    if not rot:    # no features to turn: refused for rope, and a table of no tokens is all zero
        with pytest.raises(Exception, match="no features"):
            ctx.rope_tables(torch.empty((0, 0), dtype=torch.float64, device="cuda"),
                            torch.empty((0, 0), dtype=torch.float64, device="cuda"), tokens, hd, rot, limbs)
        t = ctx.rope_tables(torch.empty((0, 1), dtype=torch.float64, device="cuda"),
                            torch.empty((0, 1), dtype=torch.float64, device="cuda"), 1024, 2, 2, limbs)
        assert not to_host(t).any()
        return
    cos, sin = angles(count, rot // 2, 3)
    got = ctx.rope_tables(to_dev(cos), to_dev(sin), tokens, hd, rot, limbs, first=first, layout=layout, pairing=pairing)
    want = [encode_ext(ck, z, limbs)
            for z in slot_vectors(ck.n, tokens, hd, rot, first, count, cos, sin, layout, pairing)]
    same(got, np.stack(want), "tables")


@pytest.mark.parametrize("length,count,rot", [(0, 16, 64), (7, 1, 64), (13, 7, 20), (31, 2, 0), (48, 3, 0)])
def test_cache_tables_split_at_the_page(length, count, rot):
    ctx, ck = ring(12, 4, 2, 2, 36)
    T, hd, limbs = 16, 64, 3
    cos, sin = angles(count, rot // 2, 4)
    got = to_host(ctx.cache_tables(to_dev(cos) if rot else None, to_dev(sin) if rot else None, T, hd, rot, length, count,
                                   limbs))
    off = length % T
    n0 = min(count, T - off)
    for b, (first, at, n) in enumerate([(off, 0, n0)] + ([(0, n0, count - n0)] if count > n0 else [])):
        want = []
        if rot:
            want = slot_vectors(ck.n, T, hd, rot, first, n, cos[at:at + n], sin[at:at + n], "tm", "half")
        ones = np.zeros((T, ck.n // 2 // T))
        ones[first:first + n] = 1.0
        same_np = np.stack([encode_ext(ck, z, limbs) for z in want + [pack(ones, "tm")]])
        assert np.array_equal(got[b], same_np), b
    assert got.shape[0] == b + 1


# ---- rope -------------------------------------------------------------------------------------------------------

ROPE = [
    # log_n n_q n_p dnum bits limbs tokens hd rot layout pairing count
    (4, 3, 1, 2, 36, 3, 1, 8, 8, "tm", "half", 2),
    (5, 4, 2, 2, 50, 2, 2, 8, 6, "tm", "interleaved", 1),
    (8, 5, 2, 3, 36, 5, 8, 16, 16, "fm", "half", 3),
    (10, 4, 2, 2, 59, 4, 16, 32, 32, "tm", "half", 2),
    (12, 4, 2, 2, 36, 4, 16, 128, 128, "tm", "half", 1),
    (12, 4, 2, 2, 36, 2, 16, 64, 64, "tm", "half", 2),
    (12, 5, 1, 5, 50, 5, 16, 128, 128, "fm", "half", 2),     # the pairs half the slots away: both rotations are one
    (12, 6, 2, 3, 0, 6, 16, 60, 44, "tm", "interleaved", 2),
    (13, 6, 2, 3, 50, 6, 16, 128, 128, "tm", "half", 3),
    (13, 8, 3, 3, 59, 7, 32, 128, 64, "fm", "interleaved", 2),
    (14, 11, 4, 3, 50, 9, 64, 80, 60, "fm", "interleaved", 5),
    (14, 4, 1, 4, 36, 4, 64, 32, 32, "tm", "half", 19),      # more than one batch
    (15, 6, 2, 3, 50, 5, 128, 128, 128, "tm", "half", 2),
    (15, 10, 10, 1, 45, 10, 64, 256, 256, "tm", "half", 1),  # more than eight sources a conversion
    (16, 13, 8, 2, 50, 9, 128, 128, 128, "tm", "half", 2),   # a digit of one limb
    (16, 4, 2, 2, 36, 3, 128, 128, 128, "tm", "interleaved", 3),
    (16, 4, 3, 2, 59, 4, 128, 128, 128, "tm", "half", 1),
    (16, 5, 2, 3, 0, 5, 128, 96, 96, "fm", "half", 1),
    (16, 9, 9, 1, 50, 9, 128, 128, 128, "tm", "half", 1),
]


def run_rope(case, arith=0, apart=False):
    log_n, n_q, n_p, dnum, bits, limbs, tokens, hd, rot, layout, pairing, count = case
    ctx, ck = ring(log_n, n_q, n_p, dnum, bits)
    steps = term_steps(ck.n, tokens, rot, layout, pairing)
    keys = random_keys(ck, steps, 11)
    cts = random_cts(ck, limbs, count, 12)
    cos, sin = angles(tokens, rot // 2, 13)
    tables = ctx.rope_tables(to_dev(cos), to_dev(sin), tokens, hd, rot, limbs, layout=layout, pairing=pairing)
    tabs = to_host(tables)
    assert sorted(keys) == ctx.rope_steps(ck.n // 2, tokens, rot, layout, pairing)
    if apart:
        gc = bufs(cts)
    else:
        from paper_2609_12378_amd import Buf
        whole = to_dev(np.stack(cts))
        gc = [Buf(whole[i], 2.0 ** 40) for i in range(count)]
    ctx.set_ntt_arith(arith)
    try:
        got = ctx.rope(gc, tables, tokens, hd, rot, dev_keys(keys), layout=layout, pairing=pairing)
    finally:
        ctx.set_ntt_arith(0)
    for i in sorted({0, count // 2, count - 1}):
        assert got[i].scale == 2.0 ** 40 and got[i].n_limbs == limbs - 1
        same(got[i].data, weighted(ck, cts[i], steps, keys, tabs), "ciphertext %d" % i)
    same(gc[0].data, cts[0], "the input")


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "n%d-%d+%d-d%d-b%d-l%d-t%d-h%d-r%d-%s-%s-x%d" % c)
def test_rope_matches_the_oracle(case):
    run_rope(case)


@pytest.mark.parametrize("case", [ROPE[4], ROPE[8], ROPE[10], ROPE[15]], ids=lambda c: "n%d" % c[0])
def test_rope_in_integer_arithmetic(case):
    run_rope(case, arith=1)


@pytest.mark.parametrize("case", [ROPE[5], ROPE[9], ROPE[11], ROPE[15]], ids=lambda c: "n%d" % c[0])
def test_rope_of_separate_ciphertexts(case):
    run_rope(case, apart=True)


# ---- append -----------------------------------------------------------------------------------------------------

APPEND = [
    # log_n n_q n_p dnum bits limbs tokens hd rot pairing heads length count src fork
    (4, 3, 1, 2, 36, 3, 2, 4, 4, "half", 1, 0, 2, 0, False),
    (5, 4, 2, 2, 50, 2, 4, 4, 2, "interleaved", 2, 5, 3, 1, True),
    (9, 4, 2, 2, 59, 3, 8, 32, 32, "half", 1, 3, 8, 0, False),
    (12, 4, 2, 2, 36, 4, 16, 64, 64, "half", 1, 7, 1, 7, False),    # a token in its own slot
    (12, 4, 2, 2, 36, 4, 16, 64, 64, "half", 2, 7, 1, 0, True),
    (12, 4, 2, 2, 36, 3, 16, 64, 0, "half", 2, 14, 5, 3, False),    # keys without positions
    (12, 4, 2, 2, 36, 2, 16, 64, 0, "half", 3, 32, 16, 0, False),   # a whole page of them: no key switch at all
    (13, 6, 2, 3, 50, 6, 16, 128, 128, "half", 2, 45, 5, 0, True),
    (13, 6, 2, 3, 50, 6, 16, 128, 128, "half", 1, 16, 16, 0, False),  # a whole new page
    (14, 5, 2, 3, 0, 5, 64, 100, 30, "interleaved", 1, 63, 2, 62, False),
    (14, 8, 3, 3, 50, 6, 64, 128, 128, "half", 9, 100, 64, 0, False),  # 18 ciphertexts, two pages each
    (15, 5, 2, 3, 50, 4, 128, 128, 128, "half", 2, 1000, 1, 104, False),
    (16, 4, 2, 2, 50, 4, 128, 128, 128, "interleaved", 1, 333, 128, 0, False),
    (16, 4, 3, 2, 59, 3, 128, 128, 96, "interleaved", 1, 129, 20, 0, True),
]


def run_append(case, arith=0):
    log_n, n_q, n_p, dnum, bits, limbs, T, hd, rot, pairing, heads, length, count, src, fork = case
    ctx, ck = ring(log_n, n_q, n_p, dnum, bits)
    from paper_2609_12378_amd import Buf
    off, first = length % T, length // T
    shift = (off - src) % T
    steps = term_steps(ck.n, T, rot, "tm", pairing, shift)
    keys = random_keys(ck, steps, 21)
    assert sorted(keys) == ctx.append_steps(ck.n // 2, T, rot, length, src, pairing)
    k, v = random_cts(ck, limbs, heads, 22), random_cts(ck, limbs, heads, 23)
    cos, sin = angles(count, rot // 2, 24)
    tables = ctx.cache_tables(to_dev(cos) if rot else None, to_dev(sin) if rot else None, T, hd, rot, length, count, limbs,
                              pairing=pairing)
    tabs = to_host(tables)
    blocks = tabs.shape[0]
    # pages in a scrambled order, one that belongs to nobody, and every page full of other values
    n_pages = heads * (blocks + 1) + 1
    old = [random_cts(ck, limbs - 1, n_pages, 25), random_cts(ck, limbs - 1, n_pages, 26)]
    pools = [bufs(p) for p in old]
    order = [int(p) for p in rng(27, 1).permutation(n_pages)]
    table = [[999999] * first + order[h * blocks:(h + 1) * blocks] for h in range(heads)]
    forks = [order[heads * blocks + (h // 2)] for h in range(heads)] if fork else None
    if not off:
        for pool in pools:
            for p in pool:
                p.scale = 3.0                                  # a begun page's old scale does not matter
    ctx.set_ntt_arith(arith)
    try:
        ctx.cache_append(bufs(k), bufs(v), tables, T, hd, rot, length, count, dev_keys(keys), pools[0], pools[1], table,
                         src=src, pairing=pairing, fork=forks)
    finally:
        ctx.set_ntt_arith(0)
    nrot = tabs.shape[1] - 1
    touched = set()
    for h in range(heads):
        check = h in (0, heads - 1)
        for b in range(blocks):
            p = table[h][first + b]
            touched.add(p)
            if not check:
                continue
            for i, (ct, st, tab) in enumerate([(k[h], steps, tabs[b][:nrot] if nrot else tabs[b]),
                                               (v[h], steps[:1], tabs[b][nrot:])]):
                want = weighted(ck, ct, st, keys, tab)
                if b == 0 and off:
                    want = ck.ct_add(want, old[i][forks[h] if fork else p])
                same(pools[i][p].data, want, "%s of head %d, page %d" % ("kv"[i], h, b))
                assert pools[i][p].scale == 2.0 ** 40
    for i in range(2):
        for p in set(range(n_pages)) - touched:
            same(pools[i][p].data, old[i][p], "a page that is not touched")


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "n%d-%d+%d-d%d-b%d-l%d-t%d-h%d-r%d-%s-x%d-at%d-n%d-s%d-f%d" % c)
def test_append_matches_the_oracle(case):
    run_append(case)


@pytest.mark.parametrize("case", [APPEND[4], APPEND[7], APPEND[10]], ids=lambda c: "n%d" % c[0])
def test_append_in_integer_arithmetic(case):
    run_append(case, arith=1)


def test_append_of_nothing_changes_nothing():
    ctx, ck = ring(12, 4, 2, 2, 36)
    old = random_cts(ck, 3, 2, 5)
    pages = bufs(old)
    x = bufs(random_cts(ck, 4, 1, 6))
    tables = ctx.cache_tables(None, None, 16, 64, 64, 5, 0, 4)
    assert tables.shape[0] == 0
    ctx.cache_append(x, x, tables, 16, 64, 64, 5, 0, {}, pages[:1], pages[1:], [[0]])
    ctx.cache_append([], [], tables, 16, 64, 64, 5, 0, {}, pages[:1], pages[1:], [])
    assert ctx.rope([], tables, 16, 64, 64, {}) == []
    same(pages[0].data, old[0], "page")


# ---- what the ciphertexts hold ----------------------------------------------------------------------------------

class Party:
    """Encrypts, makes keys and decrypts on the attention test ring."""

    def __init__(self, log_n=13, n_q=8, n_p=3, dnum=3, seed=31):
        self.ctx, _ = ring(log_n, n_q, n_p, dnum, 50)
        self.g = rng(seed, 4)
        self.s = to_dev(ternary_secret(rng(seed, 3), self.ctx.n))
        self.scale = 2.0 ** 50

    def encrypt(self, x, limbs):
        ctx = self.ctx
        pt = ctx.encode(to_dev(np.ascontiguousarray(x).reshape(-1)), None, self.scale, limbs)
        return ctx.encrypt(self.s, pt, to_dev(uniform_residues(self.g, ctx.q[:limbs], ctx.n)),
                           to_dev(gaussian_error(self.g, ctx.n)))

    def _key(self):
        ctx = self.ctx
        return (to_dev(uniform_residues(self.g, ctx.primes, ctx.n, lead=(ctx.dnum,))),
                to_dev(gaussian_error(self.g, (ctx.dnum, ctx.n))))

    def keys(self, steps):
        return {st: self.ctx.keygen_galois(self.s, self.ctx.galois_elt(st), *self._key()) for st in steps}

    def relin(self):
        return self.ctx.keygen_relin(self.s, *self._key())

    def decrypt(self, ct):
        return to_host(self.ctx.decode(self.ctx.decrypt(self.s, ct))[0])


# The decrypted slots are off by key-switching and rescale noise: at scale 2^50 the attention tests hold sums of hundreds
# of such terms to 2^-28, and a rotation here is one of them.
SLOT_BOUND = 2.0 ** -28


@pytest.mark.parametrize("layout,pairing,hd,rot", [("tm", "half", 128, 128), ("fm", "interleaved", 128, 128),
                                                   ("tm", "interleaved", 80, 60), ("fm", "half", 256, 256)])
def test_rope_turns_the_decrypted_vectors(layout, pairing, hd, rot):
    from paper_2609_12378_amd import rope_inv_freq
    P = Party()
    ctx, T = P.ctx, 16
    D = ctx.n // 2 // T
    x = rng(32, 1).uniform(-1, 1, (T, D))
    pos = np.arange(T, dtype=np.int64) + 5000
    cos, sin = ctx.rope_cos_sin(to_dev(pos), rope_inv_freq(rot, scaling="bands", factor=8.0).cuda())
    tables = ctx.rope_tables(cos, sin, T, hd, rot, 5, layout=layout, pairing=pairing)
    keys = P.keys(ctx.rope_steps(ctx.n // 2, T, rot, layout, pairing))
    ct = P.encrypt(pack(x, layout), 5)
    y = ctx.rope([ct], tables, T, hd, rot, keys, layout=layout, pairing=pairing)[0]
    H = D // hd
    want = x.copy()
    want[:, :H * hd] = plain_rope(x[:, :H * hd].reshape(T, H, hd), to_host(cos), to_host(sin), pairing).reshape(T, -1)
    err = np.max(np.abs(P.decrypt(y) - pack(want, layout)))
    say("decrypted error %.3g" % err)
    assert err < SLOT_BOUND
    # -sin turns back: the transposed rotation
    back = ctx.rope([y], ctx.rope_tables(cos, -sin, T, hd, rot, 4, layout=layout, pairing=pairing), T, hd, rot, keys,
                    layout=layout, pairing=pairing)[0]
    assert np.max(np.abs(P.decrypt(back) - pack(x, layout))) < 2 * SLOT_BOUND


def test_a_cache_filled_in_steps_and_the_attention_that_reads_it():
    """A prompt in two chunks and single tokens (one moved to its slot), a fork of the sequence, then the rotated queries'
    scores over each cached page, against plain attention scores of rotated queries and keys."""
    from paper_2609_12378_amd import Buf, rope_inv_freq
    import torch
    P = Party(seed=33)
    ctx, T, hd, limbs = P.ctx, 16, 128, 6
    D, slots = ctx.n // 2 // T, ctx.n // 2
    g = rng(34, 1)
    total = 26                                             # tokens of the prompt and the answer
    K, V = g.uniform(-1, 1, (total, hd)), g.uniform(-1, 1, (total, hd))
    freq = rope_inv_freq(hd).cuda()

    def at(first, count):
        return ctx.rope_cos_sin(torch.arange(first, first + count, device="cuda"), freq)

    def placed(rows, src):
        z = g.uniform(-1, 1, (T, hd))                      # slots of no token hold anything
        z[src:src + len(rows)] = rows
        return P.encrypt(np.tile(z, (1, D // hd)), limbs)

    pages = [[Buf(to_dev(random_cts_like(ctx, limbs - 1, 40 + i)), 1.0) for i in range(3)] for _ in range(2)]
    table = [[2, 0]]
    length = 0
    keys = P.keys(ctx.rope_steps(slots, T, hd))
    for count, src in ((11, 0), (13, 0), (1, 8), (1, 0)):
        cos, sin = at(length, count)
        tables = ctx.cache_tables(cos, sin, T, hd, hd, length, count, limbs)
        need = P.keys(s for s in ctx.append_steps(slots, T, hd, length, src) if s not in keys)
        ctx.cache_append([placed(K[length:length + count], src)], [placed(V[length:length + count], src)], tables, T, hd,
                         hd, length, count, {**keys, **need}, pages[0], pages[1], table, src=src)
        length += count
    assert length == total
    cos, sin = (to_host(x) for x in at(0, total))
    turned = plain_rope(K[:, None], cos, sin, "half")[:, 0]
    held = np.zeros((2, 2, T, hd))
    for i, rows in enumerate((turned, V)):
        held[i].reshape(2 * T, hd)[:total] = rows
    for i in range(2):
        for b, p in enumerate(table[0]):
            got = P.decrypt(pages[i][p]).reshape(T, D // hd, hd)
            err = np.max(np.abs(got - held[i][b][:, None]))
            say("%s page %d: error %.3g" % ("kv"[i], b, err))
            assert err < 4 * SLOT_BOUND                    # up to four appends' noise a page

    # another answer to the same prompt: token 24 anew, in a forked page
    k2, v2 = g.uniform(-1, 1, (1, hd)), g.uniform(-1, 1, (1, hd))
    keep = [to_host(pages[i][0].data).copy() for i in range(2)]
    tables = ctx.cache_tables(*at(26, 1), T, hd, hd, 26, 1, limbs)
    need = P.keys(s for s in ctx.append_steps(slots, T, hd, 26, 10) if s not in keys)
    ctx.cache_append([placed(k2, 10)], [placed(v2, 10)], tables, T, hd, hd, 26, 1, {**keys, **need}, pages[0], pages[1],
                     [[2, 1]], src=10, fork=[0])
    got = P.decrypt(pages[1][1]).reshape(T, D // hd, hd)[:, 0]
    want = held[1][1].copy()
    want[10] = v2[0]
    assert np.max(np.abs(got - want)) < 5 * SLOT_BOUND
    for i in range(2):
        same(pages[i][0].data, keep[i], "the page that was forked")

    # queries of 16 tokens at positions 10 .., one limb more than the pages and rotated down to theirs
    Q = g.uniform(-1, 1, (T, D))
    qcos, qsin = at(10, T)
    rq = ctx.rope([P.encrypt(Q, limbs)], ctx.rope_tables(qcos, qsin, T, hd, hd, limbs), T, hd, hd, keys)
    akeys = P.keys(attention_steps(slots, T, hd))
    S = ctx.attention_scores(rq * 2, [pages[0][p] for p in table[0]], [0, 1], T, hd, P.relin(), akeys)
    q = plain_rope(Q.reshape(T, D // hd, hd), to_host(qcos), to_host(qsin), "half")
    for b in range(2):
        got = P.decrypt(S[b]).reshape(T, D // hd, hd)
        want = np.zeros_like(got)
        for d in range(T):
            want[:, :, d] = np.einsum("thd,td->th", q, np.roll(held[0][b], -d, axis=0))
        err = np.max(np.abs(got - want))
        say("scores of page %d: error %.3g" % (b, err))
        # 128 products: a key off by 4 and a query by 1 of 2^-28, times factors of at most sqrt 2: below 2^-18
        assert err < 2.0 ** -18


def random_cts_like(ctx, limbs, seed):
    return uniform_residues(rng(seed, 1), ctx.q[:limbs], ctx.n, lead=(2,))


# ---- refusals ---------------------------------------------------------------------------------------------------

def test_refused_calls_leave_their_outputs():
    from paper_2609_12378_amd import Buf, CkksError, Context
    import torch
    ctx, ck = ring(12, 4, 2, 2, 36)
    T, hd, n = 16, 64, ctx.n
    cos, sin = (to_dev(x) for x in angles(T, hd // 2, 51))
    tables = ctx.rope_tables(cos, sin, T, hd, hd, 4)
    keys = dev_keys(random_keys(ck, term_steps(n, T, hd, "tm", "half"), 52))
    xs, old = random_cts(ck, 4, 2, 53), random_cts(ck, 3, 4, 54)
    cts, outs = bufs(xs), bufs(old[:2])

    def refused(match, fn):
        with pytest.raises(CkksError, match=match):
            fn()

    rope = lambda c=cts, t=tables, T=T, hd=hd, r=hd, k=keys, o=outs, **kw: ctx.rope(c, t, T, hd, r, k, outs=o, **kw)  # noqa
    refused("no key for step", lambda: rope(k={}))
    refused("no key for step", lambda: rope(k={32: keys[32]}))
    refused("power of two", lambda: rope(T=15))
    refused("power of two", lambda: rope(T=0))
    refused("heads of", lambda: rope(hd=129, r=64))
    refused("odd or larger", lambda: rope(r=63))
    refused("odd or larger", lambda: rope(r=66))
    refused("no features", lambda: rope(r=0))
    refused("limbs, expected", lambda: rope(o=bufs(xs)))
    refused("limbs, expected", lambda: rope(c=[cts[0], Buf(cts[1].data[:, :3].contiguous(), 1.0)]))
    refused("two outputs overlap", lambda: rope(o=[outs[0], outs[0]]))
    flat = torch.cat([cts[0].data.reshape(-1), outs[0].data.reshape(-1)])
    a, b = flat[:2 * 4 * n].view(2, 4, n), flat[n:n + 2 * 3 * n].view(2, 3, n)
    refused("overlaps an input", lambda: rope(c=[Buf(a, 1.0)], o=[Buf(b, 1.0)]))
    one = Buf(cts[0].data[:, :1].contiguous(), 1.0)
    refused("2 to 4 limbs", lambda: ctx.rope([one], torch.zeros((3, 3, n), dtype=torch.uint64, device="cuda"), T, hd, hd, keys))
    bare = Context(12, 4, 0, 1, q_bits=36)
    refused("special primes", lambda: bare.rope_tables(cos, sin, T, hd, hd, 4))
    refused("special primes", lambda: bare.rope(cts, torch.zeros((3, 4, n), dtype=torch.uint64, device="cuda"), T, hd, hd, {}))

    pools = [bufs(old), bufs(old)]
    ct = ctx.cache_tables(cos[:5].contiguous(), sin[:5].contiguous(), T, hd, hd, 13, 5, 4)
    akeys = dev_keys(random_keys(ck, term_steps(n, T, hd, "tm", "half", 13), 55))

    def append(k=cts, v=cts, t=ct, length=13, count=5, keys=akeys, kp=pools[0], vp=pools[1], table=((0, 1), (2, 3)), **kw):
        ctx.cache_append(k, v, t, T, hd, hd, length, count, keys, kp, vp, table, **kw)

    for p in pools[0] + pools[1]:
        p.scale = cts[0].scale
    refused("no key for step", lambda: append(keys={}))
    refused("no key for step", lambda: append(src=1))
    refused("page 4 of 4", lambda: append(table=((0, 4), (2, 3))))
    refused("two outputs overlap", lambda: append(table=((0, 1), (2, 1))))
    refused("two outputs overlap", lambda: append(table=((0, 0), (2, 3))))
    refused("two outputs overlap", lambda: append(vp=pools[0]))
    refused("needs block 1", lambda: append(table=((0,), (2,))))
    refused("takes over page 9", lambda: append(fork=[9, 2]))
    refused("overlaps an input", lambda: append(fork=[2, 2]))     # head 0 continues the page that head 1 writes
    refused("overlaps an input", lambda: append(fork=[1, 2]))     # or its own second page
    refused("tokens 12 .. 17 of 16", lambda: append(src=12))
    refused("scales differ", lambda: append(k=[cts[0], Buf(cts[1].data, 2.0)]))
    pools[1][2].scale = 5.0
    refused("scale", append)
    refused("limbs, expected", lambda: append(vp=bufs(random_cts(ck, 4, 4, 56))))
    refused("tokens after", lambda: append(t=ct[:1].contiguous(), length=(1 << 32) - 1, count=1, table=((0,), (2,))))
    for i in range(2):
        same(outs[i].data, old[i], "a refused call's output")
        for p in range(4):
            same(pools[i][p].data, old[p], "a refused call's page")


# ---- streams, graphs, workspaces --------------------------------------------------------------------------------

def test_a_workspace_of_the_reported_size_and_one_too_small():
    from paper_2609_12378_amd import CkksError
    import torch
    for ring_args, T, hd, limbs in (((12, 4, 2, 2, 36), 16, 64, 4), ((14, 6, 2, 3, 50), 64, 128, 5), ((10, 4, 2, 2, 59), 8, 64, 3)):
        ctx, ck = ring(*ring_args)
        steps = term_steps(ck.n, T, hd, "tm", "half", 3)
        keys = dev_keys(random_keys(ck, steps + term_steps(ck.n, T, hd, "tm", "half"), 61))
        cos, sin = (to_dev(x) for x in angles(T, hd // 2, 62))
        part = cos[:6].contiguous(), sin[:6].contiguous()
        cts = bufs(random_cts(ck, limbs, 3, 63))
        old = random_cts(ck, limbs - 1, 6, 64)

        def ops():
            tables = ctx.rope_tables(cos, sin, T, hd, hd, limbs)
            out = ctx.rope(cts, tables, T, hd, hd, keys)
            ct = ctx.cache_tables(*part, T, hd, hd, T - 3, 6, limbs)
            pools = [bufs(old, 2.0 ** 40) for _ in range(2)]
            ctx.cache_append(cts, cts, ct, T, hd, hd, T - 3, 6, keys, pools[0], pools[1], [[0, 1], [2, 3], [4, 5]], src=T - 6)
            return [to_host(x) for x in [tables, ct] + [b.data for b in out + pools[0] + pools[1]]]

        want = ops()
        sizes = [ctx.workspace_bytes(op, shape) for op, shape in ((ctx.OP_ROPE_TABLES, ()), (ctx.OP_ROPE, (limbs, 3)),
                                                                 (ctx.OP_CACHE_APPEND, (limbs, 3)))]
        assert all(s > 0 and s % 8 == 0 for s in sizes)
        mem = torch.empty(-(-max(sizes) // 256) * 32 + 64, dtype=torch.uint64, device="cuda")
        mem.fill_(7)
        ctx.set_workspace(mem[:max(sizes) // 8])
        got = ops()
        assert all(np.array_equal(a, b) for a, b in zip(got, want))
        assert bool((mem[max(sizes) // 8:] == 7).all())
        tables = torch.from_numpy(want[0]).cuda()
        ctx.set_workspace(mem[:sizes[1] // 8 - 32])
        out = bufs(old[:3])
        with pytest.raises(CkksError, match="too small"):
            ctx.rope(cts, tables, T, hd, hd, keys, outs=out)
        same(out[0].data, old[0], "output of a refused call")
        ctx.set_workspace(None)
    for op, shape in ((ctx.OP_ROPE, (1, 1)), (ctx.OP_ROPE, (99, 1)), (ctx.OP_ROPE, (3, 0)), (ctx.OP_CACHE_APPEND, (3, 0))):
        with pytest.raises(CkksError):
            ctx.workspace_bytes(op, shape)


@pytest.mark.parametrize("ring_args,T,hd,limbs", [((12, 4, 2, 2, 36), 16, 64, 4), ((14, 6, 2, 3, 50), 64, 128, 5),
                                                  ((13, 4, 2, 2, 59), 16, 64, 3)])
def test_captured_calls_replay(ring_args, T, hd, limbs):
    """A decoding step (tables from device positions, keys and values appended, the queries rotated) captured once on the
    context's own stream and replayed with other positions and ciphertexts in the same buffers."""
    import torch
    from paper_2609_12378_amd import Buf, Context, rope_inv_freq
    eager, ck = ring(*ring_args)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = Context(ck.log_n, ck.n_q, ck.n_p, ck.dnum, q=eager.q, p=eager.p, stream=stream)
    length = T + 3
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half", 3) + term_steps(ck.n, T, hd, "tm", "half"), 71))
    freq = rope_inv_freq(hd).cuda()
    pos = torch.zeros(1, dtype=torch.int64, device="cuda")
    qpos = torch.arange(T, device="cuda")
    x = [Buf(torch.zeros((2, limbs, ck.n), dtype=torch.uint64, device="cuda"), 2.0 ** 40) for _ in range(3)]
    old = random_cts(ck, limbs - 1, 3, 72)
    pools = [bufs(old) for _ in range(2)]

    def step(c, pools):
        cos, sin = c.rope_cos_sin(pos, freq)
        t = c.cache_tables(cos, sin, T, hd, hd, length, 1, limbs)
        c.cache_append(x[:1], x[1:2], t, T, hd, hd, length, 1, keys, pools[0], pools[1], [[0, 1]], fork=[2])
        qt = c.rope_tables(*c.rope_cos_sin(qpos, freq), T, hd, hd, limbs)
        return c.rope(x[2:], qt, T, hd, hd, keys)[0].data

    torch.cuda.synchronize()
    ws = torch.empty(max(ctx.workspace_bytes(ctx.OP_ROPE_TABLES), ctx.workspace_bytes(ctx.OP_ROPE, (limbs, 1)),
                         ctx.workspace_bytes(ctx.OP_CACHE_APPEND, (limbs, 1))) // 8, dtype=torch.uint64, device="cuda")
    ctx.set_workspace(ws)
    with torch.cuda.stream(stream):
        step(ctx, pools)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = step(ctx, pools)
    torch.cuda.synchronize()
    for r in range(4):
        fresh = random_cts(ck, limbs, 3, 80 + r)
        pos.fill_(length + 17 * r)
        qpos.add_(r)
        for b, a in zip(x, fresh):
            b.data.copy_(to_dev(a))
        torch.cuda.synchronize()
        epools = [bufs(old) for _ in range(2)]
        want = step(eager, epools)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same(out, to_host(want), "replay %d: queries" % r)
        for i in range(2):
            same(pools[i][1].data, to_host(epools[i][1].data), "replay %d: page" % r)
        junk = [torch.randn(1 << 20, device="cuda") for _ in range(4)]      # the program's own work between replays
        del junk
    del graph


def test_a_context_on_its_own_stream():
    """Inputs made on the default stream, the call on the context's; tensors dropped right after the call stay whole
    until it has run."""
    import torch
    from paper_2609_12378_amd import Context
    eager, ck = ring(14, 6, 2, 3, 50)
    T, hd, limbs = 64, 128, 6
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half"), 91))
    cos, sin = (to_dev(x) for x in angles(T, hd // 2, 92))
    tables = eager.rope_tables(cos, sin, T, hd, hd, limbs)
    xs = random_cts(ck, limbs, 4, 93)
    want = [to_host(b.data) for b in eager.rope(bufs(xs), tables, T, hd, hd, keys)]
    stream = torch.cuda.Stream()
    ctx = Context(ck.log_n, ck.n_q, ck.n_p, ck.dnum, q=eager.q, p=eager.p, stream=stream)
    for _ in range(3):
        cts = bufs(xs)
        torch.cuda.synchronize()
        got = ctx.rope(cts, tables, T, hd, hd, keys)
        del cts
        scrap = [torch.full((2, limbs, ck.n), 1, dtype=torch.int64, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            same(g.data, w, "rope on another stream")
        del scrap

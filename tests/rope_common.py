"""What the rotary-position and cache tests share: the operators put together from the oracle's stages (ModUp, key inner
product, ModDown, rescale), the tables from its encode, and the plain rotation of real vectors."""
import numpy as np

from workloads import rng, uniform_residues


def plain_rope(x, cos, sin, pairing):
    """x [T][H][hd], cos and sin [T][r/2]: each head's first r features turned, the others left."""
    y = x.copy()
    r = 2 * cos.shape[1]
    lo, hi = (slice(0, r // 2), slice(r // 2, r)) if pairing == "half" else (slice(0, r, 2), slice(1, r, 2))
    c, s = cos[:, None], sin[:, None]
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., hi] * c + x[..., lo] * s
    return y


def pack(x, layout):
    """[T][D] to slots."""
    return (x if layout == "tm" else x.T).reshape(-1)


def slot_vectors(n, tokens, head_dim, rot_dim, first, count, cos, sin, layout, pairing):
    """The three tables' slot vectors, each found by what it has to do to unit vectors' pairs."""
    D = n // 2 // tokens
    t = np.zeros((3, tokens, D))
    for i in range(count):
        for f in range(D):
            d = f % head_dim
            at = t[:, first + i, f]
            if f >= D // head_dim * head_dim or d >= rot_dim:
                at[0] = 1.0
                continue
            k, upper = (d % (rot_dim // 2), d >= rot_dim // 2) if pairing == "half" else (d // 2, d % 2 == 1)
            at[0] = cos[i, k]
            at[2 if upper else 1] = sin[i, k] if upper else -sin[i, k]
    return [pack(v, layout) for v in t]


def encode_ext(ck, z, limbs):
    """A slot vector at the scale of the top prime over q_0 .. q_{limbs-1} and the special primes."""
    idx = ck.ext_primes(limbs - 1)
    return ck.ntt(ck.reduce_int(ck.encode_int(z, None, float(ck.q[limbs - 1])), idx), idx)


def weighted(ck, ct, steps, keys, tables):
    """Rescale(ModDown(sum_j pt_j t_j)) of one ciphertext [2][limbs][N]; steps[j] the left rotation of term j."""
    level = ck.level_of(ct)
    ext, ql = ck.ext_primes(level), ck.level_primes(level)
    pq = [ck.P % ck.q[i] for i in ql]
    u = [np.zeros((len(ext), ck.n), dtype=np.uint64) for _ in range(2)]
    digits = ck.modup(ct[1], level)
    for step, tab in zip(steps, tables):
        step %= ck.n // 2
        if step:
            g = ck.galois_elt(step)
            t = ck.key_inner(digits, keys[step], level, g)
            c0 = ck.mul_scalar(ck.automorph(ct[0], g), pq, ql)
            t[0][:level + 1] = ck.add(t[0][:level + 1], c0, ql)
        else:
            t = [np.zeros_like(u[0]) for _ in range(2)]
            for k in range(2):
                t[k][:level + 1] = ck.mul_scalar(ct[k], pq, ql)
        for k in range(2):
            u[k] = ck.add(u[k], ck.mul(t[k], tab, ext), ext)
    return ck.rescale(np.stack([ck.moddown(x, level) for x in u]))


def term_steps(n, tokens, rot_dim, layout, pairing, shift=0):
    h = (rot_dim // 2 if pairing == "half" else 1) * (tokens if layout == "fm" else 1)
    base = -shift * (n // 2 // tokens)
    return [base, base + h, base - h] if rot_dim else [base]


def random_keys(ck, steps, seed):
    """Uniform words in place of switching keys: the operators' integers do not ask what a key encrypts."""
    g = rng(seed, 5)
    return {s: uniform_residues(g, ck.primes, ck.n, lead=(ck.dnum, 2)) for s in sorted({s % (ck.n // 2) for s in steps}) if s}


def random_cts(ck, limbs, count, seed):
    g = rng(seed, 1)
    return [uniform_residues(g, ck.q[:limbs], ck.n, lead=(2,)) for _ in range(count)]

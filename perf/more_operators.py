"""What lies between the projections of a transformer block, on ciphertexts: polynomials (activations), norms and the
projection's epilogue, as cases that can be timed and compared.

All three are made of one step at level l (L = l + 1 limbs), of ciphertexts a, b, z, small integers m and integers k:

    (d0, d1, d2) = m sum_j (a0 b0, a0 b1 + a1 b0, a1 b1)_j + sum_i k_i (z0, z1, 0)_i
    out          = Rescale((d0, d1) + ModDown(sum_d ModUp(d2)_d rlk_d)) + c        (one limb fewer)

k = round(value * scales), c = round(value * out scale).  With t = (2 x - lo - hi) / (hi - lo):

* ``poly``     sum_i c_i T_i(t), Chebyshev polynomials, D + 1 levels for a degree below 2^D;
* ``norm``     w x f(mean x^2) + r residual, f the inverse square root: a polynomial and Newton steps, the mean by
               rotations; w plaintexts (norm weights) or ciphertexts (a gate);
* ``project``  gate act(X W + bias) + r residual, the packed projection with its epilogue.

Residues (ciphertexts, switching keys) are uniform modulo their primes, as real ones are.  The outputs are residues:
whole numbers, equal bit for bit.
"""
import ctypes
import functools
import math

import numpy as np
import torch

own = False

_TOY = dict(log_n=12, n_q=6, n_p=2, dnum=3, bits=50)      # the toy attention block's ring
_N14 = dict(log_n=14, n_q=11, n_p=4, dnum=3, bits=50)
_N16 = dict(log_n=16, n_q=24, n_p=8, dnum=3, bits=50)     # the projections' and the key switch's ring
_PAPER = dict(log_n=16, n_q=37, n_p=8, dnum=5, bits=59)   # the paper's prime sizes: integer arithmetic


def listed():
    return [
        # the smallest call: a polynomial of degree 3 of one ciphertext in the toy ring; launches count
        dict(name="poly_n12_toy", kind="poly", **_TOY, limbs=4, degree=3, count=1),
        # an activation in a middle ring, an odd degree whose tree is not full, five ciphertexts
        dict(name="poly_n14", kind="poly", **_N14, limbs=9, degree=12, count=5),
        # the inverse root of one ciphertext of sums, or an exponential: one ciphertext, degree 31
        dict(name="poly_n16_one", kind="poly", **_N16, limbs=13, degree=31, count=1),
        # SiLU of eight of the gate projection's ciphertexts
        dict(name="poly_n16_silu", kind="poly", **_N16, limbs=13, degree=15, count=8),
        # the paper's prime sizes in the middle of its chain
        dict(name="poly_paper", kind="poly", **_PAPER, limbs=20, degree=7, count=2),
        # the norm of one ciphertext of the toy ring (16 tokens of 128 features), no weights
        dict(name="norm_n12_toy", kind="norm", **_TOY, limbs=6, tokens=16, layout="fm", count=1, degree=3, newton=0,
             weights="none", residual=0),
        # a token-major norm after a block: three ciphertexts, weights, one Newton step, added to the residual stream
        dict(name="norm_n14_tm", kind="norm", **_N14, limbs=11, tokens=64, layout="tm", count=3, degree=7, newton=1,
             weights="plain", residual=1),
        # a head's norm of one ciphertext, latency; the weight a ciphertext (a gate from the data)
        dict(name="norm_n16_one", kind="norm", **_N16, limbs=13, tokens=128, layout="fm", count=1, degree=7, newton=1,
             weights="cipher", residual=0),
        # 4096 features in 16 ciphertexts of 128 tokens at the top of the chain, weights and residual
        dict(name="norm_n16_block", kind="norm", **_N16, limbs=24, tokens=128, layout="fm", count=16, degree=15,
             newton=1, weights="plain", residual=1),
        # the toy projection's ring, bias and residual on the attention block's output projection
        dict(name="project_n12_toy", kind="project", log_n=12, n_q=4, n_p=2, dnum=2, bits=36, limbs=4, tokens=16,
             layout="fm", d_in=128, d_out=128, n1=16, bias=1, degree=0, gate=0, residual=1),
        # feature-major, two outputs, an activation and a gate
        dict(name="project_n14", kind="project", **_N14, limbs=9, tokens=64, layout="fm", d_in=128, d_out=256, n1=16,
             bias=0, degree=7, gate=1, residual=0),
        # token-major at N = 2^16: two ciphertexts out, bias, SiLU, gate and residual
        dict(name="project_n16_tm", kind="project", **_N16, limbs=10, tokens=128, layout="tm", d_in=256, d_out=512,
             n1=16, bias=1, degree=15, gate=1, residual=1),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], evenly over the logarithm."""
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _draw(rng):
    log_n = rng.randint(12, 16)
    bits = rng.choice([36, 45, 50, 50, 50, 59])
    n_q = rng.randint(4, 24)
    dnum = rng.randint(max(1, -(-n_q // 8)), min(5, n_q))
    ring = dict(log_n=log_n, n_q=n_q, n_p=min(8, -(-n_q // dnum)), dnum=dnum, bits=bits)
    slots = 1 << (log_n - 1)
    kind = rng.choice(["poly", "norm", "project"])
    if kind == "poly":
        degree = _spread(rng, 1, min(63, (1 << (n_q - 2)) - 1))
        need = 2 + _depth(degree)
        return dict(kind=kind, **ring, limbs=rng.randint(need, n_q), degree=degree, count=_spread(rng, 1, 8))
    layout = rng.choice(["fm", "tm"])
    if kind == "norm":
        tokens = rng.choice([t for t in (1, 8, 16, 32, 64, 128, 256) if 4 <= slots // t <= 512 or t == 1])
        newton, weights = rng.randint(0, 1), rng.choice(["none", "plain", "cipher"])
        fixed = 2 + (layout == "tm") + 2 * newton + 1          # squares, map, mask, Newton steps, the last product
        if n_q < fixed + 2:
            newton, layout, fixed = 0, "fm", 3
        degree = _spread(rng, 1, min(31, (1 << max(1, n_q - 1 - fixed)) - 1))
        need = 1 + fixed + _depth(degree)
        if need > n_q:
            return None
        return dict(kind=kind, **ring, limbs=rng.randint(need, n_q), tokens=tokens, layout=layout,
                    count=_spread(rng, 1, 16), degree=degree, newton=newton, weights=weights,
                    residual=rng.randint(0, 1))
    if layout == "tm" and bits == 59:
        layout = "fm"                                          # token-major projections take primes below 2^50
    tokens = rng.choice([t for t in (16, 32, 64, 128) if 16 <= slots // t <= 256])
    feats = slots // tokens
    degree, gate = _spread(rng, 1, 15) if rng.random() < 0.6 else 0, rng.randint(0, 1)
    need = 2 + (_depth(degree) if degree else 0) + gate
    if need > n_q:
        return None
    return dict(kind=kind, **ring, limbs=rng.randint(need, n_q), tokens=tokens, layout=layout, d_in=feats,
                d_out=feats * rng.randint(1, 2), n1=rng.choice([8, 12, 16]), bias=rng.randint(0, 1), degree=degree,
                gate=gate, residual=rng.randint(0, 1))


def draw(rng):
    every = [work(c) for c in listed()]
    most = {k: max(w[k] for w in every) for k in ("bytes", "flops")}
    while True:
        case = _draw(rng)
        if case is None:
            continue
        w = work(case)
        # integers of 59 bits cost the plain form three products in place of one
        if w["bytes"] <= most["bytes"] and w["flops"] * (3 if case["bits"] == 59 else 1) <= most["flops"]:
            return case


# ---- the shape of a polynomial's evaluation, of the sums of rotations ------------------------------------------------

def _depth(degree):
    """Levels of sum_i c_i T_i below that of T_1."""
    return max(1, degree.bit_length())


def _babies(degree):
    """Polynomials T_1 .. T_(2^b - 1) are formed, and T_(2^b), T_(2^(b+1)) ...: b of a degree below 2^D."""
    return max(1, min(3, _depth(degree) - 2))


def _split(c):
    """c of degree >= m, m the largest power of two: (q, r, m), c = q T_m + r by T_m T_i = (T_(m+i) + T_(m-i)) / 2."""
    m = 1 << ((len(c) - 1).bit_length() - 1)
    q = [c[m]] + [2 * x for x in c[m + 1:]]
    r = list(c[:m])
    for i in range(1, len(q)):
        r[m - i] -= c[m + i]
    return q, r, m


def _linear(c, b, depth):
    """Every T_i of c is a baby that is there a level above `depth`."""
    d = len(c) - 1
    return d < 1 << b and (d - 1).bit_length() <= depth - 1


def _rounds(count):
    """Radixes, at most 16 and as even as they go, whose product is `count` (a power of two)."""
    bits, n = count.bit_length() - 1, -(-(count.bit_length() - 1) // 4)
    out = []
    for i in range(n):
        out.append(-(-(bits - sum(out)) // (n - i)))
    return [1 << x for x in out]


def _sum_steps(case, sign=1):
    """Rotation steps of each round of the sum over a ciphertext's features."""
    slots = 1 << (case["log_n"] - 1)
    at, got = case["tokens"] if case["layout"] == "fm" else 1, []
    for radix in _rounds(slots // case["tokens"]):
        got.append([sign * k * at for k in range(1, radix)])
        at *= radix
    return got


def _project_steps(case):
    """(baby steps of the weights, those of the wrapped ones in the token-major layout, giant steps)."""
    D, n1 = (1 << (case["log_n"] - 1)) // case["tokens"], min(case["n1"], (1 << (case["log_n"] - 1)) // case["tokens"])
    t = case["tokens"] if case["layout"] == "fm" else 1
    wrapped = [b - D for b in range(n1)] if case["layout"] == "tm" else []
    return [t * b for b in range(n1)], wrapped, [t * n1 * g for g in range(-(-D // n1))]


def _steps(case):
    if case["kind"] == "poly":
        return []
    if case["kind"] == "norm":
        rounds = _sum_steps(case) + (_sum_steps(case, -1) if case["layout"] == "tm" else [])
        return sorted({s for r in rounds for s in r})
    return sorted({s for part in _project_steps(case) for s in part if s})


# ---- the ring -------------------------------------------------------------------------------------------------------

def _is_prime(n):
    if n % 2 == 0:
        return n == 2
    d, s = n - 1, 0
    while d % 2 == 0:
        d, s = d // 2, s + 1
    for a in (2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37):
        x = pow(a, d, n)
        if a % n == 0 or x in (1, n - 1):
            continue
        for _ in range(s - 1):
            x = x * x % n
            if x == n - 1:
                break
        else:
            return False
    return True


@functools.lru_cache(maxsize=64)
def _primes(log_n, n_q, n_p, bits):
    """The largest primes below 2^bits that are 1 modulo 2N: n_q of the chain, then n_p special ones (of 60 bits over a
    59-bit chain)."""
    two_n, got = 2 << log_n, []
    for width, count in ((bits, n_q), (60 if bits == 59 else bits, n_p)):
        c, have = ((1 << width) - 1) // two_n * two_n + 1, 0
        c -= two_n if c >= 1 << width else 0
        while have < count:
            if c not in got and _is_prime(c):
                got.append(c)
                have += 1
            c -= two_n
    return tuple(got)


@functools.lru_cache(maxsize=256)
def _psi(q, n):
    """x^((q-1)/2N) of the smallest x >= 2 for which it is a primitive 2N-th root of unity."""
    return next(r for r in (pow(x, (q - 1) // (2 * n), q) for x in range(2, 1 << 20)) if pow(r, n, q) == q - 1)


def _brev(log_n, device="cpu"):
    r = torch.zeros(1, dtype=torch.int64, device=device)
    for _ in range(log_n):
        r = torch.cat([2 * r, 2 * r + 1])
    return r


def _mul(a, b, q):
    """a b mod q of residues in int64 (q a tensor of at most 61-bit moduli): the quotient from doubles, the remainder from
    the wrapped products.  From 2^50 the quotient has more bits than a double holds, and b is taken in two parts."""
    def part(x, y):
        c = (x.double() * y.double() / q.double()).to(torch.int64)
        return (x * y - c * q).remainder(q)

    if int(q.max()) < 1 << 50:
        return part(a, b)
    high = part(part(a, b >> 30), torch.full_like(q, 1 << 30))
    return (high + part(a, b & ((1 << 30) - 1))).remainder(q)


class _Ring:
    """The chain's tables: twiddles psi^brev(i) and their inverses, [primes][N] int64."""

    def __init__(self, log_n, n_q, n_p, dnum, bits):
        self.log_n, self.n, self.n_q, self.n_p, self.dnum = log_n, 1 << log_n, n_q, n_p, dnum
        self.alpha = -(-n_q // dnum)
        self.primes = _primes(log_n, n_q, n_p, bits)
        self.q = torch.tensor(self.primes, dtype=torch.int64, device="cuda")[:, None]
        psi = [_psi(q, self.n) for q in self.primes]
        self.brev = _brev(log_n, "cuda")
        self.tw = self._powers(psi)[:, self.brev]
        self.itw = self._powers([pow(r, -1, q) for r, q in zip(psi, self.primes)])[:, self.brev]

    def _powers(self, base):
        x = torch.ones((len(base), 1), dtype=torch.int64, device="cuda")
        for k in range(self.log_n):
            step = [pow(b, 1 << k, q) for b, q in zip(base, self.primes)]
            x = torch.cat([x, _mul(x, torch.tensor(step, device="cuda")[:, None], self.q)], 1)
        return x

    def consts(self, values):
        return torch.tensor(values, dtype=torch.int64, device="cuda")[:, None]

    def top(self, limbs):
        """The top prime of that many limbs, as a double."""
        return float(self.primes[limbs - 1])

    def ext(self, limbs):
        return list(range(limbs)) + list(range(self.n_q, self.n_q + self.n_p))

    def ntt(self, x, idx):
        """[..., len(idx), N] coefficients -> values at psi^(2 brev(j) + 1)."""
        lead, q, m = x.shape[:-1], self.q[idx][..., None], 1
        while m < self.n:
            v = x.reshape(*lead, m, 2, self.n // (2 * m))
            w = _mul(v[..., 1, :], self.tw[idx, m:2 * m, None], q)
            x = torch.stack([v[..., 0, :] + w, v[..., 0, :] - w], -2).remainder(q[..., None])
            m *= 2
        return x.reshape(*lead, self.n)

    def intt(self, x, idx):
        lead, q, m = x.shape[:-1], self.q[idx][..., None], self.n // 2
        while m:
            v = x.reshape(*lead, m, 2, self.n // (2 * m))
            s = (v[..., 0, :] + v[..., 1, :]).remainder(q)
            w = _mul((v[..., 0, :] - v[..., 1, :]).remainder(q), self.itw[idx, m:2 * m, None], q)
            x = torch.stack([s, w], -2)
            m //= 2
        return _mul(x.reshape(*lead, self.n), self.consts([pow(self.n, -1, self.primes[i]) for i in idx]), self.q[idx])

    def automorph(self, x, steps):
        g = pow(5, steps % (self.n // 2), 2 * self.n)
        e = (2 * self.brev + 1) * g % (2 * self.n)
        return x[..., self.brev[(e - 1) // 2]]

    def centred(self, x, idx):
        q = self.q[idx]
        return torch.where(x > q // 2, x - q, x)

    def convert(self, coef, src, dst):
        """Coefficients modulo the primes src -> dst: sum of the centred digits times Q / q_i, uncorrected."""
        big = math.prod(self.primes[i] for i in src)
        hat = [big // self.primes[i] for i in src]
        y = _mul(coef, self.consts([pow(h, -1, self.primes[i]) for h, i in zip(hat, src)]), self.q[src])
        y, q = self.centred(y, src), self.q[dst]
        out = 0
        for k, h in enumerate(hat):
            w = self.consts([h % self.primes[t] for t in dst])
            out = out + _mul(y[..., k:k + 1, :].remainder(q), w, q)
        return out.remainder(q)

    def modup(self, c):
        limbs = c.shape[-2]
        ext, got = self.ext(limbs), []
        for lo in range(0, limbs, self.alpha):
            own_rows = list(range(lo, min(lo + self.alpha, limbs)))
            at = [r for r in range(len(ext)) if r not in own_rows]
            to = [ext[r] for r in at]
            d = torch.empty((*c.shape[:-2], len(ext), self.n), dtype=torch.int64, device="cuda")
            d[..., own_rows, :] = c[..., own_rows, :]
            d[..., at, :] = self.ntt(self.convert(self.intt(c[..., own_rows, :], own_rows), own_rows, to), to)
            got.append(d)
        return got

    def key_sum(self, digits, key, limbs, steps=0):
        """sum_d sigma(digit_d) key_d over Q u P: [..., 2, ext, N]."""
        ext = self.ext(limbs)
        u = 0
        for d, dig in enumerate(digits):
            turned = self.automorph(dig, steps) if steps else dig
            u = u + torch.stack([_mul(turned, key[d, k, ext], self.q[ext]) for k in range(2)], -3)
        return u.remainder(self.q[ext])

    def moddown(self, u, limbs):
        low, p = list(range(limbs)), list(range(self.n_q, self.n_q + self.n_p))
        big = math.prod(self.primes[i] for i in p)
        c = self.ntt(self.convert(self.intt(u[..., limbs:, :], p), p, low), low)
        return _mul((u[..., :limbs, :] - c).remainder(self.q[low]),
                    self.consts([pow(big, -1, self.primes[i]) for i in low]), self.q[low])

    def rescale(self, v):
        limbs = v.shape[-2]
        top = self.centred(self.intt(v[..., limbs - 1:, :], [limbs - 1]), [limbs - 1])
        low, ql = list(range(limbs - 1)), self.primes[limbs - 1]
        c = self.ntt(top.expand(*top.shape[:-2], limbs - 1, self.n).remainder(self.q[low]), low)
        return _mul((v[..., :limbs - 1, :] - c).remainder(self.q[low]),
                    self.consts([pow(ql, -1, self.primes[i]) for i in low]), self.q[low])

    def rotate(self, x, steps, keys):
        """Rotations of ciphertexts x [..., 2, limbs, N] from one ModUp, one after another."""
        limbs, digits = x.shape[-2], self.modup(x[..., 1, :, :])
        for s in steps:
            v = self.moddown(self.key_sum(digits, keys[s], limbs, s), limbs)
            v[..., 0, :, :] = (v[..., 0, :, :] + self.automorph(x[..., 0, :, :], s)).remainder(self.q[:limbs])
            yield v


@functools.lru_cache(maxsize=3)
def _ring(log_n, n_q, n_p, dnum, bits):
    return _Ring(log_n, n_q, n_p, dnum, bits)


@functools.lru_cache(maxsize=3)
def _context(log_n, n_q, n_p, dnum, bits):
    from paper_2609_12378_amd import Context
    return Context(log_n, n_q, n_p, dnum, q_bits=bits, p_bits=60 if bits == 59 else bits)


def _chain(case):
    return tuple(case[k] for k in ("log_n", "n_q", "n_p", "dnum", "bits"))


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _fit(fn, degree, lo, hi):
    """Chebyshev coefficients of fn interpolated on [lo, hi] at degree + 1 nodes."""
    n = degree + 1
    at = [math.cos(math.pi * (k + 0.5) / n) for k in range(n)]
    f = [fn((hi - lo) / 2 * x + (hi + lo) / 2) for x in at]
    c = [2.0 / n * sum(f[k] * math.cos(math.pi * j * (k + 0.5) / n) for k in range(n)) for j in range(n)]
    return [c[0] / 2] + c[1:]


def _silu(x):
    return x / (1 + math.exp(-x))


@functools.lru_cache(maxsize=16)
def _slots_at(n):
    """Slot j sits at 5^j = 4 s + 1 modulo 2N."""
    at, p = np.empty(n // 2, dtype=np.int64), 1
    for j in range(n // 2):
        at[j] = (p - 1) // 4
        p = p * 5 % (2 * n)
    return at


def _encode(ring, slots, scale, limbs):
    """Real slot vectors [count][N/2] as plaintexts [count][limbs][N]."""
    n, count = ring.n, len(slots)
    y = np.zeros((count, n // 2), dtype=np.complex128)
    y[:, _slots_at(n)] = slots
    v = np.fft.fft(y, axis=1) * np.exp(-1j * np.pi * np.arange(n // 2) / n) * (scale * 2.0 / n)
    m = torch.from_numpy(np.rint(np.concatenate([v.real, v.imag], 1)).astype(np.int64)).cuda()
    idx = list(range(limbs))
    return ring.ntt(m[:, None].remainder(ring.q[idx]), idx)


def _residues(g, primes, n, *lead):
    q = torch.tensor(list(primes), dtype=torch.int64, device="cuda")
    x = torch.randint(0, 1 << 62, (*lead, len(primes), n), dtype=torch.int64, device="cuda", generator=g)
    return x.remainder_(q[:, None])


def _features(case, v):
    """A value a feature, in the case's slot order, the same for every token: [count][D] -> [count][N/2]."""
    T = case["tokens"]
    return np.repeat(v, T, axis=1) if case["layout"] == "fm" else np.tile(v, (1, T))


def _inputs(case, seed):
    """Everything a program has in hand: ciphertexts, keys, weights, coefficients; scales a little below 2^bits."""
    ring, limbs, n = _ring(*_chain(case)), case["limbs"], 1 << case["log_n"]
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    r = np.random.default_rng(int(seed))
    key = lambda: _residues(g, ring.primes, n, case["dnum"], 2)  # noqa: E731
    scale = 2.0 ** case["bits"]
    st = {"scale": scale, "rlk": key(), "keys": {s: key() for s in _steps(case)}}
    cts = lambda count, L: _residues(g, ring.primes[:L], n, count, 2)  # noqa: E731
    if case["kind"] == "poly":
        st["x"] = cts(case["count"], limbs)
        st["poly"] = (_fit(_silu, case["degree"], -8.0, 8.0), -8.0, 8.0)
        return ring, st
    D = n // 2 // case["tokens"]
    if case["kind"] == "norm":
        st["x"] = cts(case["count"], limbs)
        st["features"] = case["count"] * D
        st["poly"] = (_fit(lambda v: (v + 1e-5) ** -0.5, case["degree"], 0.05, 2.0), 0.05, 2.0)
        if case["weights"] == "plain":
            st["w"] = _encode(ring, _features(case, r.normal(1.0, 0.2, (case["count"], D))), scale, limbs)[:, None]
        elif case["weights"] == "cipher":
            st["w"] = cts(case["count"], limbs)
        if case["layout"] == "tm":
            first = np.zeros((1, D))
            first[0, 0] = 1.0
            st["mask"] = _encode(ring, _features(case, first), scale, limbs - 1)
        st["residual"] = cts(case["count"], limbs) if case["residual"] else None
        return ring, st
    n_out = case["d_out"] // D
    st["x"] = cts(case["d_in"] // D, limbs)
    st["W"] = 0.02 * torch.randn((case["d_in"], case["d_out"]), dtype=torch.float64, device="cuda", generator=g)
    if case["bias"]:
        st["bias"] = _encode(ring, _features(case, r.normal(0, 0.1, (n_out, D))), scale, limbs)
    if case["degree"]:
        st["poly"] = (_fit(_silu, case["degree"], -6.0, 10.0), -6.0, 10.0)
    st["gate"] = cts(n_out, limbs - 1) if case["gate"] else None
    st["residual"] = cts(n_out, limbs) if case["residual"] else None
    return ring, st


def prepare(case, seed):
    ring, st = _inputs(case, seed)
    st.update(case=case, ring=ring)
    if not own:
        return st
    from paper_2609_12378_amd import Buf, Epilogue, Poly
    words, scale = (lambda x: x.view(torch.uint64)), st["scale"]
    bufs = lambda x: None if x is None else [Buf(words(c), scale) for c in x]  # noqa: E731
    got = dict(case=case, ctx=_context(*_chain(case)), x=bufs(st["x"]), rlk=words(st["rlk"]),
               keys={k: words(v) for k, v in st["keys"].items()})
    poly = Poly(*st["poly"]) if "poly" in st else None
    if case["kind"] == "project":
        bias = bufs(st["bias"][:, None]) if case["bias"] else None
        got.update(W=st["W"], epilogue=Epilogue(bias=bias, act=poly, gate=bufs(st["gate"]),
                                                residual=bufs(st["residual"]), residual_scale=_RESIDUAL, rlk=got["rlk"]))
    else:
        got["poly"] = poly
    if case["kind"] == "norm":
        got.update(features=st["features"], w=bufs(st.get("w")), residual=bufs(st["residual"]),
                   mask=Buf(words(st["mask"]), scale) if "mask" in st else None)
    return got


_RESIDUAL, _EPS = 0.75, 1e-5


# ---- the operators --------------------------------------------------------------------------------------------------

def _step(ring, limbs, rlk, products=(), mult=1, terms=(), const=0):
    """The step of the heading on ciphertexts [..., 2, >= limbs, N] (terms [..., 1, ..] count for the first component)."""
    low, q = list(range(limbs)), ring.q[:limbs]
    d = [0, 0, 0]
    for a, b in products:
        a0, a1, b0, b1 = a[..., 0, low, :], a[..., 1, low, :], b[..., 0, low, :], b[..., 1, low, :]
        d = [(d[0] + _mul(a0, b0, q)).remainder(q), (d[1] + _mul(a0, b1, q) + _mul(a1, b0, q)).remainder(q),
             (d[2] + _mul(a1, b1, q)).remainder(q)]
    if products and mult != 1:
        d = [(mult * x).remainder(q) for x in d]
    for z, k in terms:
        by = ring.consts([k % p for p in ring.primes[:limbs]])
        for i in range(z.shape[-3]):
            d[i] = (d[i] + _mul(z[..., i, low, :], by, q)).remainder(q)
    v = torch.stack(torch.broadcast_tensors(d[0], d[1]), -3)
    if products:
        u = ring.key_sum(ring.modup(d[2]), rlk, limbs)
        scaled = ring.consts([math.prod(ring.primes[ring.n_q:]) % p for p in ring.primes[:limbs]])
        u[..., low, :] = (u[..., low, :] + _mul(v, scaled, q)).remainder(q)
        v = ring.moddown(u, limbs)
    out = ring.rescale(v)
    if const:
        out[..., 0, :, :] = (out[..., 0, :, :] + ring.consts([const % p for p in ring.primes[:limbs - 1]])).remainder(q[:-1])
    return out


def _map(poly, s1):
    """(2 / (hi - lo) s1, the constant's integer) of t = (2 x - lo - hi) / (hi - lo) at scale s1."""
    _, lo, hi = poly
    return 2.0 / (hi - lo) * s1, round(-(lo + hi) / (hi - lo) * s1)


def _chebyshev(ring, t1, s1, coefs, target, rlk, extra=()):
    """sum_i c_i T_i(t) at scale `target` of t1 (scale s1); extra: terms of the last step."""
    L1, b, have = t1.shape[-2], _babies(len(coefs) - 1), {1: (t1, s1)}

    def power(i):                                              # T_i = 2 T_(i - i/2) T_(i/2) - T_(i mod 2)
        if i not in have:
            (x, sx), (y, sy) = power(i - i // 2), power(i // 2)
            limbs = L1 + 1 - (i - 1).bit_length()
            s = sx * sy / ring.top(limbs)
            if i % 2:
                have[i] = _step(ring, limbs, rlk, [(x, y)], 2, [(t1, -round(sx * sy / s1))]), s
            else:
                have[i] = _step(ring, limbs, rlk, [(x, y)], 2, const=-round(s)), s
        return have[i]

    def node(c, depth, target, extra=()):
        limbs = L1 + 1 - depth
        up = target * ring.top(limbs)
        term = lambda i, k: (power(i)[0], round(k * (up / power(i)[1])))  # noqa: E731
        if _linear(c, b, depth):
            return _step(ring, limbs, rlk, terms=[term(i, c[i]) for i in range(1, len(c))] + list(extra),
                         const=round(c[0] * target))
        q, r, m = _split(c)
        terms, products, const = list(extra), [], 0
        if len(q) == 1:
            terms.append(term(m, q[0]))
        else:
            products = [(node(q, depth - 1, up / power(m)[1]), power(m)[0])]
        if m - 1 < 1 << b:
            terms += [term(i, r[i]) for i in range(1, m)]
            const = round(r[0] * target)
        else:
            terms.append((node(r, depth - 1, target), ring.primes[limbs - 1]))
        return _step(ring, limbs, rlk, products, 1, terms, const)

    return node(list(coefs), _depth(len(coefs) - 1), target, extra)


def _run_poly(st, ring):
    x, S, poly, rlk = st["x"], st["scale"], st["poly"], st["rlk"]
    L, s1 = x.shape[-2], ring.top(x.shape[-2] - 1)
    by, const = _map(poly, s1)
    t1 = _step(ring, L, rlk, terms=[(x, round(by * (ring.top(L) / S)))], const=const)
    return _chebyshev(ring, t1, s1, poly[0], S, rlk)


def _sum_rounds(ring, x, rounds, keys):
    for steps in rounds:
        limbs, digits = x.shape[-2], ring.modup(x[1])
        q, u = ring.q[:limbs], 0
        scaled = ring.consts([math.prod(ring.primes[ring.n_q:]) % p for p in ring.primes[:limbs]])
        for s in steps:
            t = ring.key_sum(digits, keys[s], limbs, s)
            t[0, :limbs] = (t[0, :limbs] + _mul(ring.automorph(x[0], s), scaled, q)).remainder(q)
            u = u + t
            u = u.remainder(ring.q[ring.ext(limbs)])
        x = (x + ring.moddown(u, limbs)).remainder(q)
    return x


def _run_norm(st, ring):
    case, x, S, rlk, keys = st["case"], st["x"], st["scale"], st["rlk"], st["keys"]
    L, d, top = x.shape[-2], float(st["features"]), ring.top
    v = _step(ring, L, rlk, [(c, c) for c in x])
    sv = S * S / top(L)
    v = _sum_rounds(ring, v, _sum_steps(case), keys)
    if case["layout"] == "tm":
        sv = sv * S / top(L - 1)
        v = ring.rescale(_mul(v, st["mask"][0][:L - 1], ring.q[:L - 1]))
        v = _sum_rounds(ring, v, _sum_steps(case, -1), keys)
    Lv = v.shape[-2]
    m0 = Lv - 1 - _depth(case["degree"])
    m = m0 - 2 * case["newton"]                                # limbs of the inverse root
    sx = S * S / top(m + 1) if "w" in st else S
    last = S * top(m) / sx
    # the mean on the polynomial's interval
    s1 = top(Lv - 1)
    by, const = _map(st["poly"], s1)
    t1 = _step(ring, Lv, rlk, terms=[(v, round(by / d * (top(Lv) / sv)))], const=const)
    sy = top(m0) if case["newton"] else last
    y = _chebyshev(ring, t1, s1, st["poly"][0], sy, rlk)
    for j in range(case["newton"]):                            # y (3 - (mean + eps) y^2) / 2
        limbs = y.shape[-2]
        to = top(limbs - 2) if j + 1 < case["newton"] else last
        qa, qb = top(limbs), top(limbs - 1)
        st_ = sy * sy / qa
        sn = to / 2 * qb / st_ * qa / sy
        mean = _step(ring, Lv, rlk, terms=[(v, round(sn / d * (top(Lv) / sv)))], const=round(_EPS * sn))
        sp = sn * sy / qa * st_ / qb
        a, b = _step(ring, limbs, rlk, [(mean, y)]), _step(ring, limbs, rlk, [(y, y)])
        y = _step(ring, limbs - 1, rlk, [(a, b)], -1, [(y, round(3.0 * (sp * qb / sy)))])
        sy = to
    if case["weights"] == "plain":
        q = ring.q[:m + 1]
        x = ring.rescale(_mul(x[..., :m + 1, :], st["w"][..., :m + 1, :], q))
    elif case["weights"] == "cipher":
        x = _step(ring, m + 1, rlk, [(x, st["w"])])
    terms = [(st["residual"], round(_RESIDUAL * (S * top(m) / S)))] if case["residual"] else []
    return _step(ring, m, rlk, [(x, y.expand(x.shape[0], *y.shape))], 1, terms)


@functools.lru_cache(maxsize=8)
def _turns(n):
    """cos and sin of 2 pi e / M (e < M / 2) and of pi k / N (k < M), M = N / 2, from the C library's sincos: the encoder's
    rounding is defined on these."""
    libm = ctypes.CDLL("libm.so.6")
    libm.sincos.argtypes, libm.sincos.restype = [ctypes.c_double] + 2 * [ctypes.POINTER(ctypes.c_double)], None
    s, c, M = ctypes.c_double(), ctypes.c_double(), n // 2

    def both(angles):
        out = np.empty((len(angles), 2))
        for i, a in enumerate(angles):
            libm.sincos(a, ctypes.byref(s), ctypes.byref(c))
            out[i] = c.value, s.value
        return out
    return (both([2.0 * math.pi * float(e) / float(M) for e in range(max(1, M // 2))]),
            both([math.pi * float(k) / float(n) for k in range(M)]))


def _coefficients(vectors, scale):
    """Integer coefficients [P][2 M] of real slot vectors [P][M] (torch float64 on the GPU): the radix-2 transform whose
    products and sums round one by one, then round half away from zero."""
    M = vectors.shape[1]
    n = 2 * M
    w, twist = (torch.from_numpy(t).cuda() for t in _turns(n))
    re = torch.empty_like(vectors)
    re[:, _brev(M.bit_length() - 1, "cuda")[torch.from_numpy(_slots_at(n)).cuda()]] = vectors
    im, half = torch.zeros_like(re), 1
    while half < M:
        e = torch.arange(half, device="cuda") * (M // (2 * half))
        wr, wi = w[e, 0], -w[e, 1]
        ar, ai = re.reshape(-1, M // (2 * half), 2, half), im.reshape(-1, M // (2 * half), 2, half)
        tr, ti = wr * ar[:, :, 1] - wi * ai[:, :, 1], wr * ai[:, :, 1] + wi * ar[:, :, 1]
        re = torch.stack([ar[:, :, 0] + tr, ar[:, :, 0] - tr], 2).reshape(-1, M)
        im = torch.stack([ai[:, :, 0] + ti, ai[:, :, 0] - ti], 2).reshape(-1, M)
        half *= 2
    c, tr, ti = scale * (2.0 / n), twist[:, 0], -twist[:, 1]
    x = torch.cat([c * (tr * re - ti * im), c * (tr * im + ti * re)], 1)
    whole = torch.trunc(x)
    return (whole + torch.where((x - whole).abs() >= 0.5, torch.sign(x), torch.zeros_like(x))).to(torch.int64)


def _weights(case, ring, W, i, j, g, n1, scale, limbs):
    """Plaintexts [baby steps][limbs][N] of giant step g, input i and output j (token-major: those that do not wrap, then
    those that do)."""
    T, n = case["tokens"], ring.n
    D = n // 2 // T
    b = torch.arange(min(n1, D - n1 * g), device="cuda")[:, None]
    o = (torch.arange(D, device="cuda") - n1 * g) % D
    vals = W[i * D + (o + n1 * g + b) % D, j * D + o]
    if case["layout"] == "fm":
        m = _coefficients(vals.repeat_interleave(T, 1), scale)
    else:
        wraps = o + n1 * g + b >= D
        zero = torch.zeros_like(vals)
        short = _coefficients(torch.cat([torch.where(wraps, zero, vals), torch.where(wraps, vals, zero)]), scale)
        m = torch.zeros((len(short), n), dtype=torch.int64, device="cuda")
        m[:, ::n // (2 * D)] = short
    idx = list(range(limbs))
    return ring.ntt(m[:, None].remainder(ring.q[idx]), idx)


def _run_project(st, ring):
    case, x, S, rlk, keys, W = st["case"], st["x"], st["scale"], st["rlk"], st["keys"], st["W"]
    L, top, q = x.shape[-2], ring.top, ring.q[:x.shape[-2]]
    D = ring.n // 2 // case["tokens"]
    baby, wrapped, giant = _project_steps(case)
    n1, n_out = len(baby), case["d_out"] // D
    # scales: of the projection's rescaled sums, then of what the gate multiplies
    m = L - 1 - (_depth(case["degree"]) if case["degree"] else 0)
    before_gate = S * top(m) / S if case["gate"] else S
    if case["degree"]:
        s1 = top(L - 1)
        by, const = _map(st["poly"], s1)
        w_scale, k_bias = top(L) * (by / S), round(by * (top(L) / S))
    else:
        const, w_scale, k_bias = 0, top(L) * (before_gate / S), round(before_gate * top(L) / S)
    rot = []
    for c in x:
        turned = [c] + list(ring.rotate(c, baby[1:], keys))
        rot.append((torch.stack(turned), torch.stack(list(ring.rotate(c, wrapped, keys))) if wrapped else None))
    sums = []
    for j in range(n_out):
        total = 0
        for g, step in enumerate(giant):
            acc = 0
            for i, (r0, r1) in enumerate(rot):
                pt = _weights(case, ring, W, i, j, g, n1, w_scale, L)
                use = min(n1, D - n1 * g)
                r = r0[:use] if r1 is None else torch.cat([r0[:use], r1[:use]])
                for p, c in zip(pt, r):
                    acc = (acc + _mul(c, p, q)).remainder(q)
            total = total + (next(ring.rotate(acc, [step], keys)) if step else acc)
        sums.append(total.remainder(q))
    y = torch.stack(sums)
    residual = lambda limbs: [(st["residual"], round(_RESIDUAL * (S * top(limbs) / S)))] if case["residual"] else []  # noqa: E731
    terms = [(st["bias"][:, None], k_bias)] if case["bias"] else []
    if not case["degree"] and not case["gate"]:
        terms += residual(L)
    y = _step(ring, L, rlk, terms=[(y, 1)] + terms, const=const)
    if case["degree"]:
        y = _chebyshev(ring, y, s1, st["poly"][0], before_gate, rlk, () if case["gate"] else residual(m + 1))
    if case["gate"]:
        y = _step(ring, m, rlk, [(y, st["gate"])], 1, residual(m))
    return y


def run(st):
    case = st["case"]
    if not own:
        return list({"poly": _run_poly, "norm": _run_norm, "project": _run_project}[case["kind"]](st, st["ring"]))
    ctx = st["ctx"]
    if case["kind"] == "poly":
        out = ctx.poly_eval(st["x"], st["poly"], st["rlk"])
    elif case["kind"] == "norm":
        out = ctx.rms_norm(st["x"], case["tokens"], st["features"], st["poly"], st["rlk"], st["keys"],
                           layout=case["layout"], weights=st["w"], mask=st["mask"], newton=case["newton"], eps=_EPS,
                           residual=st["residual"], residual_scale=_RESIDUAL)
    else:
        out = ctx.linear_project(st["x"], st["W"], case["tokens"], len(_project_steps(case)[0]), st["keys"],
                                 layout=case["layout"], epilogue=st["epilogue"])
    return [b.data.view(torch.int64) for b in out]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def _poly_steps(degree, L1):
    """(limbs, product?, terms) of every step after T_1's."""
    got, b, have = [], _babies(degree), {1}

    def power(i):
        if i not in have:
            have.add(i)
            power(i - i // 2)
            power(i // 2)
            got.append((L1 + 1 - (i - 1).bit_length(), 1, i % 2))

    def node(c, depth):
        limbs = L1 + 1 - depth
        if _linear(c, b, depth):
            for i in range(1, len(c)):
                power(i)
            got.append((limbs, 0, len(c) - 1))
            return
        q, r, m = _split(c)
        power(m)
        if len(q) > 1:
            node(q, depth - 1)
        if m - 1 < 1 << b:
            for i in range(1, m):
                power(i)
        else:
            node(r, depth - 1)
        got.append((limbs, int(len(q) > 1), m - 1 if m - 1 < 1 << b else 1))

    node([0.0] * (degree + 1), _depth(degree))
    return got


def work(case):
    """Bytes: each input, key and weight once, each output once.  flops: two for every modular product."""
    n, log_n, L, K = 1 << case["log_n"], case["log_n"], case["limbs"], case["n_p"]
    alpha, half, row = -(-case["n_q"] // case["dnum"]), n * log_n / 2, 8.0 * n
    digits = lambda limbs: (limbs - 1) // alpha + 1  # noqa: E731
    rescale = lambda limbs: 2 * (half * limbs + 2 * n * limbs)  # noqa: E731
    key_rows = lambda limbs: digits(limbs) * 2 * (limbs + K)  # noqa: E731

    def up(limbs):
        return half * digits(limbs) * (limbs + K) + n * limbs * (limbs + K)

    def switch(limbs, rotations=1):                            # one ModUp, sums of key products, one ModDown
        down = 2 * (half * (K + limbs) + n * K * limbs + n * limbs)
        return up(limbs) + rotations * n * key_rows(limbs) + down

    def step(limbs, products, terms):
        f = rescale(limbs) + 2 * n * limbs * terms
        return f + 4 * n * limbs * products + switch(limbs) if products else f

    def poly(degree, L1):
        return step(L1 + 1, 0, 1) + sum(step(*s) for s in _poly_steps(degree, L1))

    if case["kind"] == "poly":
        out = L - 1 - _depth(case["degree"])
        return {"bytes": row * (case["count"] * 2 * (L + out) + (key_rows(L - 1) if case["degree"] > 1 else 0)),
                "flops": 2 * case["count"] * poly(case["degree"], L - 1)}
    if case["kind"] == "norm":
        count, tm = case["count"], case["layout"] == "tm"
        Lv = L - 1 - tm
        m = Lv - 1 - _depth(case["degree"]) - 2 * case["newton"]
        rounds = [(len(s), L - 1) for s in _sum_steps(case)] + [(len(s), Lv) for s in (_sum_steps(case, -1) if tm else [])]
        by = row * (count * 2 * (L + m - 1) + key_rows(L) + sum(r * key_rows(limbs) for r, limbs in rounds))
        by += row * count * ({"none": 0, "plain": 1, "cipher": 2}[case["weights"]] * (m + 1) + 2 * m * case["residual"])
        f = step(L, count, 0) + sum(switch(limbs, r) for r, limbs in rounds) + (rescale(L - 1) if tm else 0)
        f += poly(case["degree"], Lv - 1)
        for j in range(case["newton"]):
            at = m + 2 * (case["newton"] - j)
            f += step(Lv, 0, 1) + 2 * step(at, 1, 0) + step(at - 1, 1, 1)
        f += count * step(m, 1, case["residual"])
        f += count * {"none": 0, "plain": rescale(m + 1), "cipher": step(m + 1, 1, 0)}[case["weights"]]
        return {"bytes": by, "flops": 2 * f}
    D = n // 2 // case["tokens"]
    n_in, n_out = case["d_in"] // D, case["d_out"] // D
    baby, wrapped, giant = _project_steps(case)
    turns = len(baby) - 1 + len(wrapped)
    m = L - 1 - (_depth(case["degree"]) if case["degree"] else 0)
    out = m - case["gate"]
    by = row * (2 * n_in * L + 2 * n_out * out + len(_steps(case)) * key_rows(L)) + 8.0 * case["d_in"] * case["d_out"]
    by += row * n_out * (case["bias"] * L + 2 * m * case["gate"] + 2 * (out + 1) * case["residual"])
    by += row * key_rows(m) if case["degree"] or case["gate"] else 0
    down = 2 * (half * (K + L) + n * K * L + n * L)
    f = n_in * (up(L) + turns * (n * key_rows(L) + down)) + n_out * (len(giant) - 1) * switch(L)
    plain = case["d_in"] * n_out * (2 if wrapped else 1)       # weight plaintexts
    small = 2 * D if wrapped else n                            # the ring they are encoded in
    f += plain * L * (2 * n + small * math.log2(small) / 2)
    f += n_out * step(L, 0, case["bias"])
    f += n_out * sum(step(*s) for s in _poly_steps(case["degree"], L - 1)) if case["degree"] else 0
    f += n_out * step(m, 1, case["residual"]) if case["gate"] else 0
    return {"bytes": by, "flops": 2 * f}


# ---- the definition, on the host ------------------------------------------------------------------------------------

class _Exact:
    """Residue arithmetic in numpy: polynomials are held by their values at psi^(2 k + 1) in the natural order of k, a
    ciphertext as [components][limbs][N]."""

    def __init__(self, ring):
        self.primes, self.n, self.n_q, self.n_p, self.alpha = ring.primes, ring.n, ring.n_q, ring.n_p, ring.alpha
        self.order = ring.brev.cpu().numpy()                   # library position j <-> k = brev(j)
        self.special = list(range(self.n_q, self.n_q + self.n_p))
        self.P = math.prod(self.primes[self.n_q:])
        self.roots = {}

    @staticmethod
    def mul(a, b, q):
        a, b = np.asarray(a, dtype=np.int64), np.asarray(b, dtype=np.int64)
        c = np.floor(a.astype(np.longdouble) * b.astype(np.longdouble) / np.longdouble(q)).astype(np.int64)
        with np.errstate(over="ignore"):
            return (a * b - c * np.int64(q)) % np.int64(q)

    def powers(self, base, q, count):
        x = np.ones(1, dtype=np.int64)
        while len(x) < count:
            x = np.concatenate([x, self.mul(x, pow(base, len(x), q), q)])
        return x[:count]

    def root(self, i, inverse):
        if (i, inverse) not in self.roots:
            q = self.primes[i]
            psi = _psi(q, self.n)
            psi = pow(psi, -1, q) if inverse else psi
            self.roots[i, inverse] = (self.powers(psi, q, self.n), self.powers(psi * psi % q, q, self.n // 2))
        return self.roots[i, inverse]

    def cyclic(self, x, w, q):
        """sum_i x_i omega^(i k), natural order in and out."""
        n, s = self.n, 1
        while n > 1:
            m = n // 2
            a, b = x.reshape(n, s)[:m], x.reshape(n, s)[m:]
            x = np.stack([(a + b) % q, self.mul((a - b) % q, w[::s][:, None], q)], 1).reshape(-1)
            n, s = m, 2 * s
        return x

    def values(self, coef, i):
        q, (psi, w) = self.primes[i], self.root(i, False)
        return self.cyclic(self.mul(coef % q, psi, q), w, q)

    def coefs(self, x, i):
        q, (psi, w) = self.primes[i], self.root(i, True)
        y = self.mul(self.mul(self.cyclic(x, w, q), psi, q), pow(self.n, -1, q), q)
        return np.where(y > q // 2, y - q, y)

    def natural(self, x):
        y = np.empty_like(x)
        y[..., self.order] = x
        return y

    def turn(self, x, steps):
        g = pow(5, steps % (self.n // 2), 2 * self.n)
        return x[..., (((2 * np.arange(self.n) + 1) * g % (2 * self.n)) - 1) // 2]

    def spread(self, rows, src, dst):
        """Centred coefficient rows modulo src as values modulo each prime of dst."""
        big = math.prod(self.primes[i] for i in src)
        y = []
        for c, i in zip(rows, src):
            q = self.primes[i]
            d = self.mul(c % q, pow(big // q, -1, q), q)
            y.append(np.where(d > q // 2, d - q, d))
        out = []
        for t in dst:
            q = self.primes[t]
            out.append(self.values(sum(self.mul(d % q, big // self.primes[i] % q, q) for d, i in zip(y, src)) % q, t))
        return out

    def times(self, x, k):
        """Rows [..., limbs, N] by an integer."""
        return np.stack([self.mul(x[..., i, :], k % self.primes[i], self.primes[i]) for i in range(x.shape[-2])], -2)

    def plus(self, a, b):
        return (a + b) % np.array(self.primes[:a.shape[-2]], dtype=np.int64)[:, None]

    def product(self, a, b):
        return np.stack([self.mul(a[..., i, :], b[..., i, :], self.primes[i]) for i in range(a.shape[-2])], -2)

    def rescaled(self, ct):
        l = ct.shape[-2] - 1
        out = np.empty((len(ct), l, self.n), dtype=np.int64)
        for k, x in enumerate(ct):
            top = self.coefs(x[l], l)
            for i in range(l):
                q = self.primes[i]
                out[k, i] = self.mul((x[i] - self.values(top, i)) % q, pow(self.primes[l], -1, q), q)
        return out

    def switched(self, c, turns):
        """sum over (key, steps) of the key switch of c turned by steps, one division by P: [2][limbs][N]; c0 adds."""
        return self.divided(self.summed(c, turns), len(c))

    def digits(self, c):
        L, ext = len(c), list(range(len(c))) + self.special
        out = []
        for lo in range(0, L, self.alpha):
            mine = list(range(lo, min(lo + self.alpha, L)))
            rows = self.spread([self.coefs(c[i], i) for i in mine], mine, [e for e in ext if e not in mine])
            out.append([c[e] if e in mine else rows.pop(0) for e in ext])
        return out

    def summed(self, c, turns):
        ext = list(range(len(c))) + self.special
        digits, u = self.digits(c), np.zeros((2, len(ext), self.n), dtype=np.int64)
        for key, steps in turns:
            for d, dig in enumerate(digits):
                for r, e in enumerate(ext):
                    x = self.turn(dig[r], steps)
                    for k in range(2):
                        u[k, r] = (u[k, r] + self.mul(x, key[d, k, e], self.primes[e])) % self.primes[e]
        return u

    def divided(self, u, L):
        out = np.empty((2, L, self.n), dtype=np.int64)
        for k in range(2):
            c = self.spread([self.coefs(u[k, L + i], e) for i, e in enumerate(self.special)], self.special, range(L))
            for i in range(L):
                q = self.primes[i]
                out[k, i] = self.mul((u[k, i] - c[i]) % q, pow(self.P, -1, q), q)
        return out

    def rotated(self, ct, steps, key):
        if not steps:
            return ct
        out = self.switched(ct[1], [(key, steps)])
        out[0] = self.plus(out[0], self.turn(ct[0], steps))
        return out

    def step(self, L, rlk, products=(), mult=1, terms=(), const=0):
        v, d2 = np.zeros((2, L, self.n), dtype=np.int64), 0
        for a, b in products:
            a, b = a[:, :L], b[:, :L]
            v = self.plus(v, self.times(np.stack([self.product(a[0], b[0]), self.plus(
                self.product(a[0], b[1]), self.product(a[1], b[0]))]), mult))
            d2 = self.plus(self.times(self.product(a[1], b[1]), mult), d2)
        for z, k in terms:
            v[:len(z)] = self.plus(v[:len(z)], self.times(z[:, :L], k))
        if len(products):
            v = self.plus(v, self.switched(d2, [(rlk, 0)]))
        out = self.rescaled(v)
        out[0] = self.plus(out[0], np.array([const % q for q in self.primes[:L - 1]], dtype=np.int64)[:, None])
        return out

    # the operators, each from its own formula

    def series(self, t1, s1, c, target, rlk, extra=()):
        """sum c_i T_i(t) with T_i and the tree of quotients by T_(2^s) as the operator defines them."""
        L1, D = t1.shape[1], len(bin(len(c) - 1)) - 2
        b, T, q = min(3, max(1, D - 2)), {1: (t1, s1)}, [float(p) for p in self.primes]

        def cheb(i):
            if i in T:
                return T[i]
            lo, hi = cheb(i // 2), cheb((i + 1) // 2)
            L = min(lo[0].shape[1], hi[0].shape[1])
            s = hi[1] * lo[1] / q[L - 1]
            odd = [(t1, -round(hi[1] * lo[1] / s1))] if i & 1 else []
            T[i] = self.step(L, rlk, [(hi[0], lo[0])], 2, odd, 0 if odd else -round(s)), s
            return T[i]

        def value(c, L, target, extra):                        # from L limbs to L - 1
            up, d = target * q[L - 1], len(c) - 1
            scaled = lambda i, x: (cheb(i)[0], round(x * (up / cheb(i)[1])))  # noqa: E731
            if d < 2 ** b and (d == 1 or math.ceil(math.log2(d)) <= L1 - L):
                return self.step(L, rlk, (), 1, [scaled(i, c[i]) for i in range(1, d + 1)] + extra, round(c[0] * target))
            m = 2 ** int(math.log2(d))
            quot, rem = {0: c[m]}, {j: c[j] for j in range(m)}
            for i in range(1, d - m + 1):                      # c T_(m+i) = 2 c T_m T_i - c T_(m-i)
                quot[i] = 2 * c[m + i]
                rem[m - i] -= c[m + i]
            quot, rem = [quot[i] for i in sorted(quot)], [rem[j] for j in sorted(rem)]
            prods, terms, const = [], list(extra), 0
            if d == m:
                terms.append(scaled(m, quot[0]))
            else:
                prods.append((value(quot, L + 1, up / cheb(m)[1], []), cheb(m)[0]))
            if m <= 2 ** b:
                terms += [scaled(j, rem[j]) for j in range(1, m)]
                const = round(rem[0] * target)
            else:
                terms.append((value(rem, L + 1, target, []), self.primes[L - 1]))
            return self.step(L, rlk, prods, 1, terms, const)

        return value(list(c), L1 + 1 - D, target, list(extra))

    def poly(self, case, st):
        (c, lo, hi), S, rlk, out = st["poly"], st["scale"], st["rlk"], []
        for x in st["x"]:
            L = x.shape[1]
            s1, top = float(self.primes[L - 2]), float(self.primes[L - 1])
            t1 = self.step(L, rlk, (), 1, [(x, round(2.0 / (hi - lo) * s1 * (top / S)))], round(-(lo + hi) / (hi - lo) * s1))
            out.append(self.series(t1, s1, c, S, rlk))
        return out

    def all_features(self, ct, case, keys, sign):
        D, unit = self.n // 2 // case["tokens"], case["tokens"] if case["layout"] == "fm" else 1
        bits = D.bit_length() - 1
        left = -(-bits // 4)
        while bits:
            take = -(-bits // left)
            steps = [sign * unit * k for k in range(1, 2 ** take)]
            L = ct.shape[1]
            u = self.summed(ct[1], [(keys[s], s) for s in steps])
            c0 = sum(self.turn(ct[0], s) for s in steps)
            for i in range(L):
                u[0, i] = (u[0, i] + self.mul(c0[i] % self.primes[i], self.P % self.primes[i], self.primes[i])) % self.primes[i]
            ct = self.plus(ct, self.divided(u, L))
            bits, left, unit = bits - take, left - 1, unit * 2 ** take
        return ct

    def norm(self, case, st):
        (c, lo, hi), S, rlk, keys, q = st["poly"], st["scale"], st["rlk"], st["keys"], [float(p) for p in self.primes]
        L, d = st["x"][0].shape[1], float(st["features"])
        v = self.all_features(self.step(L, rlk, [(x, x) for x in st["x"]]), case, keys, 1)
        sv = S * S / q[L - 1]
        if case["layout"] == "tm":
            v = self.rescaled(np.stack([self.product(z, st["mask"][0][:L - 1]) for z in v]))
            v, sv = self.all_features(v, case, keys, -1), sv * S / q[L - 2]
        Lv = v.shape[1]
        D = len(bin(case["degree"])) - 2
        m = Lv - 1 - D - 2 * case["newton"]
        sx = S * S / q[m] if "w" in st else S
        s1, end = q[Lv - 2], S * q[m - 1] / sx
        t1 = self.step(Lv, rlk, (), 1, [(v, round(2.0 / (hi - lo) * s1 / d * (q[Lv - 1] / sv)))],
                       round(-(lo + hi) / (hi - lo) * s1))
        sy = q[Lv - 2 - D] if case["newton"] else end
        y = self.series(t1, s1, c, sy, rlk)
        for left in range(case["newton"] - 1, -1, -1):
            k = y.shape[1]
            to, qa, qb = (q[k - 3] if left else end), q[k - 1], q[k - 2]
            s2 = sy * sy / qa
            sn = to / 2 * qb / s2 * qa / sy
            mean = self.step(Lv, rlk, (), 1, [(v, round(sn / d * (q[Lv - 1] / sv)))], round(_EPS * sn))
            sp = sn * sy / qa * s2 / qb
            y = self.step(k - 1, rlk, [(self.step(k, rlk, [(mean, y)]), self.step(k, rlk, [(y, y)]))], -1,
                          [(y, round(3.0 * (sp * qb / sy)))])
            sy = to
        out = []
        for i, x in enumerate(st["x"]):
            if case["weights"] == "plain":
                x = self.rescaled(np.stack([self.product(z, st["w"][i][0][:m + 1]) for z in x[:, :m + 1]]))
            elif case["weights"] == "cipher":
                x = self.step(m + 1, rlk, [(x, st["w"][i])])
            res = [(st["residual"][i], round(_RESIDUAL * (S * q[m - 1] / S)))] if case["residual"] else []
            out.append(self.step(m, rlk, [(x, y)], 1, res))
        return out

    def encoded(self, z, scale, L):
        """A slot vector's plaintext over L limbs, by decimation in time with every product and sum rounded."""
        M = len(z)
        n, stride = 2 * M, self.n // (2 * M)
        w, twist = _turns(n)
        rev = _brev(M.bit_length() - 1).numpy()
        re, im, half = np.empty(M), np.zeros(M), 1
        re[rev[_slots_at(n)]] = z
        while half < M:
            for k in range(half):
                wr, wi = w[k * (M // (2 * half)), 0], -w[k * (M // (2 * half)), 1]
                xr, xi = re[k + half::2 * half], im[k + half::2 * half]
                tr, ti = wr * xr - wi * xi, wr * xi + wi * xr
                ur, ui = re[k::2 * half].copy(), im[k::2 * half].copy()
                re[k::2 * half], im[k::2 * half] = ur + tr, ui + ti
                re[k + half::2 * half], im[k + half::2 * half] = ur - tr, ui - ti
            half *= 2
        f, c, s = scale * (2.0 / n), twist[:, 0], -twist[:, 1]
        x = np.concatenate([f * (c * re - s * im), f * (c * im + s * re)])
        m = np.zeros(self.n, dtype=np.int64)
        m[::stride] = [int(math.copysign(math.floor(abs(v)) + (abs(v) - math.floor(abs(v)) >= 0.5), v)) for v in x]
        return np.stack([self.values(m, i) for i in range(L)])

    def project(self, case, st):
        S, rlk, keys, q = st["scale"], st["rlk"], st["keys"], [float(p) for p in self.primes]
        W, T, L, fm = st["W"], case["tokens"], st["x"][0].shape[1], case["layout"] == "fm"
        D = self.n // 2 // T
        n1, unit = min(case["n1"], D), T if fm else 1
        depth = len(bin(case["degree"])) - 2 if case["degree"] else 0
        m = L - 1 - depth
        target, const = S * q[m - 1] / S if case["gate"] else S, 0
        if depth:
            c, lo, hi = st["poly"]
            s1 = q[L - 2]
            by, const = 2.0 / (hi - lo) * s1, round(-(lo + hi) / (hi - lo) * s1)
            scale, k_bias = q[L - 1] * (by / S), round(by * (q[L - 1] / S))
        else:
            scale, k_bias = q[L - 1] * (target / S), round(target * q[L - 1] / S)
        turned = lambda x, s: self.rotated(x, s, keys.get(s))  # noqa: E731
        rots = [([turned(x, unit * b) for b in range(n1)], [] if fm else [turned(x, b - D) for b in range(n1)])
                for x in st["x"]]
        out = []
        for j in range(case["d_out"] // D):
            total = 0
            for g in range(-(-D // n1)):
                acc = 0
                for i, (plain, wrapped) in enumerate(rots):
                    for b in range(min(n1, D - n1 * g)):
                        k = n1 * g + b
                        o = (np.arange(D) - n1 * g) % D
                        diag = W[i * D + (o + k) % D, j * D + o]
                        if fm:
                            parts = [(np.repeat(diag, T), plain[b])]
                        else:
                            parts = [(np.where(o + k < D, diag, 0.0), plain[b]), (np.where(o + k < D, 0.0, diag), wrapped[b])]
                        for z, x in parts:
                            pt = self.encoded(z, scale, L)
                            acc = self.plus(np.stack([self.product(v, pt) for v in x]), acc)
                total = self.plus(turned(acc, unit * n1 * g), total)
            res = lambda limbs: [(st["residual"][j], round(_RESIDUAL * (S * q[limbs - 1] / S)))] if case["residual"] else []  # noqa: E731
            terms = [(total, 1)] + ([(st["bias"][j][None], k_bias)] if case["bias"] else [])
            y = self.step(L, rlk, (), 1, terms + ([] if depth or case["gate"] else res(L)), const)
            if depth:
                y = self.series(y, s1, c, target, rlk, [] if case["gate"] else res(m + 1))
            if case["gate"]:
                y = self.step(m, rlk, [(y, st["gate"][j])], 1, res(m))
            out.append(y)
        return out


def exact(case, seed):
    """The residues by the definition in integers; None where numpy would take too long over it."""
    if work(case)["flops"] * (2 if case["kind"] == "project" else 1) > 2e8:
        return None
    ring, st = _inputs(case, seed)
    E = _Exact(ring)
    plain = lambda v: E.natural(v.cpu().numpy()) if v.dtype == torch.int64 else v.cpu().numpy()  # noqa: E731
    host = {k: {s: plain(x) for s, x in v.items()} if isinstance(v, dict) else plain(v) if torch.is_tensor(v) else v
            for k, v in st.items()}
    got = {"poly": E.poly, "norm": E.norm, "project": E.project}[case["kind"]](case, host)
    return [torch.from_numpy(np.ascontiguousarray(x[..., E.order])) for x in got]

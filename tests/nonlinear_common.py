"""What the tests of polynomials, norms and the projection's epilogue share: the operators put together from the oracle's
stages, and bounds on what their decrypted values may be off by."""
import math

import numpy as np


def step(ck, L, rlk=None, products=(), mult=1, terms=(), const=0):
    """Rescale(relin(mult sum a b) + sum k z) + const of ciphertexts cut to L limbs; b or z of one polynomial: a plaintext."""
    idx = ck.level_primes(L - 1)
    v, d2 = np.zeros((2, L, ck.n), dtype=np.uint64), None
    for a, b in products:
        a, b = (np.ascontiguousarray(x[:, :L]) for x in (a, b))
        if len(b) == 1:
            v = ck.ct_add(v, ck.ct_mul_plain(a, b[0]))
            continue
        d = ck.tensor(a, b)
        d = np.stack([ck.mul_scalar(x, [mult] * L, idx) for x in d])
        v = ck.ct_add(v, d[:2])
        d2 = d[2] if d2 is None else ck.add(d2, d[2], idx)
    if d2 is not None:
        v = ck.relin(np.concatenate([v, d2[None]]), rlk)
    for z, k in terms:
        for i in range(len(z)):
            v[i] = ck.add(v[i], ck.mul_scalar(z[i, :L], [k] * L, idx), idx)
    out = ck.rescale(v)
    low = idx[:-1]
    out[0] = ck.add(out[0], np.stack([np.full(ck.n, const % ck.q[i], dtype=np.uint64) for i in low]), low)
    return out


def series(ck, t1, s1, coefs, target, rlk, extra=()):
    """sum c_i T_i of the ciphertext t1, as the header defines it."""
    L1, deg = t1.shape[1], len(coefs) - 1
    D = deg.bit_length()
    b = min(3, max(1, D - 2))
    top = lambda L: float(ck.q[L - 1])  # noqa: E731
    at = lambda i: math.ceil(math.log2(i))  # noqa: E731
    known = {1: (t1, s1)}

    def cheb(i):
        if i not in known:
            (x, sx), (y, sy) = cheb(i - i // 2), cheb(i // 2)
            L = L1 - at(i) + 1
            s = sx * sy / top(L)
            if i % 2:
                known[i] = step(ck, L, rlk, [(x, y)], 2, [(t1, -round(sx * sy / s1))]), s
            else:
                known[i] = step(ck, L, rlk, [(x, y)], 2, (), -round(s)), s
        return known[i]

    def total(c, depth, s, extra):
        L, d = L1 - depth + 1, len(c) - 1
        def term(i, x):
            z, sz = cheb(i)
            return z, round(x * ((s * top(L)) / sz))
        if d < 2 ** b and at(d) < depth:
            return step(ck, L, None, (), 1, [term(i, c[i]) for i in range(1, d + 1)] + extra, round(c[0] * s))
        m = 1 << (d.bit_length() - 1)
        q, r = [c[m]] + [2 * x for x in c[m + 1:]], list(c[:m])
        for i in range(1, len(q)):
            r[m - i] -= c[m + i]
        prods, terms, const = [], list(extra), 0
        if len(q) > 1:
            prods = [(total(q, depth - 1, s * top(L) / cheb(m)[1], []), cheb(m)[0])]
        else:
            terms.append(term(m, q[0]))
        if m <= 2 ** b:
            terms += [term(i, r[i]) for i in range(1, m)]
            const = round(r[0] * s)
        else:
            terms.append((total(r, depth - 1, s, []), ck.q[L - 1]))
        return step(ck, L, rlk, prods, 1, terms, const)

    return total(list(coefs), D, target, list(extra))


def mapped(poly, s1):
    return 2.0 / (poly.hi - poly.lo) * s1, round(-(poly.lo + poly.hi) / (poly.hi - poly.lo) * s1)


def poly_eval(ck, ct, scale, poly, rlk):
    L = ct.shape[1]
    s1, top = float(ck.q[L - 2]), float(ck.q[L - 1])
    by, const = mapped(poly, s1)
    t1 = step(ck, L, None, (), 1, [(ct, round(by * (top / scale)))], const)
    return series(ck, t1, s1, poly.coefs, scale, rlk)


def radixes(count):
    bits, out = count.bit_length() - 1, []
    for left in range(-(-bits // 4), 0, -1):
        out.append(1 << -(-bits // left))
        bits -= out[-1].bit_length() - 1
    return out


def all_positions(ck, ct, count, stride, keys):
    slots = ck.n // 2
    for radix in radixes(count):
        steps = [k * stride for k in range(1, radix)]
        ct = ck.ct_add(ct, ck.rotate_sum_lazy([ct] * len(steps), steps, [keys[s % slots] for s in steps]))
        stride *= radix
    return ct


def rms_norm(ck, cts, scale, tokens, features, poly, rlk, keys, layout, weights=None, w_scale=1.0, mask=None, m_scale=1.0,
             newton=0, eps=0.0, residual=None, r_scale=1.0, residual_scale=1.0):
    top = lambda L: float(ck.q[L - 1])  # noqa: E731
    L, D, d = cts[0].shape[1], ck.n // 2 // tokens, float(features)
    v = all_positions(ck, step(ck, L, rlk, [(x, x) for x in cts]), D, tokens if layout == "fm" else 1, keys)
    sv, Lv = scale * scale / top(L), L - 1
    if layout == "tm":
        v = all_positions(ck, step(ck, L - 1, None, [(v, mask)]), D, -1, keys)
        sv, Lv = sv * m_scale / top(L - 1), L - 2
    m0 = Lv - 1 - poly.depth
    m = m0 - 2 * newton
    sx = scale * w_scale / top(m + 1) if weights is not None else scale
    last, s1 = scale * top(m) / sx, top(Lv - 1)
    by, const = mapped(poly, s1)
    t1 = step(ck, Lv, None, (), 1, [(v, round(by / d * (top(Lv) / sv)))], const)
    sy = top(m0) if newton else last
    y = series(ck, t1, s1, poly.coefs, sy, rlk)
    for j in range(newton):
        a, b, k = top(m0 - 2 * j), top(m0 - 2 * j - 1), m0 - 2 * j
        to = top(k - 2) if j + 1 < newton else last
        s2 = sy * sy / a
        sn = to / 2 * b / s2 * a / sy
        n = step(ck, Lv, None, (), 1, [(v, round(sn / d * (top(Lv) / sv)))], round(eps * sn))
        sp = sn * sy / a * s2 / b
        y = step(ck, k - 1, rlk, [(step(ck, k, rlk, [(n, y)]), step(ck, k, rlk, [(y, y)]))], -1,
                 [(y, round(3.0 * (sp * b / sy)))])
        sy = to
    out = []
    for i, x in enumerate(cts):
        if weights is not None:
            x = step(ck, m + 1, rlk, [(x, weights[i])])
        res = [(residual[i], round(residual_scale * (scale * top(m) / r_scale)))] if residual is not None else []
        out.append(step(ck, m, rlk, [(x, y)], 1, res))
    return out


def projected_sums(ck, cts, W, T, n1, keys, layout, w_scale, lazy=False):
    """The sums of the oracle's projection before its rescale, from weights encoded at w_scale."""
    level, D = ck.level_of(cts[0]), ck.n // 2 // T
    unit = T if layout == "fm" else 1
    rots = []
    for c in cts:
        got = [c] + [ck.rotate(c, unit * b, keys[unit * b]) for b in range(1, n1)]
        rots.append((got, [ck.rotate(c, b - D, keys[b - D]) for b in range(n1)] if layout == "tm" else []))
    outs = []
    for j in range(W.shape[1] // D):
        total = None
        for g in range(-(-D // n1)):
            acc = None
            for i, (plain, wrapped) in enumerate(rots):
                for b in range(min(n1, D - n1 * g)):
                    if layout == "fm":
                        parts = [(ck.encode(ck.diag_slot_vector(W, T, D, j, i, n1, g, b), None, w_scale, level + 1), plain[b])]
                    else:
                        u, v = ck.periodic_diag_vectors(W, D, j, i, n1, g, b)
                        parts = [(ck.encode_periodic(z, w_scale, level + 1), x) for z, x in ((u, plain[b]), (v, wrapped[b]))]
                    for pt, x in parts:
                        t = ck.ct_mul_plain(x, pt)
                        acc = t if acc is None else ck.ct_add(acc, t)
            total = ck._giant_step(total, acc, g, unit * n1 * g, keys, lazy)
        outs.append(ck._giant_finish(total, lazy))
    return outs


def project(ck, cts, scale, W, T, n1, keys, layout, rlk, bias=None, b_scale=1.0, act=None, gate=None, g_scale=1.0,
            residual=None, r_scale=1.0, residual_scale=1.0, lazy=False):
    top = lambda L: float(ck.q[L - 1])  # noqa: E731
    L = cts[0].shape[1]
    m = L - 1 - (act.depth if act else 0)
    to, const = scale * top(m) / g_scale if gate is not None else scale, 0
    if act:
        by, const = mapped(act, top(L - 1))
        w_scale, kb = top(L) * (by / scale), round(by * (top(L) / b_scale))
    else:
        w_scale, kb = top(L) * (to / scale), round(to * top(L) / b_scale)
    res = lambda j, L: [(residual[j], round(residual_scale * (scale * top(L) / r_scale)))] if residual is not None else []  # noqa: E731
    out = []
    for j, s in enumerate(projected_sums(ck, cts, W, T, n1, keys, layout, w_scale, lazy)):
        terms = [(s, 1)] + ([(bias[j], kb)] if bias is not None else [])
        y = step(ck, L, None, (), 1, terms + ([] if act or gate is not None else res(j, L)), const)
        if act:
            y = series(ck, y, top(L - 1), act.coefs, to, rlk, [] if gate is not None else res(j, m + 1))
        if gate is not None:
            y = step(ck, m, rlk, [(y, gate[j])], 1, res(j, m))
        out.append(y)
    return out


def poly_bound(coefs, e1, d):
    """What sum c_i T_i (|T_i| <= 1) may be off by where T_1 is off by e1 and every step adds at most d of its own, along
    the header's tree: errors of T_i, then of sums, |q| <= sum |c|."""
    deg = len(coefs) - 1
    D = deg.bit_length()
    b = min(3, max(1, D - 2))
    et = {1: e1}

    def e(i):
        if i not in et:
            x, y = e(i - i // 2), e(i // 2)
            et[i] = 2 * (x + y + x * y) + (e1 if i % 2 else 0) + d
        return et[i]

    def total(c, depth):
        n = len(c) - 1
        if n < 2 ** b and math.ceil(math.log2(n)) < depth:
            return sum(abs(c[i]) * e(i) for i in range(1, n + 1)) + d
        m = 1 << (n.bit_length() - 1)
        q, r = [c[m]] + [2 * x for x in c[m + 1:]], list(c[:m])
        for i in range(1, len(q)):
            r[m - i] -= c[m + i]
        rest = sum(abs(r[i]) * e(i) for i in range(1, m)) if m <= 2 ** b else total(r, depth - 1)
        if len(q) == 1:
            return abs(q[0]) * e(m) + rest + d
        eq = total(q, depth - 1)
        return eq + (sum(map(abs, q)) + eq) * e(m) + rest + d
    return total(list(coefs), D)

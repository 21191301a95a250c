"""The calls' arguments as the binding checks them, on the CPU: each case is refused before the library is reached.  Also
the polynomials' fits and values, the rotation steps, and the plan of a sum against plain evaluation."""
import math

import numpy as np
import pytest
import torch

import nonlinear_common as nc
from paper_2609_12378_amd import Buf, CkksError, Context, Epilogue, Poly
from test_rope_args import ct, ctx, key  # noqa: F401


P2 = Poly((0.5, 1.0, 0.25), -1.0, 1.0)


def pt(limbs=3):
    return Buf(torch.zeros((1, limbs, 16), dtype=torch.uint64), 2.0 ** 20)


def weights(*shape, dtype=torch.float64):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("call", [
    lambda c: c.poly_eval([ct(3)], P2, key(c, torch.int64)),
    lambda c: c.poly_eval([ct(3)], P2, key(c)[:1]),
    lambda c: c.poly_eval([ct(3)], P2, None),
    lambda c: c.poly_eval([ct(3, n=8)], P2, key(c)),
    lambda c: c.poly_eval([ct(3, dtype=torch.int64)], P2, key(c)),
    lambda c: c.poly_eval([ct(3), ct(3)], P2, key(c), outs=[ct(1)]),
    lambda c: c.poly_eval([ct(3)], Poly((), 0.0, 1.0), key(c), outs=[ct(1)]),
    lambda c: norm(c, layout="rows"),
    lambda c: norm(c, tokens=2.0),
    lambda c: norm(c, features=-1),
    lambda c: norm(c, newton=1 << 32),
    lambda c: norm(c, weights=[]),
    lambda c: norm(c, residual=[]),
    lambda c: norm(c, keys={1: key(c, torch.int32)}),
    lambda c: norm(c, keys={1 << 31: key(c)}),
    lambda c: norm(c, mask=Buf(torch.zeros((1, 3, 8), dtype=torch.uint64), 1.0)),
    lambda c: norm(c, outs=[]),
    lambda c: proj(c, bias=[]),
    lambda c: proj(c, gate=[]),
    lambda c: proj(c, residual=[Buf(torch.zeros((2, 3, 16), dtype=torch.int64), 1.0)]),
    lambda c: proj(c, rlk=key(c)[:1]),
    lambda c: c.norm_mask(3, 2, 1.0),
    lambda c: c.norm_mask(0, 2, 1.0),
])
def test_refused_by_the_binding(ctx, call):  # noqa: F811
    with pytest.raises(CkksError):
        call(ctx)


def norm(c, tokens=2, features=4, keys=None, **kw):
    kw.setdefault("outs", [ct(1)])
    return c.rms_norm([ct(3)], tokens, features, P2, key(c), {} if keys is None else keys, **kw)


def proj(c, **kw):
    return c.linear_project([ct(3)], weights(4, 4), 2, 2, {}, outs=[ct(1)], epilogue=Epilogue(**kw))


def test_a_well_formed_call_reaches_the_library(ctx):  # noqa: F811
    for call in (lambda c: c.poly_eval([ct(3)], P2, key(c), outs=[ct(1)]),
                 lambda c: norm(c, weights=[pt()], residual=[ct(3)], mask=pt(), layout="tm"),
                 lambda c: proj(c, bias=[pt()], act=P2, gate=[ct(3)], residual=[ct(3)], rlk=key(c)), lambda c: proj(c)):
        with pytest.raises(AssertionError, match="the library was called"):
            call(ctx)


def test_nothing_to_do_is_not_an_error(ctx):  # noqa: F811
    assert ctx.poly_eval([], P2, key(ctx)) == []
    assert ctx.rms_norm([], 2, 4, P2, key(ctx), {}) == []


def test_norm_steps():
    assert Context.norm_steps(2048, 16) == sorted([16 * k for k in range(1, 16)] + [256 * k for k in range(1, 8)])
    assert Context.norm_steps(64, 8) == [8 * k for k in range(1, 8)]
    assert Context.norm_steps(64, 16, "tm") == [1, 2, 3, 61, 62, 63]
    assert Context.norm_steps(64, 64) == []
    # every sum of one step or none a round is each multiple of the stride once
    for slots, tokens in ((32768, 128), (32768, 1), (4096, 8)):
        seen, unit = {0}, tokens
        for radix in nc.radixes(slots // tokens):
            seen = {a + k * unit for a in seen for k in range(radix)}
            unit *= radix
        assert sorted(seen) == list(range(0, slots, tokens))


@pytest.mark.parametrize("degree", [1, 2, 7, 15, 40])
def test_fit_and_value(degree):
    """Exact at the nodes (sums of degree + 1 products of at most 1: 2 (degree + 1)^2 roundings of 2^-53), and the same sum
    as numpy's."""
    fn = lambda x: 1 / (1 + x * x)  # noqa: E731
    p = Poly.fit(fn, degree, -2.0, 3.0)
    assert p.degree == degree and p.depth == math.ceil(math.log2(degree + 1))
    for k in range(degree + 1):
        x = 2.5 * math.cos(math.pi * (k + 0.5) / (degree + 1)) + 0.5
        assert abs(p(x) - fn(x)) < 2 * (degree + 2) ** 2 * 2.0 ** -53
    at = np.linspace(-2, 3, 41)
    want = np.polynomial.chebyshev.chebval((at - 0.5) / 2.5, np.array(p.coefs))
    assert np.max(np.abs([p(x) for x in at] - want)) < 4 * (degree + 2) ** 2 * 2.0 ** -53
    with pytest.raises(CkksError):
        Poly.fit(fn, 0, 0.0, 1.0)
    with pytest.raises(CkksError):
        Poly.fit(fn, 3, 1.0, 1.0)


class Plain:
    """The oracle's interface with real numbers for ciphertexts: a value times its scale, a level's limbs as its length."""
    n = 2

    def __init__(self, primes):
        self.q = primes


@pytest.mark.parametrize("degree", list(range(1, 34)) + [47, 63, 64, 100, 127])
def test_the_tree_of_a_sum_is_the_sum(degree, monkeypatch):
    """The tree with exact arithmetic in place of ciphertexts gives the sum, within the rounding of its integers (below
    2^-49 of each of at most 2 degree terms of size sum |c| 2^7), and takes no more levels than the degree's bits."""
    class Value:
        def __init__(self, v, limbs):
            self.v, self.shape = v, (2, limbs)
    lowest = []

    def step(ck, L, rlk=None, products=(), mult=1, terms=(), const=0):
        assert all(x.shape[1] >= L for p in products for x in p) and all(z.shape[1] >= L for z, _ in terms)
        assert len(terms) <= 8 and len(products) <= 1
        v = sum(mult * a.v * b.v for a, b in products) + sum(z.v * k for z, k in terms)
        lowest.append(L - 1)
        return Value(v / ck.q[L - 1] + const, L - 1)

    monkeypatch.setattr(nc, "step", step)
    ck = Plain([2 ** 50 - 2 ** 20 * i - 1 for i in range(10)])
    c = np.random.default_rng(degree).normal(0, 1, degree + 1)
    for t in (-1.0, -0.3, 0.77, 1.0):
        lowest.clear()
        s1, target = float(ck.q[8]), 1.01 * 2.0 ** 49
        got = nc.series(ck, Value(t * s1, 9), s1, list(c), target, None)
        want = np.polynomial.chebyshev.chebval(t, c)
        assert got.shape[1] == min(lowest) == 9 - math.ceil(math.log2(degree + 1))
        assert abs(got.v / target - want) < 2.0 ** -49 * 2 * degree * np.sum(np.abs(c)) * 2 ** 7

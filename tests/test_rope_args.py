"""The rotary and cache calls' arguments as the binding checks them, on the CPU: each case is refused before the library
is reached.  Also the frequencies, and the plain helpers that the GPU tests compare with."""
import math

import numpy as np
import pytest
import torch

import paper_2609_12378_amd as pkg
from paper_2609_12378_amd import Buf, CkksError, Context, rope_inv_freq
from rope_common import plain_rope
from test_binding_args import _host_ptr, _NoLibrary


@pytest.fixture
def ctx(monkeypatch):
    monkeypatch.setattr(pkg, "_ptr", _host_ptr)
    c = Context.__new__(Context)
    c.lib, c.h, c._stream, c.device = _NoLibrary(), None, None, 0
    c.log_n, c.n, c.n_q, c.n_p, c.dnum, c.alpha = 4, 16, 3, 1, 2, 2
    c.q, c.p = [97, 193, 257], [353]
    c.primes = c.q + c.p
    return c


def ct(limbs=2, n=16, dtype=torch.uint64):
    return Buf(torch.zeros((2, limbs, n), dtype=dtype), 2.0 ** 20)


def tab(*lead, limbs=2, dtype=torch.uint64):
    return torch.zeros((*lead, limbs + 1, 16), dtype=dtype)


def key(c, dtype=torch.uint64):
    return torch.zeros(c.key_shape(), dtype=dtype)


def f64(*shape):
    return torch.zeros(shape, dtype=torch.float64)


@pytest.mark.parametrize("call", [
    lambda c: c.rope_cos_sin(f64(3), f64(2)),
    lambda c: c.rope_cos_sin(torch.zeros(3, dtype=torch.int32), f64(2)),
    lambda c: c.rope_cos_sin(torch.zeros((3, 1), dtype=torch.int64), f64(2)),
    lambda c: c.rope_cos_sin(torch.zeros(3, dtype=torch.int64), torch.zeros(2)),
    lambda c: c.rope_cos_sin([1, 2], f64(2)),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 1), 2, 4, 4, 2),
    lambda c: c.rope_tables(f64(2, 1), f64(2, 1), 2, 4, 4, 2),
    lambda c: c.rope_tables(torch.zeros((2, 2)), torch.zeros((2, 2)), 2, 4, 4, 2),
    lambda c: c.rope_tables(f64(4), f64(4), 2, 4, 4, 2),
    lambda c: c.rope_tables(f64(3, 2), f64(3, 2), 2, 4, 4, 2),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 2, first=1),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 2, first=-1),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 4),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 2, out=tab(2)),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 2, out=tab(3, dtype=torch.int64)),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 2, layout="rows"),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 2, pairing="both"),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2.0, 4, 4, 2),
    lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, -4, 4, 2),
    lambda c: c.rope([ct()], tab(3, limbs=3), 2, 4, 4, {2: key(c), 6: key(c)}),
    lambda c: c.rope([ct()], tab(2), 2, 4, 4, {2: key(c), 6: key(c)}),
    lambda c: c.rope([ct()], tab(3, dtype=torch.int64), 2, 4, 4, {2: key(c), 6: key(c)}),
    lambda c: c.rope([ct(n=8)], tab(3), 2, 4, 4, {2: key(c), 6: key(c)}),
    lambda c: c.rope([ct(dtype=torch.int64)], tab(3), 2, 4, 4, {2: key(c), 6: key(c)}),
    lambda c: c.rope([ct(), ct()], tab(3), 2, 4, 4, {2: key(c), 6: key(c)}, outs=[ct(1)]),
    lambda c: c.rope([ct()], tab(3), 2, 4, 4, {2: key(c, torch.int64)}),
    lambda c: c.rope([ct()], tab(3), 2, 4, 4, {2: key(c)[:1]}),
    lambda c: c.rope([ct()], tab(3), 2, 4, 4, {1 << 31: key(c)}),
    lambda c: c.rope([ct()], tab(3), 2, 4, 4, {2: key(c)}, outs=[Buf(torch.zeros((2, 1, 16)), 1.0)]),
    lambda c: c.cache_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 0, 3, 2),
    lambda c: c.cache_tables(f64(2, 2), f64(2, 2), 2, 4, 4, -1, 2, 2),
    lambda c: c.cache_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 1 << 32, 2, 2),
    lambda c: c.cache_tables(f64(1, 2), f64(2, 2), 2, 4, 4, 0, 2, 2, out=tab(1, 4)),
    lambda c: c.cache_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 1, 2, 2, out=tab(1, 4)),
    lambda c: append(c, tables=tab(2, 4)),
    lambda c: append(c, tables=tab(1, 3)),
    lambda c: append(c, length=1),
    lambda c: append(c, v=[]),
    lambda c: append(c, v=[ct(), ct()]),
    lambda c: append(c, table=[]),
    lambda c: append(c, table=[[0], [1]]),
    lambda c: append(c, table=[[-1]]),
    lambda c: append(c, fork=[0, 0]),
    lambda c: append(c, fork=[-1]),
    lambda c: append(c, vp=[]),
    lambda c: append(c, kp=[ct(1, n=8)]),
    lambda c: append(c, src=3),
    lambda c: append(c, src=-1),
    lambda c: append(c, count=3),
    lambda c: append(c, keys={0: key(c, torch.int32)}),
])
def test_refused_by_the_binding(ctx, call):
    with pytest.raises(CkksError):
        call(ctx)


def append(c, k=None, v=None, tables=None, length=0, count=2, keys=None, kp=None, vp=None, table=None, **kw):
    c.cache_append([ct()] if k is None else k, [ct()] if v is None else v, tab(1, 4) if tables is None else tables, 2, 4, 4,
                   length, count, {} if keys is None else keys, [ct(1)] if kp is None else kp,
                   [ct(1)] if vp is None else vp, [[0]] if table is None else table, **kw)


def test_a_well_formed_call_reaches_the_library(ctx):
    """The counterpart of the refusals: nothing above is refused for another reason than its own."""
    for call in (lambda c: append(c), lambda c: append(c, fork=[0], src=0),
                 lambda c: c.rope([ct()], tab(3), 2, 4, 4, {2: key(c), 6: key(c)}, outs=[ct(1)]),
                 lambda c: c.rope_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 2, out=tab(3)),
                 lambda c: c.cache_tables(f64(2, 2), f64(2, 2), 2, 4, 4, 1, 2, 2, out=tab(2, 4)),
                 lambda c: c.rope_cos_sin(torch.zeros(3, dtype=torch.int64), f64(2))):
        with pytest.raises(AssertionError, match="the library was called"):
            call(ctx)


def test_nothing_to_do_is_not_an_error(ctx):
    assert ctx.rope([], tab(3), 2, 4, 4, {}) == []
    append(ctx, k=[], v=[], table=[])
    append(ctx, count=0)


def test_steps():
    assert Context.rope_steps(2048, 16, 64) == [32, 2016]
    assert Context.rope_steps(2048, 16, 64, pairing="interleaved") == [1, 2047]
    assert Context.rope_steps(2048, 16, 64, layout="fm") == [512, 1536]
    assert Context.rope_steps(2048, 16, 128, layout="fm") == [1024]
    assert Context.append_steps(2048, 16, 64, 7, 7) == [32, 2016]
    assert Context.append_steps(2048, 16, 64, 18, 0) == sorted([2048 - 256, 2048 - 256 + 32, 2048 - 256 - 32])
    assert Context.append_steps(2048, 16, 0, 2, 5) == [2048 - 13 * 128]
    assert Context.append_steps(2048, 16, 0, 32, 0) == []


def test_inv_freq():
    f = rope_inv_freq(8, base=10000.0)
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(rope_inv_freq(8, scaling="linear", factor=4.0), f / 4)
    n = rope_inv_freq(8, scaling="ntk", factor=4.0)
    assert n[0] == 1.0 and abs(n[-1] * 4 / f[-1] - 1) < 1e-14
    b = rope_inv_freq(128, base=500000.0, scaling="bands", factor=8.0, original=8192)
    p = rope_inv_freq(128, base=500000.0)
    turns = 8192 * p / (2 * math.pi)
    assert torch.equal(b[turns > 4], p[turns > 4]) and torch.allclose(b[turns < 1], p[turns < 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and (b[mid] < p[mid]).all() and (b[mid] > p[mid] / 8).all()
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, base=0.0), dict(rot_dim=8, scaling="linear", factor=0.0),
                dict(rot_dim=8, scaling="other"), dict(rot_dim=8, scaling="bands", low=4.0, high=1.0)):
        with pytest.raises(CkksError):
            rope_inv_freq(**bad)


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_the_transposed_rotation_is_the_gradient(pairing):
    """d/dx of <w, rope(x)> is rope(w) with -sin, by the formula and by differences (linear in x: exact to rounding)."""
    g = np.random.default_rng(7)
    x, w = g.normal(size=(2, 3, 2, 8))
    a = g.uniform(-3, 3, (3, 3))
    grad = plain_rope(w, np.cos(a), -np.sin(a), pairing)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = 1.0
        diff = np.sum(w * (plain_rope(x + d, np.cos(a), np.sin(a), pairing) - plain_rope(x, np.cos(a), np.sin(a), pairing)))
        assert abs(diff - grad[i]) < 1e-12


@pytest.mark.parametrize("logs", [6, 7, 8])
def test_the_sums_column_pass_stays_in_its_bounds(logs):
    """In units of q: a reducing stage maps a bound b to 1 + 0.375 b, a lazy one to 0.5 + 1.375 b; the converted values are
    at most q / 2, every value stays below 8 q and the rows that the row pass takes below its 4.3 q."""
    import os
    import re
    path = os.path.join(os.path.dirname(__file__), "..", "paper_2609_12378_amd", "csrc", "wsum.hip")
    body = re.search(r"constexpr unsigned quot_col_mask\(int logs\)\s*\{\s*return (.*?);", open(path).read(), re.S).group(1)
    masks = {int(k): int(v, 16) for k, v in re.findall(r"== (\d) \? (0x[0-9a-f]+)", body)}
    mask = masks.get(logs, int(re.search(r"(0x[0-9a-f]+)\s*$", body).group(1), 16))
    b = peak = 0.5
    for s in range(logs):
        b = (1 + 0.375 * b if (mask >> s) & 1 else 1.375 * b + 0.5) * (1 + 2.0 ** -40)
        peak = max(peak, b)
    assert peak < 8 and b < 2

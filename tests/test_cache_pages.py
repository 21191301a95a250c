"""An append sees of a pool the pages that it writes and the ones that it forks, on the CPU: a stand-in for the library
that does what the call documents of its descriptors (the written pages' scales become the new tokens') and notes what
it was handed."""
import ctypes

import pytest
import torch

import paper_2609_12378_amd as pkg
from paper_2609_12378_amd import Buf, CkksError, Context
from test_binding_args import _host_ptr

N, T = 16, 2


class Library:
    """ckks_cache_append's bookkeeping: pages by the block table, scales of the written ones."""

    def __init__(self):
        self.calls = []

    def ckks_cache_append(self, h, k, v, heads, shape, src, length, count, tables, ks, kp, nk, cache, fork):
        c = cache._obj
        first, blocks = length // T, (length + count - 1) // T - length // T + 1
        pages = [c.table[i * c.n_blocks + b] for i in range(heads) for b in range(first, first + blocks)
                 if b < c.n_blocks]
        if c.n_blocks < first + blocks or any(p >= c.n_pages for p in pages + [fork[i] for i in range(heads) if fork]):
            return 1
        seen = {"k": {}, "v": {}}
        for name, pool, x in (("k", c.k_pages, k), ("v", c.v_pages, v)):
            for i in range(heads):
                for b in range(blocks):
                    p = c.table[i * c.n_blocks + first + b]
                    seen[name][p] = (pool[p].data, pool[p].scale)
                    if b == 0 and length % T and fork:
                        seen[name][fork[i]] = (pool[fork[i]].data, pool[fork[i]].scale)
            for i in range(heads):
                for b in range(blocks):
                    pool[c.table[i * c.n_blocks + first + b]].scale = x[i].scale
        self.calls.append(seen)
        return 0


@pytest.fixture
def ctx(monkeypatch):
    monkeypatch.setattr(pkg, "_ptr", _host_ptr)
    c = Context.__new__(Context)
    c.lib, c.h, c._stream, c.device = Library(), ctypes.c_void_p(), None, 0
    c.log_n, c.n, c.n_q, c.n_p, c.dnum, c.alpha = 4, N, 3, 1, 2, 2
    c.q, c.p = [97, 193, 257], [353]
    c.primes = c.q + c.p
    monkeypatch.setattr(Context, "__del__", lambda self: None)
    return c


class Counted(Buf):
    """A page that counts how often it is described to the library."""
    described = 0

    def c(self, n=None):
        self.described += 1
        return super().c(n)


def page(scale=1.0, kind=Buf):
    return kind(torch.zeros((2, 1, N), dtype=torch.uint64), scale)


def append(ctx, kp, vp, table, length=0, count=2, scale=8.0, fork=None):
    heads = len(table)
    x = [Buf(torch.zeros((2, 2, N), dtype=torch.uint64), scale) for _ in range(heads)]
    blocks = (length + count - 1) // T - length // T + 1
    tables = torch.zeros((blocks, 1, 3, N), dtype=torch.uint64)
    ctx.cache_append(x, x, tables, T, 4, 0, length, count, {}, kp, vp, table, fork=fork)


def test_a_page_that_the_pool_holds_twice_gets_the_new_scale(ctx):
    """Two indices may name one buffer; the one that is not written says nothing of it."""
    a, b, c = page(3.0), page(), page(3.0)
    append(ctx, [a, b, a], [c, b, c], [[0]])
    assert a.scale == c.scale == 8.0 and b.scale == 1.0


def test_other_pages_scales_are_not_written(ctx):
    """A page that another call changes meanwhile keeps what that call gave it."""
    pools = [[page(), page()] for _ in range(2)]
    real = ctx.lib.ckks_cache_append

    def meanwhile(*args):
        pools[0][1].scale = 77.0
        return real(*args)

    ctx.lib.ckks_cache_append = meanwhile
    append(ctx, pools[0], pools[1], [[0]])
    assert [p.scale for p in pools[0]] == [8.0, 77.0] and [p.scale for p in pools[1]] == [8.0, 1.0]


def test_pages_of_no_concern_may_be_missing(ctx):
    """Pages not yet made, and pages of another level or ring, beside the written and the forked one."""
    other = Buf(torch.zeros((2, 3, 8), dtype=torch.uint64), 1.0)
    pools = [[None, page(), other, page(8.0), None] for _ in range(2)]
    append(ctx, *pools, [[4, 1]], length=T, count=2)
    append(ctx, *pools, [[4, 1]], length=T + 1, count=1, fork=[3])
    for pool in pools:
        assert pool[1].scale == 8.0 and pool[3].scale == 8.0
    for seen in ctx.lib.calls[1].values():
        assert sorted(seen) == [1, 3] and all(data for data, _ in seen.values())
    for bad in ([[0]], [[5]], [[2]]):       # but a written or forked one may not
        with pytest.raises(CkksError):
            append(ctx, *pools, bad)
    with pytest.raises(CkksError):
        append(ctx, *pools, [[1]], length=1, count=1, fork=[0])
    with pytest.raises(CkksError):
        append(ctx, *pools, [[1]], length=1, count=1, fork=[5])
    assert len(ctx.lib.calls) == 2


def test_the_call_describes_the_pages_it_touches_alone(ctx):
    """Two heads over a page border in a long context: four pages of each pool, and the forked one."""
    pools = [[page(8.0, Counted) for _ in range(1000)] for _ in range(2)]
    length = 400 * T + 1
    table = [list(range(h * 450, h * 450 + 402)) for h in range(2)]
    append(ctx, *pools, table, length=length, count=2, fork=[990, 990])
    touched = {400, 401, 850, 851, 990}
    for pool in pools:
        assert {i for i, p in enumerate(pool) if p.described} == touched


def test_a_short_table_reaches_the_library_as_it_is(ctx):
    """The library, which knows the blocks that it needs, refuses it."""
    with pytest.raises(CkksError, match="failed"):
        append(ctx, [page()], [page()], [[0]], length=T, count=1)

"""Calls of more ciphertexts than a batch of 16 takes: every output against the same ciphertext's in a call of its own,
and those on either side of each border of 16 against the oracle's stages.
"""
import pytest

from gpu_common import to_dev, to_host
from rope_common import random_cts, random_keys, term_steps, weighted
from test_gpu_rope import angles, bufs, dev_keys, ring, same

pytestmark = pytest.mark.gpu

BATCH = 16
RINGS = [((8, 5, 2, 3, 36), 8, 16, 4),       # integers, single-pass transforms
         ((12, 4, 2, 2, 36), 16, 64, 4),     # whole rows a block
         ((12, 4, 2, 2, 59), 16, 64, 3),     # integers
         ((13, 6, 2, 3, 50), 16, 128, 5),
         ((14, 4, 1, 4, 36), 64, 32, 4),     # two passes, conversions with their column pass
         ((16, 4, 2, 2, 50), 128, 128, 3)]   # two passes, column passes in the conversions
ids = dict(ids=lambda c: "n%d-b%d" % (c[0], c[4]) if isinstance(c, tuple) else str(c))


def borders(n):
    return [i for b in range(BATCH, n + 1, BATCH) for i in (b - 1, b) if i < n]


@pytest.mark.parametrize("chain,T,hd,limbs", RINGS, **ids)
def test_every_ciphertext_of_rope(chain, T, hd, limbs):
    ctx, ck = ring(*chain)
    count = 35
    steps = term_steps(ck.n, T, hd, "tm", "half")
    keys = random_keys(ck, steps, 121)
    dk = dev_keys(keys)
    tables = ctx.rope_tables(*(to_dev(x) for x in angles(T, hd // 2, 122)), T, hd, hd, limbs)
    xs = random_cts(ck, limbs, count, 123)
    got = ctx.rope(bufs(xs), tables, T, hd, hd, dk)
    tabs = to_host(tables)
    for i, x in enumerate(xs):
        same(got[i].data, to_host(ctx.rope(bufs([x]), tables, T, hd, hd, dk)[0].data), "ciphertext %d" % i)
        if i in borders(count):
            same(got[i].data, weighted(ck, x, steps, keys, tabs), "ciphertext %d" % i)


@pytest.mark.parametrize("moved", [True, False], ids=["moved", "in-place"])
@pytest.mark.parametrize("chain,T,hd,limbs", RINGS, **ids)
def test_every_page_of_an_append(chain, T, hd, limbs, moved):
    """17 heads, keys then values: batches of 16, 16 and 2, the middle one of both kinds (the integer sums take rotated
    and unrotated ones apart).  Over a page border, or a token in its own slot, whose values are not rotated."""
    ctx, ck = ring(*chain)
    heads, length = 17, 2 * T - 2
    src, count = (0, 3) if moved else (T - 2, 1)
    shift = (length - src) % T
    steps = term_steps(ck.n, T, hd, "tm", "half", shift)
    keys = random_keys(ck, steps, 131)
    dk = dev_keys(keys)
    tables = ctx.cache_tables(*(to_dev(x) for x in angles(count, hd // 2, 132)), T, hd, hd, length, count, limbs)
    tabs = to_host(tables)
    blocks = tabs.shape[0]
    x = [random_cts(ck, limbs, heads, 133 + i) for i in range(2)]
    old = [random_cts(ck, limbs - 1, heads, 135 + i) for i in range(2)]
    new = random_cts(ck, limbs - 1, 1, 137)

    def append(which):
        """The pages of each of these heads, [head][kv][block]."""
        pools = [bufs([old[i][h] for h in which] + new * len(which)) for i in range(2)]
        n = len(which)
        k, v = (bufs([x[i][h] for h in which]) for i in range(2))
        ctx.cache_append(k, v, tables, T, hd, hd, length, count, dk, *pools,
                         [[0, h, n + h][:1 + blocks] for h in range(n)], src=src)
        return [[[to_host(pools[i][h + b * n].data) for b in range(blocks)] for i in range(2)] for h in range(n)]

    got = append(range(heads))
    for h in range(heads):
        want = append([h])[0]
        for i in range(2):
            at = i * heads + h                     # keys first, then values
            for b in range(blocks):
                assert (got[h][i][b] == want[i][b]).all(), ("kv"[i], h, b)
                if at not in borders(2 * heads):
                    continue
                st, tab = ((steps, tabs[b][:3]), (steps[:1], tabs[b][3:]))[i]
                w = weighted(ck, x[i][h], st, keys, tab)
                assert (got[h][i][b] == (w if b else ck.ct_add(w, old[i][h]))).all(), ("kv"[i], h, b)

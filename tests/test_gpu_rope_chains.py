"""Rotary positions and cache appends in fp64 chains whose primes differ in size, bit for bit against the oracle's
stages: some digits' conversions are in fp64 and some in integers, and the sums are in integers over fp64 rows.
"""
import numpy as np
import pytest

from gpu_common import to_dev, to_host
from rope_common import random_cts, random_keys, term_steps, weighted
from test_gpu_mixed_chains import Chain
from test_gpu_rope import angles, bufs, dev_keys, same

pytestmark = pytest.mark.gpu

_CHAINS = {}


def chain(log_n, kind):
    if (log_n, kind) not in _CHAINS:
        _CHAINS.clear()
        _CHAINS[log_n, kind] = Chain(log_n, kind)
    env = _CHAINS[log_n, kind]
    return env.ctx, env.ck


@pytest.mark.parametrize("log_n", [12, 13, 15, 16])
@pytest.mark.parametrize("kind,limbs", [("special50", 4), ("base50", 4), ("base50", 3), ("base50", 2),
                                        ("sources17", 5)])
def test_rope_and_append(log_n, kind, limbs):
    """base50: the first digit's conversion is in integers, and with 3 or 4 limbs the last one's in fp64."""
    ctx, ck = chain(log_n, kind)
    T, hd, rot, count, length = 16, 64, 64, 2, 13
    steps = term_steps(ck.n, T, rot, "tm", "half")
    moved = term_steps(ck.n, T, rot, "tm", "half", length)
    keys = random_keys(ck, steps + moved, 101)
    dk = dev_keys(keys)
    cos, sin = (to_dev(x) for x in angles(T, rot // 2, 102))
    tables = ctx.rope_tables(cos, sin, T, hd, rot, limbs)
    tabs = to_host(tables)
    xs = random_cts(ck, limbs, 3, 103)
    for x, o in zip(xs, ctx.rope(bufs(xs), tables, T, hd, rot, dk)):
        same(o.data, weighted(ck, x, steps, keys, tabs), "rope")
    n = 5                                          # tokens 13 .. 17 from slot 0: over the page border
    ct = ctx.cache_tables(cos[:n].contiguous(), sin[:n].contiguous(), T, hd, rot, length, n, limbs)
    old = random_cts(ck, limbs - 1, 4, 104)
    pools = [bufs(old), bufs(old)]
    ctx.cache_append(bufs(xs[:count]), bufs(xs[1:]), ct, T, hd, rot, length, n, dk, *pools, [[3, 1], [0, 2]])
    ct = to_host(ct)
    for i, (st, tab) in enumerate([(moved, ct[:, :3]), (moved[:1], ct[:, 3:])]):
        for h, pages in enumerate([(3, 1), (0, 2)]):
            for b, p in enumerate(pages):
                want = weighted(ck, xs[h + i], st, keys, tab[b])
                same(pools[i][p].data, want if b else ck.ct_add(want, old[p]), "%s page %d" % ("kv"[i], p))


@pytest.mark.parametrize("log_n", [12, 13, 14, 15])
@pytest.mark.parametrize("kind,limbs", [("base50", 4), ("sources17", 17)])
def test_the_digits_own_rows_are_not_transformed(log_n, kind, limbs):
    """A digit's own rows hold what the ciphertext does and are read there: of the scratch, which the sums in integers
    use whole, exactly these rows - as many as the ciphertexts have limbs - are never written."""
    import torch
    ctx, ck = chain(log_n, kind)
    T, hd, count = 16, 64, 3
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half"), 111))
    tables = ctx.rope_tables(*(to_dev(x) for x in angles(T, hd // 2, 112)), T, hd, hd, limbs)
    xs = random_cts(ck, limbs, count, 113)
    want = [to_host(b.data) for b in ctx.rope(bufs(xs), tables, T, hd, hd, keys)]
    mark = 0x5A5A5A5A5A5A5A5A
    ws = torch.full((ctx.workspace_bytes(ctx.OP_ROPE, (limbs, count)) // 8 // ck.n, ck.n), mark, dtype=torch.int64,
                    device="cuda")
    ctx.set_workspace(ws.view(torch.uint64))
    try:
        got = [to_host(b.data) for b in ctx.rope(bufs(xs), tables, T, hd, hd, keys)]
    finally:
        ctx.set_workspace(None)
    assert all(np.array_equal(g, w) for g, w in zip(got, want))
    rows = int((ws == mark).all(1).sum())
    assert rows == count * limbs

"""Calls of rope and cache_append that their description allows at its edges: pages of one token and of all slots, keys
named by other representatives of their steps, a fork in place, the arithmetic switched under a workspace, and two
contexts that append to one pool at once.
"""
import numpy as np
import pytest

from gpu_common import to_dev, to_host
from rope_common import random_cts, random_keys, term_steps, weighted
from test_gpu_rope import angles, bufs, dev_keys, ring, run_append, same

pytestmark = pytest.mark.gpu

APPEND = [
    # log_n n_q n_p dnum bits limbs tokens hd rot pairing heads length count src fork
    (5, 4, 2, 2, 50, 3, 1, 8, 8, "half", 2, 3, 1, 0, False),         # a page a token
    (12, 4, 2, 2, 36, 2, 1, 2048, 2048, "half", 1, 5, 1, 0, False),
    (5, 4, 2, 2, 50, 3, 16, 1, 0, "half", 2, 21, 16, 0, True),       # a feature a token: every slot another token
    (12, 4, 2, 2, 36, 3, 2048, 1, 0, "half", 1, 2049, 2047, 1, False),
    (13, 6, 2, 3, 50, 4, 2048, 2, 2, "interleaved", 2, 100, 1, 100, True),   # a fork in the token's own slot
    (14, 6, 2, 3, 50, 5, 64, 128, 128, "half", 2, 63, 1, 63, True),  # the page's last slot
    (16, 4, 2, 2, 50, 3, 32768, 1, 0, "half", 1, 70000, 9, 32000, False),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "n%d-%d+%d-d%d-b%d-l%d-t%d-h%d-r%d-%s-x%d-at%d-n%d-s%d-f%d" % c)
def test_append_at_the_edges(case):
    run_append(case)


@pytest.mark.parametrize("chain,T,hd", [((12, 4, 2, 2, 36), 16, 64), ((14, 6, 2, 3, 50), 64, 128)], ids=["n12", "n14"])
def test_keys_by_any_representative(chain, T, hd):
    """Steps are taken modulo N/2, and keys that no term needs do not matter."""
    ctx, ck = ring(*chain)
    slots, limbs = ck.n // 2, 4
    steps = term_steps(ck.n, T, hd, "tm", "half")
    keys = random_keys(ck, steps + [1, 3], 161)
    tables = ctx.rope_tables(*(to_dev(x) for x in angles(T, hd // 2, 162)), T, hd, hd, limbs)
    x = random_cts(ck, limbs, 1, 163)
    want = weighted(ck, x[0], steps, keys, to_host(tables))
    dk = dev_keys(keys)
    h = hd // 2
    for named in ({h: dk[h], -h: dk[slots - h]}, {h - slots: dk[h], 3 * slots - h: dk[slots - h], 1: dk[1], 3: dk[3]}):
        same(ctx.rope(bufs(x), tables, T, hd, hd, named)[0].data, want, "rope")


@pytest.mark.parametrize("chain,T,hd,limbs", [((12, 4, 2, 2, 36), 16, 64, 4), ((14, 6, 2, 3, 50), 64, 128, 5)],
                         ids=["n12", "n14"])
def test_a_workspace_serves_both_arithmetics(chain, T, hd, limbs):
    import torch
    ctx, ck = ring(*chain)
    count = 3
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half"), 171))
    tables = ctx.rope_tables(*(to_dev(x) for x in angles(T, hd // 2, 172)), T, hd, hd, limbs)
    xs = random_cts(ck, limbs, count, 173)
    want = [to_host(b.data) for b in ctx.rope(bufs(xs), tables, T, hd, hd, keys)]
    size = ctx.workspace_bytes(ctx.OP_ROPE, (limbs, count))
    mem = torch.full((size // 8 + 64,), 7, dtype=torch.int64, device="cuda")
    ctx.set_workspace(mem[:size // 8].view(torch.uint64))
    try:
        for mode in (1, 0, 1):
            ctx.set_ntt_arith(mode)
            assert ctx.workspace_bytes(ctx.OP_ROPE, (limbs, count)) == size
            for b, w in zip(ctx.rope(bufs(xs), tables, T, hd, hd, keys), want):
                same(b.data, w, "arithmetic %d" % mode)
    finally:
        ctx.set_ntt_arith(0)
        ctx.set_workspace(None)
    assert bool((mem[size // 8:] == 7).all())


def test_two_contexts_append_to_one_pool():
    """Two sequences of one pool, each on a context and a stream of its own, sharing their prompt's page: many steps
    queued without waits between the contexts."""
    import torch
    from paper_2609_12378_amd import Context
    eager, ck = ring(14, 6, 2, 3, 50)
    T, hd, limbs, n = 64, 128, 4, 6
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half"), 181))
    cos, sin = (to_dev(x) for x in angles(n, hd // 2, 182))
    tables = [eager.cache_tables(cos[t:t + 1].contiguous(), sin[t:t + 1].contiguous(), T, hd, hd, T + 5 + t, 1, limbs)
              for t in range(n)]
    x = [[bufs(random_cts(ck, limbs, 2, 183 + 10 * i + t)) for t in range(n)] for i in range(2)]
    old = random_cts(ck, limbs - 1, 4, 184)

    def run(contexts):
        pools = [bufs(old) for _ in range(2)]
        torch.cuda.synchronize()
        for t in range(n):
            for i, c in enumerate(contexts):
                c.cache_append(x[i][t][:1], x[i][t][1:], tables[t], T, hd, hd, T + 5 + t, 1, keys, *pools,
                               [[0, 2 + i]], src=5 + t, fork=None if t else [1])
        torch.cuda.synchronize()
        return [[to_host(p.data) for p in pool] for pool in pools]

    want = run([eager, eager])
    both = [Context(ck.log_n, ck.n_q, ck.n_p, ck.dnum, q=eager.q, p=eager.p, stream=torch.cuda.Stream())
            for _ in range(2)]
    for _ in range(3):
        got = run(both)
        for i in range(2):
            for p in range(4):
                assert np.array_equal(got[i][p], want[i][p]), ("kv"[i], p)

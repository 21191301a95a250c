"""Rotary positions and the cache on both sides of the rules that choose their kernels, bit for bit against the oracle's
stages: numbers of digits, special primes and ciphertexts, primes at the ends of the arithmetics, rings below 2^12 points,
and ciphertexts, tables and pages that start at an odd word.
"""
import numpy as np
import pytest

from rope_common import random_cts, random_keys, term_steps, weighted
from test_gpu_rope import angles, dev_keys, ring, run_append, run_rope, same
from gpu_common import to_dev, to_host

pytestmark = pytest.mark.gpu

ROPE = [
    # log_n n_q n_p dnum bits limbs tokens hd rot layout pairing count
    (11, 4, 2, 2, 59, 4, 16, 32, 32, "tm", "half", 2),
    (11, 6, 1, 6, 50, 6, 16, 32, 32, "tm", "interleaved", 2),   # fp64 primes in exact sums: six digits
    (12, 6, 1, 6, 50, 6, 16, 64, 64, "tm", "half", 2),
    (13, 6, 1, 6, 45, 5, 16, 64, 64, "tm", "half", 3),          # five of its six digits
    (14, 7, 1, 7, 45, 7, 64, 64, 64, "tm", "half", 2),
    (12, 10, 1, 10, 59, 10, 16, 64, 64, "tm", "half", 2),       # more than eight products a sum
    (12, 9, 1, 9, 62, 9, 16, 64, 64, "tm", "half", 1),          # the same at the largest primes
    (12, 10, 9, 1, 62, 10, 16, 64, 64, "fm", "half", 2),        # more than eight of them a conversion
    (12, 8, 8, 1, 60, 8, 16, 64, 64, "tm", "half", 2),          # eight at the largest primes of the split sums
    (13, 8, 8, 1, 61, 8, 16, 64, 64, "tm", "half", 2),          # and above them
    (12, 3, 17, 1, 59, 3, 16, 64, 64, "tm", "half", 2),
    (12, 4, 17, 2, 36, 4, 16, 64, 64, "tm", "half", 2),         # too many special primes for the fp64 conversions
    (14, 4, 1, 4, 50, 4, 64, 128, 128, "tm", "half", 3),
    (14, 5, 1, 5, 50, 5, 64, 128, 128, "tm", "half", 2),
    (15, 10, 8, 2, 50, 10, 128, 128, 128, "tm", "half", 16),    # conversions of many reads, in two launches
    (15, 10, 10, 1, 45, 10, 128, 128, 128, "tm", "half", 16),
    (16, 4, 2, 2, 50, 4, 128, 128, 128, "tm", "half", 9),       # a block for every CU: the columns go along
    (16, 9, 8, 2, 50, 4, 128, 128, 128, "fm", "half", 8),
    (16, 9, 8, 2, 50, 9, 128, 128, 128, "tm", "half", 1),
    (16, 10, 8, 2, 59, 3, 128, 128, 128, "tm", "half", 4),
]


@pytest.mark.parametrize("case", ROPE, ids=lambda c: "n%d-%d+%d-d%d-b%d-l%d-t%d-h%d-r%d-%s-%s-x%d" % c)
def test_rope_of_either_rule(case):
    run_rope(case)


APPEND = [
    # log_n n_q n_p dnum bits limbs tokens hd rot pairing heads length count src fork
    (11, 4, 2, 2, 59, 4, 16, 32, 32, "half", 2, 13, 9, 2, True),
    (12, 10, 1, 10, 59, 9, 16, 64, 64, "interleaved", 2, 13, 9, 2, False),
    (12, 10, 1, 10, 59, 9, 16, 64, 64, "half", 2, 13, 3, 13, False),
    (13, 6, 1, 6, 45, 6, 16, 128, 64, "half", 3, 13, 9, 2, True),
    (12, 4, 2, 2, 36, 4, 16, 64, 48, "interleaved", 17, 13, 9, 2, False),   # 34 ciphertexts of two pages: three batches
    (13, 6, 2, 3, 50, 6, 16, 128, 128, "interleaved", 2, 15, 1, 15, True),
    (14, 5, 1, 5, 50, 5, 64, 128, 128, "half", 2, 60, 64, 0, False),
    (15, 10, 8, 2, 50, 9, 128, 128, 128, "half", 8, 130, 5, 0, False),
    (16, 4, 2, 2, 50, 3, 128, 128, 128, "half", 4, 120, 20, 0, True),       # 32 outputs' polynomials
    (16, 9, 8, 2, 50, 4, 128, 128, 128, "half", 8, 7, 1, 7, False),         # rotated keys, values in their slots
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "n%d-%d+%d-d%d-b%d-l%d-t%d-h%d-r%d-%s-x%d-at%d-n%d-s%d-f%d" % c)
def test_append_of_either_rule(case):
    run_append(case)


def odd_words(arrays, scale=2.0 ** 40):
    """Buffers that start one word after the allocation."""
    import torch
    from paper_2609_12378_amd import Buf
    out = []
    for a in arrays:
        flat = torch.empty(a.size + 1, dtype=torch.uint64, device="cuda")
        view = flat[1:].view(*a.shape)
        view.copy_(to_dev(a))
        assert view.data_ptr() % 16 == 8
        out.append(Buf(view, scale))
    return out


@pytest.mark.parametrize("chain,T,hd,limbs", [((9, 4, 2, 2, 36), 8, 16, 4), ((12, 4, 2, 2, 36), 16, 64, 4),
                                              ((12, 4, 2, 2, 59), 16, 64, 4), ((13, 6, 2, 3, 50), 16, 128, 6),
                                              ((14, 6, 2, 3, 50), 64, 128, 5), ((16, 4, 2, 2, 50), 128, 128, 3)],
                         ids=lambda c: "n%d-b%d" % (c[0], c[4]) if isinstance(c, tuple) else str(c))
def test_buffers_at_an_odd_word(chain, T, hd, limbs):
    ctx, ck = ring(*chain)
    steps = term_steps(ck.n, T, hd, "tm", "half")
    moved = term_steps(ck.n, T, hd, "tm", "half", T - 3)
    keys = random_keys(ck, steps + moved, 31)
    dk = {s: b.data for s, b in zip(keys, odd_words([keys[s] for s in keys]))}
    cos, sin = (to_dev(x) for x in angles(T, hd // 2, 33))
    tables = to_host(ctx.rope_tables(cos, sin, T, hd, hd, limbs))
    xs = random_cts(ck, limbs, 2, 34)
    old = random_cts(ck, limbs - 1, 8, 35)
    outs = odd_words(old[:2])
    ctx.rope(odd_words(xs), odd_words([tables])[0].data, T, hd, hd, dk, outs=outs)
    for x, o in zip(xs, outs):
        same(o.data, weighted(ck, x, steps, keys, tables), "rope")
    n = 6                                                            # tokens T - 3 .. T + 2
    ct = to_host(ctx.cache_tables(cos[:n].contiguous(), sin[:n].contiguous(), T, hd, hd, T - 3, n, limbs))
    pools = [odd_words(old[:4]), odd_words(old[4:])]
    ctx.cache_append(odd_words(xs[:1]), odd_words(xs[1:]), odd_words([ct])[0].data, T, hd, hd, T - 3, n, dk, *pools,
                     [[2, 1]])
    for i, (st, tab) in enumerate([(moved, ct[:, :3]), (moved[:1], ct[:, 3:])]):
        for b, p in enumerate((2, 1)):
            want = weighted(ck, xs[i], st, keys, tab[b])
            same(pools[i][p].data, want if b else ck.ct_add(want, old[4 * i + 2]), "page %d" % p)
        same(pools[i][0].data, old[4 * i], "a page that is not touched")


def test_two_contexts_at_once():
    """Two contexts of one ring on streams of their own, their calls queued without waits between them."""
    import torch
    from paper_2609_12378_amd import Buf, Context
    eager, ck = ring(14, 6, 2, 3, 50)
    T, hd, limbs = 64, 128, 6
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half"), 41))
    cos, sin = (to_dev(x) for x in angles(T, hd // 2, 42))
    tables = eager.rope_tables(cos, sin, T, hd, hd, limbs)
    xs = [random_cts(ck, limbs, 3, 43 + i) for i in range(2)]
    cts = [[Buf(to_dev(a), 1.0) for a in x] for x in xs]
    want = [[to_host(b.data) for b in eager.rope(c, tables, T, hd, hd, keys)] for c in cts]
    both = [Context(ck.log_n, ck.n_q, ck.n_p, ck.dnum, q=eager.q, p=eager.p, stream=torch.cuda.Stream()) for _ in range(2)]
    torch.cuda.synchronize()
    got = [[both[i].rope(cts[i], tables, T, hd, hd, keys) for i in range(2)] for _ in range(6)]
    torch.cuda.synchronize()
    for run in got:
        for i in range(2):
            for g, w in zip(run[i], want[i]):
                assert np.array_equal(to_host(g.data), w)


@pytest.mark.parametrize("chain,T,hd,limbs", [((12, 4, 2, 2, 36), 16, 64, 4), ((14, 6, 2, 3, 50), 64, 128, 5),
                                              ((16, 4, 2, 2, 59), 128, 128, 3)], ids=lambda c: "n%d" % c[0]
                         if isinstance(c, tuple) else str(c))
def test_a_ciphertext_given_twice(chain, T, hd, limbs):
    """Inputs may repeat: two outputs of one ciphertext, and one ciphertext as the key and the value of two heads."""
    from paper_2609_12378_amd import Buf
    ctx, ck = ring(*chain)
    steps, moved = term_steps(ck.n, T, hd, "tm", "half"), term_steps(ck.n, T, hd, "tm", "half", 2)
    keys = random_keys(ck, steps + moved, 51)
    dk = dev_keys(keys)
    cos, sin = (to_dev(x) for x in angles(T, hd // 2, 52))
    x = random_cts(ck, limbs, 1, 53)[0]
    b = Buf(to_dev(x), 2.0 ** 40)
    tables = ctx.rope_tables(cos, sin, T, hd, hd, limbs)
    want = weighted(ck, x, steps, keys, to_host(tables))
    for out in ctx.rope([b, b], tables, T, hd, hd, dk):
        same(out.data, want, "rope")
    ct = ctx.cache_tables(cos[:3].contiguous(), sin[:3].contiguous(), T, hd, hd, 2, 3, limbs)
    old = random_cts(ck, limbs - 1, 4, 54)
    pools = [[Buf(to_dev(a), 2.0 ** 40) for a in old] for _ in range(2)]
    ctx.cache_append([b, b], [b, b], ct, T, hd, hd, 2, 3, dk, *pools, [[1], [3]], fork=[0, 0])
    tab = to_host(ct)[0]
    for i, (st, t) in enumerate([(moved, tab[:3]), (moved[:1], tab[3:])]):
        want = ck.ct_add(weighted(ck, x, st, keys, t), old[0])
        for p in (1, 3):
            same(pools[i][p].data, want, "page %d" % p)
        for p in (0, 2):
            same(pools[i][p].data, old[p], "page %d" % p)


@pytest.mark.parametrize("chain,T,limbs,count", [((16, 4, 2, 2, 50), 128, 4, 9), ((16, 4, 3, 2, 59), 128, 3, 2),
                                                 ((15, 6, 2, 3, 50), 128, 5, 2)], ids=lambda c: "n%d-b%d" % (c[0], c[4])
                         if isinstance(c, tuple) else str(c))
def test_large_rings_captured(chain, T, limbs, count):
    import torch
    from paper_2609_12378_amd import Buf, Context
    eager, ck = ring(*chain)
    hd = 128
    stream = torch.cuda.Stream()
    ctx = Context(ck.log_n, ck.n_q, ck.n_p, ck.dnum, q=eager.q, p=eager.p, stream=stream)
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half"), 61))
    cos, sin = (to_dev(x) for x in angles(T, hd // 2, 62))
    tables = eager.rope_tables(cos, sin, T, hd, hd, limbs)
    x = [Buf(torch.zeros((2, limbs, ck.n), dtype=torch.uint64, device="cuda"), 1.0) for _ in range(count)]
    ws = torch.empty(ctx.workspace_bytes(ctx.OP_ROPE, (limbs, count)) // 8, dtype=torch.uint64, device="cuda")
    ctx.set_workspace(ws)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        ctx.rope(x, tables, T, hd, hd, keys)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = ctx.rope(x, tables, T, hd, hd, keys)
    torch.cuda.synchronize()
    for r in range(3):
        for b, a in zip(x, random_cts(ck, limbs, count, 63 + r)):
            b.data.copy_(to_dev(a))
        want = eager.rope(x, tables, T, hd, hd, keys)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(out, want):
            same(o.data, to_host(w.data), "replay %d" % r)
        junk = torch.randn(1 << 22, device="cuda").sum()
        del junk
    del graph

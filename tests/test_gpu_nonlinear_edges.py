"""Polynomials, norms and the projection's epilogue at the edges of what they allow: residues at the ends of their ranges,
buffers and keys that start at an odd word, operands that are one another, primes of 62 bits, scales that leave the doubles."""
import math

import numpy as np
import pytest

import nonlinear_common as nc
from gpu_common import to_dev, to_host
from rope_common import random_cts, random_keys
from test_gpu_nonlinear import SCALE, norm_inputs, plaintexts, proj_keys, rlk_of, some_poly
from test_gpu_rope import bufs, dev_keys, ring, same
from test_gpu_rope_rules import odd_words
from workloads import rng

pytestmark = pytest.mark.gpu


def extremes(ck, lead, primes, seed, mixed):
    """Canonical residues that are q - 1 everywhere, or one of 0, 1, (q - 1) / 2, (q + 1) / 2 and q - 1."""
    g = rng(seed, 3)
    out = np.empty((*lead, len(primes), ck.n), dtype=np.uint64)
    for i, q in enumerate(primes):
        values = np.array([q - 1, 0, 1, q // 2, q // 2 + 1], dtype=np.uint64)
        out[..., i, :] = values[g.integers(0, 5, (*lead, ck.n))] if mixed else values[0]
    return out


EXTREME = [((8, 9, 3, 3, 62), 2.0 ** 60), ((8, 9, 3, 3, 50), SCALE), ((12, 9, 3, 3, 50), SCALE), ((13, 9, 5, 2, 50), SCALE),
           ((14, 9, 3, 3, 50), SCALE), ((10, 9, 9, 1, 59), 2.0 ** 58), ((12, 9, 1, 9, 50), SCALE)]


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("ring_args,scale", EXTREME, ids=str)
def test_residues_at_the_ends_of_their_ranges(ring_args, scale, mixed):
    """Every lazy sum at its largest: a polynomial of nine terms a step, a norm of five ciphertexts with a Newton step."""
    ctx, ck = ring(*ring_args)
    limbs, T = 9, ck.n // 32
    make = lambda lead, primes, seed: extremes(ck, lead, primes, seed, mixed)  # noqa: E731
    xs = [make((2,), ck.q[:limbs], 400 + i) for i in range(5)]
    rlk = make((ck.dnum, 2), ck.primes, 410)
    poly, inv = some_poly(13, 411), some_poly(3, 412, 0.5, 3.0)
    got = ctx.poly_eval(bufs(xs[:2], scale), poly, to_dev(rlk))
    for g, x in zip(got, xs):
        same(g.data, nc.poly_eval(ck, x, scale, poly, rlk), "polynomial")
    st = norm_inputs(ck, limbs, T, "fm", 1, None, None, 420)
    keys = {s: make((ck.dnum, 2), ck.primes, 430 + s) for s in st["keys"]}
    ws = [make((1,), ck.q[:limbs], 440 + i) for i in range(5)]
    x = bufs(xs, scale)
    got = ctx.rms_norm(x, T, 5 * 16, inv, to_dev(rlk), dev_keys(keys), weights=bufs(ws, scale), newton=1, eps=0.5, residual=x)
    want = nc.rms_norm(ck, xs, scale, T, 5 * 16, inv, rlk, keys, "fm", ws, scale, newton=1, eps=0.5, residual=xs,
                       r_scale=scale)
    for g, w in zip(got, want):
        same(g.data, w, "norm")


@pytest.mark.parametrize("ring_args,near", [((8, 8, 3, 3, 50), 1.0), ((12, 8, 3, 3, 50), 1.0), ((14, 8, 3, 3, 50), 1.0),
                                            ((10, 8, 3, 3, 59), 2.0 ** 9)], ids=str)
def test_buffers_at_an_odd_word(ring_args, near):
    from paper_2609_12378_amd import Epilogue
    ctx, ck = ring(*ring_args)
    limbs, T, scale = 8, ck.n // 32, SCALE * near
    xs, rlk, poly = random_cts(ck, limbs, 2, 500), rlk_of(ck, 501), some_poly(9, 502)
    odd = lambda a, s=scale: odd_words(a, s)  # noqa: E731
    outs = odd([np.zeros((2, 3, ck.n), dtype=np.uint64)] * 2)
    k = odd([rlk])[0].data
    ctx.poly_eval(odd(xs), poly, k, outs=outs)
    for g, x in zip(outs, xs):
        same(g.data, nc.poly_eval(ck, x, scale, poly, rlk), "polynomial")
    for layout in ("fm", "tm"):
        st = norm_inputs(ck, limbs, T, layout, 2, "plain", "other", 510)
        inv = some_poly(3, 511, 0.5, 3.0)
        keys = {s: odd([v])[0].data for s, v in st["keys"].items()}
        got = ctx.rms_norm(odd(st["xs"]), T, 2 * 16, inv, odd([st["rlk"]])[0].data, keys, layout=layout,
                           weights=odd(st["ws"]), mask=odd([st["mask"]])[0] if layout == "tm" else None,
                           residual=odd(st["res"]))
        want = nc.rms_norm(ck, st["xs"], scale, T, 2 * 16, inv, st["rlk"], st["keys"], layout, st["ws"], scale, st["mask"],
                           scale, residual=st["res"], r_scale=scale)
        for g, w in zip(got, want):
            same(g.data, w, "norm, %s" % layout)
    keys, W = proj_keys(ck, T, "fm", 5), rng(520, 2).normal(0, 0.02, (16, 16))
    b, gate, res = plaintexts(ck, limbs, 1, 521), random_cts(ck, limbs, 1, 522), random_cts(ck, limbs, 1, 523)
    act = some_poly(3, 524)
    got = ctx.linear_project(odd(xs[:1]), to_dev(W), T, 5, {s: odd([v])[0].data for s, v in keys.items()}, epilogue=Epilogue(
        bias=odd(b), act=act, gate=odd(gate), residual=odd(res), rlk=k))
    want = nc.project(ck, xs[:1], scale, W, T, 5, keys, "fm", rlk, [b[0][0][None]], scale, act, gate, scale, res, scale)
    same(got[0].data, want[0], "projection")


@pytest.mark.parametrize("ring_args", [(8, 8, 3, 3, 50), (12, 8, 3, 3, 50), (14, 8, 3, 3, 50)], ids=str)
def test_operands_that_are_one_another(ring_args):
    """A ciphertext twice in a list, weights and residual that are the input, one gate for two outputs that is their
    residual too."""
    from paper_2609_12378_amd import Epilogue
    ctx, ck = ring(*ring_args)
    limbs, T = 8, ck.n // 32
    x, rlk, poly = random_cts(ck, limbs, 1, 600), rlk_of(ck, 601), some_poly(6, 602)
    two, both = bufs(x, SCALE) * 2, x * 2
    for g in ctx.poly_eval(two, poly, to_dev(rlk)):
        same(g.data, nc.poly_eval(ck, x[0], SCALE, poly, rlk), "polynomial")
    keys, inv = norm_inputs(ck, limbs, T, "fm", 1, None, None, 603)["keys"], some_poly(3, 604, 0.5, 3.0)
    got = ctx.rms_norm(two, T, 20, inv, to_dev(rlk), dev_keys(keys), weights=two, residual=two, residual_scale=2.0)
    want = nc.rms_norm(ck, both, SCALE, T, 20, inv, rlk, keys, "fm", both, SCALE, residual=both, r_scale=SCALE,
                       residual_scale=2.0)
    for g, w in zip(got, want):
        same(g.data, w, "norm")
    keys, W = proj_keys(ck, T, "fm", 16), rng(605, 2).normal(0, 0.02, (32, 32))
    act = some_poly(3, 606)
    got = ctx.linear_project(two, to_dev(W), T, 16, dev_keys(keys), epilogue=Epilogue(act=act, gate=two, residual=two,
                                                                                      rlk=to_dev(rlk)))
    want = nc.project(ck, both, SCALE, W, T, 16, keys, "fm", rlk, None, 1.0, act, both, SCALE, both, SCALE)
    for g, w in zip(got, want):
        same(g.data, w, "projection")


def test_scales_that_leave_the_doubles():
    """Products of scales that overflow or vanish would turn factors into zeros: refused, outputs as they were."""
    from paper_2609_12378_amd import Buf, CkksError, Epilogue
    ctx, ck = ring(8, 8, 3, 3, 50)
    limbs, T = 8, ck.n // 32
    st = norm_inputs(ck, limbs, T, "fm", 1, "plain", None, 700)
    x, inv, old = to_dev(st["xs"][0]), some_poly(3, 701, 0.5, 3.0), random_cts(ck, 3, 1, 702)
    out, rlk, keys = bufs(old, 1.0), to_dev(st["rlk"]), dev_keys(st["keys"])
    w = to_dev(st["ws"][0])
    for scale, w_scale in ((1e200, 1.0), (1e-200, 1.0), (1e150, 1e200), (1e-150, 1e-220), (SCALE, 1e308)):
        with pytest.raises(CkksError, match="scale"):
            ctx.rms_norm([Buf(x, scale)], T, 16, inv, rlk, keys, weights=[Buf(w, w_scale)], outs=out)
    keys, W = dev_keys(proj_keys(ck, T, "fm", 16)), to_dev(rng(703, 2).normal(0, 0.02, (16, 16)))
    x = x[:, :7].contiguous()
    for scale, g_scale in ((1e-200, 1e200), (1e200, 1e-150), (math.inf, 1.0)):
        with pytest.raises(CkksError, match="scale"):
            ctx.linear_project([Buf(x, scale)], W, T, 16, keys, outs=out, epilogue=Epilogue(
                act=inv, gate=[Buf(x, g_scale)], rlk=rlk))
    assert np.array_equal(to_host(out[0].data), old[0])


@pytest.mark.parametrize("log_n,q_bits,p_bits", [(8, 45, 60), (12, 45, 60), (14, 45, 60), (14, 50, 40), (13, 30, 50)])
def test_special_primes_of_another_size(log_n, q_bits, p_bits):
    """Transforms in fp64 with conversions and sums in integers, and the other way round; both layouts of a norm and a
    projection with everything behind it."""
    from oracle import Ckks
    from paper_2609_12378_amd import Buf, Context, Epilogue
    ctx = Context(log_n, 8, 3, 3, q_bits=q_bits, p_bits=p_bits)
    ck = Ckks(log_n, ctx.q, ctx.p, 3)
    limbs, T, scale = 8, ck.n // 32, 1.01 * 2.0 ** (q_bits - 1)
    xs, rlk, poly = random_cts(ck, limbs, 2, 800), rlk_of(ck, 801), some_poly(11, 802)
    for g, x in zip(ctx.poly_eval(bufs(xs, scale), poly, to_dev(rlk)), xs):
        same(g.data, nc.poly_eval(ck, x, scale, poly, rlk), "polynomial")
    inv = some_poly(3, 803, 0.5, 3.0)
    for layout in ("fm", "tm"):
        st = norm_inputs(ck, limbs, T, layout, 2, "plain", "in", 810)
        got = ctx.rms_norm(bufs(st["xs"], scale), T, 32, inv, to_dev(st["rlk"]), dev_keys(st["keys"]), layout=layout,
                           weights=bufs(st["ws"], scale), residual=bufs(st["xs"], scale),
                           mask=Buf(to_dev(st["mask"]), scale) if layout == "tm" else None)
        want = nc.rms_norm(ck, st["xs"], scale, T, 32, inv, st["rlk"], st["keys"], layout, st["ws"], scale, st["mask"], scale,
                           residual=st["xs"], r_scale=scale)
        for g, w in zip(got, want):
            same(g.data, w, "norm, %s" % layout)
    keys, W, act = proj_keys(ck, T, "fm", 5), rng(820, 2).normal(0, 0.02, (16, 16)), some_poly(2, 821)
    got = ctx.linear_project(bufs(xs[:1], scale), to_dev(W), T, 5, dev_keys(keys), epilogue=Epilogue(
        act=act, gate=bufs(xs[1:], scale), residual=bufs(xs[:1], scale), rlk=to_dev(rlk)))
    want = nc.project(ck, xs[:1], scale, W, T, 5, keys, "fm", rlk, None, 1.0, act, xs[1:], scale, xs[:1], scale)
    same(got[0].data, want[0], "projection")


@pytest.mark.parametrize("ring_args,limbs", [((12, 7, 2, 4, 50), 7), ((14, 7, 3, 3, 50), 7)], ids=str)
def test_one_workspace_for_either_arithmetic(ring_args, limbs):
    """Polynomials and norms by integers in the workspace that was asked for under fp64, the same words."""
    import torch
    from test_gpu_nonlinear import three_calls
    ctx, ck = ring(*ring_args)
    T = ck.n // 64
    x, gate = (bufs(random_cts(ck, limbs, 2, seed), SCALE) for seed in (900, 901))
    calls, sizes = three_calls(ck, limbs, T, x, gate)
    want = [to_host(b.data) for b in calls(ctx)]
    mem = torch.full((max(sizes(ctx)) // 8 + 64,), 7, dtype=torch.uint64, device="cuda")
    try:
        ctx.set_workspace(mem[:-64])
        for arith in (1, 0):
            ctx.set_ntt_arith(arith)
            for b, w in zip(calls(ctx), want):
                same(b.data, w, "arithmetic %d" % arith)
        assert bool((mem[-64:] == 7).all())
    finally:
        ctx.set_ntt_arith(0)
        ctx.set_workspace(None)


@pytest.mark.parametrize("log_n", [8, 12])
def test_two_keys_for_one_rotation(log_n, monkeypatch):
    """One token a ciphertext, token-major: left rotations by k and by k - N/2 are one. A key for each is given, and each is
    used where its step is asked for, whatever their order; one key alone serves both."""
    from paper_2609_12378_amd import Buf
    ctx, ck = ring(log_n, 8, 3, 3, 50)
    limbs, slots = 8, ck.n // 2
    st = norm_inputs(ck, limbs, 1, "tm", 1, None, None, 950)
    there, unit = {}, 1
    for radix in nc.radixes(slots):
        there.update({k * unit: None for k in range(1, radix)})
        unit *= radix
    back = random_keys(ck, there, 951)
    there = random_keys(ck, there, 952)
    spread = {(-s) % slots: back[s] for s in back}
    plain = nc.all_positions
    inv, mask = some_poly(3, 953, 0.5, 3.0), Buf(to_dev(st["mask"]), SCALE)

    def want(fwd, rev):
        monkeypatch.setattr(nc, "all_positions", lambda ck, v, n, stride, keys: plain(ck, v, n, stride,
                                                                                      fwd if stride > 0 else rev))
        return nc.rms_norm(ck, st["xs"], SCALE, 1, slots, inv, st["rlk"], {}, "tm", None, 1.0, st["mask"], SCALE)[0]

    def got(keys):
        return ctx.rms_norm(bufs(st["xs"], SCALE), 1, slots, inv, to_dev(st["rlk"]), dev_keys(keys), layout="tm", mask=mask)[0]

    signed, both = {-s: back[s] for s in back}, want(there, spread)
    same(got({**signed, **there}).data, both, "the keys back first")
    same(got({**there, **signed}).data, both, "the keys there first")
    one = {**spread, **there}
    same(got(one).data, want(one, one), "one key a rotation")

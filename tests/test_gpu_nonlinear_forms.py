"""Polynomials, norms and the projection's epilogue in the forms of their calls that lie apart from the common ones: every
call in a workspace of its own reported size with guard words right behind it, in every kind of ring, both layouts and
either arithmetic (the token-major projection takes primes below 2^50 in fp64 alone); workspaces in which the token-major epilogue takes fewer giant steps a launch; token-major calls captured
and replayed; batches of 16 and more steps in the two-pass rings; the epilogue over lazily divided sums in larger rings."""
import numpy as np
import pytest

import nonlinear_common as nc
from gpu_common import say, to_dev, to_host
from rope_common import random_cts, random_keys
from test_gpu_nonlinear import SCALE, near, norm_inputs, plaintexts, proj_keys, rlk_of, some_poly
from test_gpu_rope import bufs, dev_keys, ring, same
from workloads import rng

pytestmark = pytest.mark.gpu

# one ring of every kind of kernel: 128-bit sums, whole rows in a block (two sizes), two passes, 59-bit primes below and
# above 2^14, a chain of mixed primes; limbs and tokens of a ciphertext
KINDS = [((8, 8, 3, 3, 50), 8, 8), ((12, 8, 3, 3, 50), 8, 64), ((13, 8, 2, 4, 50), 8, 128), ((14, 8, 3, 3, 50), 8, 128),
         ((10, 8, 3, 3, 59), 8, 32), ((14, 8, 3, 3, 59), 8, 128), ((13, 8, 3, 3, 0), 8, 128)]


def scale_of(ring_args):
    return near(ring_args) if ring_args[4] else SCALE * 2.0 ** -5      # 45-bit primes in the mixed chain


def one_call_each(ck, limbs, T, layout, x, gate, scale, seed=1081):
    """{name: (the call on a context, op, shape)} of a polynomial, a norm and a projection with everything behind it, the
    last two in `layout`; x and gate: two ciphertexts each."""
    from paper_2609_12378_amd import Buf, Context, Epilogue
    D, rlk, fm = ck.n // 2 // T, to_dev(rlk_of(ck, seed)), int(layout == "fm")
    keys = dev_keys({**random_keys(ck, Context.norm_steps(ck.n // 2, T, layout), seed), **proj_keys(ck, T, layout, 4)})
    W = to_dev(rng(seed, 2).normal(0, 0.02, (2 * D, 2 * D)))
    ws, bs = bufs(plaintexts(ck, limbs, 2, seed + 1), scale), bufs(plaintexts(ck, limbs, 2, seed + 2), scale)
    mask = None if fm else Buf(to_dev(plaintexts(ck, limbs - 1, 1, seed + 3)[0]), scale)
    p5, p3, p1 = some_poly(5, 1), some_poly(3, 2), some_poly(1, 3)
    return {
        "polynomial": (lambda c: c.poly_eval(x, p5, rlk), Context.OP_POLY_EVAL, (limbs, 2, 5)),
        "norm": (lambda c: c.rms_norm(x, T, 2 * D, p1, rlk, keys, layout=layout, weights=ws, mask=mask, newton=1, eps=0.1,
                                      residual=x), Context.OP_RMS_NORM, (limbs, 2, T, fm, 1, 1)),
        "projection": (lambda c: c.linear_project(x, W, T, 4, keys, layout=layout, epilogue=Epilogue(
            bias=bs, act=p3, gate=gate, residual=x, rlk=rlk)), Context.OP_PROJECT_EPILOGUE,
            (limbs, T, 2 * D, 2 * D, 4, fm, 3, 1))}


GUARD = 1 << 20


@pytest.mark.parametrize("layout", ["fm", "tm"])
@pytest.mark.parametrize("ring_args,limbs,T", KINDS, ids=str)
def test_every_call_in_a_workspace_of_its_own(ring_args, limbs, T, layout):
    """Each call alone, in as many bytes as are reported for it, under either arithmetic: the same words as in the library's
    own arena, and not a word behind the workspace written."""
    import torch
    from paper_2609_12378_amd import CkksError
    ctx, ck = ring(*ring_args)
    scale = scale_of(ring_args)
    x, gate = (bufs(random_cts(ck, limbs, 2, seed), scale) for seed in (1082, 1083))
    calls = one_call_each(ck, limbs, T, layout, x, gate, scale)
    ctx.set_proj_batch(8)
    try:
        for name, (call, op, shape) in calls.items():
            if name == "projection" and layout == "tm" and ring_args[4] != 50:
                with pytest.raises(CkksError, match="below 2.50"):
                    call(ctx)
                continue
            want = [to_host(b.data) for b in call(ctx)]
            need = ctx.workspace_bytes(op, shape)
            assert need > 0 and need % 8 == 0
            mem = torch.full((need // 8 + GUARD,), 7, dtype=torch.uint64, device="cuda")
            for arith in (0, 1):
                ctx.set_ntt_arith(arith)
                if name == "projection" and layout == "tm" and arith:
                    with pytest.raises(CkksError, match="below 2.50"):
                        call(ctx)
                    continue
                if ctx.workspace_bytes(op, shape) != need:      # another arithmetic's projection may take another size
                    assert name == "projection"
                    need = ctx.workspace_bytes(op, shape)
                    mem = torch.full((need // 8 + GUARD,), 7, dtype=torch.uint64, device="cuda")
                for fill in (0, 2 ** 62 + 12345):               # nothing is read that the call has not written
                    mem[:need // 8].fill_(fill)
                    ctx.set_workspace(mem[:need // 8])
                    for b, w in zip(call(ctx), want):
                        same(b.data, w, "%s, arithmetic %d" % (name, arith))
                    assert bool((mem[need // 8:] == 7).all()), "%s, arithmetic %d: words behind the workspace" % (name, arith)
                if name != "projection":                        # a projection may do with fewer giant steps a launch
                    ctx.set_workspace(mem[:need // 8 - 1])
                    with pytest.raises(CkksError, match="too small"):
                        call(ctx)
            ctx.set_ntt_arith(0)
            ctx.set_workspace(None)
    finally:
        ctx.set_ntt_arith(0)
        ctx.set_workspace(None)
        ctx.set_proj_batch(0)


@pytest.mark.parametrize("lazy", [False, True])
@pytest.mark.parametrize("ring_args,limbs,T", [KINDS[1], KINDS[2], KINDS[3]], ids=str)
def test_token_major_epilogue_in_smaller_workspaces(ring_args, limbs, T, lazy):
    """Fewer giant steps share a launch where the workspace has no room for all of them, down to one; the same words, and
    none behind the workspace; a workspace without room for one is refused before anything is written."""
    import torch
    from paper_2609_12378_amd import CkksError
    ctx, ck = ring(*ring_args)
    scale = scale_of(ring_args)
    x, gate = (bufs(random_cts(ck, limbs, 2, seed), scale) for seed in (1092, 1093))
    call, op, shape = one_call_each(ck, limbs, T, "tm", x, gate, scale)["projection"]
    ctx.set_lazy_moddown(lazy)
    try:
        want = [to_host(b.data) for b in call(ctx)]
        need = ctx.workspace_bytes(op, shape)
        mem = torch.full((need // 8 + GUARD,), 7, dtype=torch.uint64, device="cuda")
        taken = []
        for part in range(15, 0, -1):
            words = need // 8 * part // 16 // 32 * 32
            mem.fill_(7)
            ctx.set_workspace(mem[:words])
            try:
                got = call(ctx)
            except CkksError as e:
                assert "too small" in str(e)
                assert bool((mem == 7).all())
                break
            for b, w in zip(got, want):
                same(b.data, w, "%d of 16 parts" % part)
            assert bool((mem[words:] == 7).all())
            taken.append(part)
        say("parts of 16 that were room enough:", taken)
        assert len(taken) >= 3 and taken[-1] > 1
    finally:
        ctx.set_workspace(None)
        ctx.set_lazy_moddown(False)


@pytest.mark.parametrize("ring_args,limbs,T", [KINDS[1], KINDS[2], KINDS[3]], ids=str)
def test_token_major_calls_captured_and_replayed(ring_args, limbs, T):
    """A token-major norm (both of its sets of rounds) and a token-major projection with everything behind it, in a caller's
    workspace, replayed on new inputs between the program's own work."""
    import torch
    from paper_2609_12378_amd import Buf, Context
    eager, ck = ring(*ring_args)
    scale = scale_of(ring_args)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = Context(ck.log_n, ck.n_q, ck.n_p, ck.dnum, q=eager.q, p=eager.p, stream=stream)
    x, gate = ([Buf(torch.zeros((2, limbs, ck.n), dtype=torch.uint64, device="cuda"), scale) for _ in range(2)]
               for _ in range(2))
    made = one_call_each(ck, limbs, T, "tm", x, gate, scale)
    calls = lambda c: [b for name in ("norm", "projection") for b in made[name][0](c)]  # noqa: E731
    torch.cuda.synchronize()
    ws = torch.empty(max(ctx.workspace_bytes(op, shape) for _, op, shape in made.values()) // 8, dtype=torch.uint64,
                     device="cuda")
    ctx.set_workspace(ws)
    with torch.cuda.stream(stream):
        calls(ctx)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = calls(ctx)
    torch.cuda.synchronize()
    for r in range(4):
        for b, a in zip(x + gate, random_cts(ck, limbs, 4, 1100 + r)):
            b.data.copy_(to_dev(a))
        torch.cuda.synchronize()
        want = [to_host(b.data) for b in calls(eager)]
        graph.replay()
        torch.cuda.synchronize()
        for i, (g, w) in enumerate(zip(out, want)):
            same(g.data, w, "replay %d: output %d" % (r, i))
        junk = [torch.randn(1 << 20, device="cuda") for _ in range(4)]
        del junk
    del graph


# ---- batches of the two-pass rings --------------------------------------------------------------------------------

@pytest.mark.parametrize("ring_args", [(14, 5, 2, 3, 50), (15, 5, 2, 3, 50)], ids=str)
def test_more_ciphertexts_than_a_batch_of_steps(ring_args):
    """17 ciphertexts: two batches of every depth, and depths of more than 16 steps that switch a key."""
    ctx, ck = ring(*ring_args)
    poly, rlk = some_poly(7, 1200), rlk_of(ck, 1201)
    xs = random_cts(ck, 5, 17, 1202)
    got = ctx.poly_eval(bufs(xs, SCALE), poly, to_dev(rlk))
    for r in (0, 1, 15, 16):
        same(got[r].data, nc.poly_eval(ck, xs[r], SCALE, poly, rlk), "ciphertext %d" % r)


@pytest.mark.parametrize("log_n,count,weights", [(14, 15, "plain"), (14, 16, "plain"), (14, 17, "plain"), (14, 16, "cipher"),
                                                 (12, 16, "plain"), (8, 16, "cipher")])
def test_norms_at_the_borders_of_a_batch(log_n, count, weights):
    """The weights' products in one batch with the last Newton step (15 and it are 16), after it (16), in two (17)."""
    ctx, ck = ring(log_n, 7, 2, 4, 50)
    limbs, T = 7, ck.n // 16
    st = norm_inputs(ck, limbs, T, "fm", count, weights, "in", 1210)
    inv = some_poly(1, 1211, 0.5, 3.0)
    x = bufs(st["xs"], SCALE)
    got = ctx.rms_norm(x, T, 8 * count, inv, to_dev(st["rlk"]), dev_keys(st["keys"]), weights=bufs(st["ws"], SCALE),
                       newton=1, eps=1e-3, residual=x, residual_scale=0.5)
    want = nc.rms_norm(ck, st["xs"], SCALE, T, 8 * count, inv, st["rlk"], st["keys"], "fm", st["ws"], SCALE, newton=1,
                       eps=1e-3, residual=st["xs"], r_scale=SCALE, residual_scale=0.5)
    for r in range(count):
        same(got[r].data, want[r], "ciphertext %d" % r)


@pytest.mark.parametrize("ring_args,limbs,degree", [((14, 9, 1, 9, 50), 9, 12), ((14, 9, 1, 9, 50), 7, 5),
                                                    ((15, 6, 1, 6, 50), 6, 8), ((16, 6, 1, 6, 50), 5, 4)], ids=str)
def test_many_digits_in_two_passes(ring_args, limbs, degree):
    """A step's digits end their transforms four to a reduction, its own apart: five to nine of them, and odd counts left."""
    ctx, ck = ring(*ring_args)
    poly, rlk = some_poly(degree, 1220 + degree), rlk_of(ck, 1221)
    xs = random_cts(ck, limbs, 2, 1222)
    for g, x in zip(ctx.poly_eval(bufs(xs, SCALE), poly, to_dev(rlk)), xs):
        same(g.data, nc.poly_eval(ck, x, SCALE, poly, rlk), "polynomial")


# ---- the epilogue over lazily divided sums ------------------------------------------------------------------------

# ring, limbs, tokens, layout, d_in and d_out in ciphertexts, n1, degree
LAZY = [((9, 6, 2, 3, 59), 5, 16, "fm", 2, 2, 4, 3), ((9, 6, 2, 3, 50), 5, 16, "tm", 2, 2, 4, 3),
        ((12, 5, 2, 3, 50), 5, 64, "fm", 2, 3, 8, 3), ((12, 5, 2, 3, 50), 5, 64, "tm", 2, 3, 8, 3),
        ((14, 5, 2, 3, 50), 5, 256, "fm", 2, 2, 8, 3), ((14, 5, 2, 3, 50), 5, 128, "tm", 2, 2, 16, 3),
        ((16, 4, 2, 2, 50), 4, 4096, "fm", 1, 1, 4, 1), ((16, 4, 2, 2, 50), 4, 4096, "tm", 1, 2, 4, 1)]


@pytest.mark.parametrize("lazy", [False, True])
@pytest.mark.parametrize("case", LAZY, ids=str)
def test_epilogue_of_lazy_sums(case, lazy):
    """Several inputs and outputs, bias, activation, gate and residual, with one ModDown an output or one a rotation."""
    from paper_2609_12378_amd import Epilogue
    ring_args, limbs, tokens, layout, n_in, n_out, n1, degree = case
    ctx, ck = ring(*ring_args)
    D, scale = ck.n // 2 // tokens, near(ring_args)
    xs, rlk, keys = random_cts(ck, limbs, n_in, 1300), rlk_of(ck, 1301), proj_keys(ck, tokens, layout, n1)
    W = rng(1302, 2).normal(0, 0.02, (n_in * D, n_out * D))
    act, bs = some_poly(degree, degree), plaintexts(ck, limbs, n_out, 1303)
    gs, rs = random_cts(ck, limbs - 1, n_out, 1304), random_cts(ck, limbs, n_out, 1305)
    ctx.set_lazy_moddown(lazy)
    try:
        got = ctx.linear_project(bufs(xs, scale), to_dev(W), tokens, n1, dev_keys(keys), layout=layout, epilogue=Epilogue(
            bias=bufs(bs, 0.7 * scale), act=act, gate=bufs(gs, 0.8 * scale), residual=bufs(rs, 0.9 * scale),
            residual_scale=0.5, rlk=to_dev(rlk)))
    finally:
        ctx.set_lazy_moddown(False)
    want = nc.project(ck, xs, scale, W, tokens, n1, keys, layout, rlk, [b[0][None] for b in bs], 0.7 * scale, act, gs,
                      0.8 * scale, rs, 0.9 * scale, 0.5, lazy)
    assert len(got) == n_out
    for j in range(n_out):
        same(got[j].data, want[j], "output %d" % j)

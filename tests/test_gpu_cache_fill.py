"""What a page holds after many appends: every append adds its own noise to all slots of a started page."""
import numpy as np
import pytest

from gpu_common import say, to_dev, to_host
from rope_common import plain_rope
from test_gpu_rope import SLOT_BOUND, Party
from workloads import rng

pytestmark = pytest.mark.gpu


def test_a_page_filled_token_by_token():
    """128 appends of one token each.  Decrypted slots are sums of the appends', each within SLOT_BOUND of its own (a
    rotary token in its slot, zero elsewhere): a page of n appends is within n SLOT_BOUND.  The noises are independent,
    so that a page of n is far inside that: about sqrt(n) times one append's."""
    import torch
    from paper_2609_12378_amd import Buf, rope_inv_freq
    P = Party(seed=141)
    ctx, T, hd, limbs = P.ctx, 128, 32, 4
    D, slots = ctx.n // 2 // T, ctx.n // 2
    g = rng(142, 1)
    K, V = g.uniform(-1, 1, (T, hd)), g.uniform(-1, 1, (T, hd))
    cos, sin = ctx.rope_cos_sin(torch.arange(T, device="cuda"), rope_inv_freq(hd).cuda())
    keys = P.keys(ctx.rope_steps(slots, T, hd))
    pages = [[Buf(torch.zeros((2, limbs - 1, ctx.n), dtype=torch.uint64, device="cuda"), 1.0)] for _ in range(2)]
    held = np.zeros((2, T, hd))
    turned = plain_rope(K[:, None], to_host(cos), to_host(sin), "half")[:, 0]
    errs = []
    for t in range(T):
        def placed(row):
            z = np.zeros((T, hd))
            z[t] = row
            return P.encrypt(np.tile(z, (1, D // hd)), limbs)
        tables = ctx.cache_tables(cos[t:t + 1].contiguous(), sin[t:t + 1].contiguous(), T, hd, hd, t, 1, limbs)
        ctx.cache_append([placed(K[t])], [placed(V[t])], tables, T, hd, hd, t, 1, keys, *pages, [[0]], src=t)
        held[0][t], held[1][t] = turned[t], V[t]
        if t + 1 in (1, 2, 16, T):
            err = [float(np.max(np.abs(P.decrypt(pages[i][0]).reshape(T, D // hd, hd) - held[i][:, None])))
                   for i in range(2)]
            say("%d appends: keys %.3g, values %.3g" % (t + 1, *err))
            errs.append(max(err))
            assert errs[-1] < (t + 1) * SLOT_BOUND

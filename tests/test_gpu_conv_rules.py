"""Which launches a conversion takes on either side of its rules, read from the event profiler, and the same words on
both: rotary positions of several ciphertexts against those of each alone.
"""
import numpy as np
import pytest

from gpu_common import to_dev, to_host
from rope_common import random_cts, random_keys, term_steps
from test_gpu_rope import angles, bufs, dev_keys, ring

pytestmark = pytest.mark.gpu


def launches(chain, T, hd, limbs, count):
    ctx, ck = ring(*chain)
    keys = dev_keys(random_keys(ck, term_steps(ck.n, T, hd, "tm", "half"), 151))
    tables = ctx.rope_tables(*(to_dev(x) for x in angles(T, hd // 2, 152)), T, hd, hd, limbs)
    xs = bufs(random_cts(ck, limbs, count, 153))
    want = [to_host(ctx.rope([x], tables, T, hd, hd, keys)[0].data) for x in xs]
    ctx.profile(True)
    ctx.profile_reset()
    got = ctx.rope(xs, tables, T, hd, hd, keys)
    seen = {k: v[1] for k, v in ctx.profile_all().items()}
    ctx.profile(False)
    assert all(np.array_equal(to_host(g.data), w) for g, w in zip(got, want))
    return seen


@pytest.mark.parametrize("chain,limbs,count,apart", [
    ((15, 6, 2, 3, 50), 6, 8, 0),       # 1280 reads of the quotient, 2688 of the ModUp
    ((15, 16, 8, 2, 50), 16, 2, 0),     # 3840, 5888
    ((15, 16, 8, 2, 50), 16, 4, 1),     # 7680: the quotient's column pass is a launch of its own; 11776
    ((14, 24, 8, 3, 50), 24, 4, 1),     # 5888, 11904
    ((14, 24, 8, 3, 50), 24, 8, 2),     # 11776, 23808: the ModUp's as well
], ids=lambda c: "n%d" % c[0] if isinstance(c, tuple) else str(c))
def test_forward_column_passes(chain, limbs, count, apart):
    T = 64 if chain[0] == 14 else 128
    assert launches(chain, T, 128, limbs, count).get("ntt_fwd_col", 0) == apart


@pytest.mark.parametrize("count,apart", [(1, 2), (4, 2), (5, 0), (7, 0)])
def test_inverse_column_passes(count, apart):
    """N = 2^16, two digits: 32 count blocks of 16 columns a conversion, in the ModUp and in the quotient.  Up to 128 the
    sources' column passes are launches of their own, as their targets are split over blocks."""
    assert launches((16, 4, 2, 2, 50), 128, 128, 4, count).get("ntt_inv_col", 0) == apart

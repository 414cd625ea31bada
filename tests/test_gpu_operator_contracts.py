"""What the operators around the cache promise beyond the ordinary call: every group size of query heads, values that are no numbers, caches
whose places are used again, arrays that move along.  Against the plain 64-bit forms."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from operator_refs import DP
from paper_2602_22593_amd import binding as kv
from paper_2602_22593_amd import workloads as wl

from test_gpu_operators import DEV, dev, host, view_of, within

pytestmark = pytest.mark.gpu
WIDE = 150000      # a bound of the lengths for which heads of a token are read side by side


def decode_case(geom, ctx, index=80):
    c = ref.case(geom, (DP, 1, 0), ctx, [min(n, 1) for n in ctx], index=index)
    c.q = wl.randn_bf16((len(ctx), geom[0], geom[2]), wl.generator(index, wl.SUB_QUERY))
    return c


def wide_table(c, bound):
    return np.pad(c.table, ((0, 0), (0, max(0, -(-bound // c.info["block_tokens"]) - c.table.shape[1]))), constant_values=-1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,ctx,bound", [
    (2, [2900, 1111, 33], 3000),
    (4, [2900, 1111, 33], WIDE),
    (10, [12000, 3001], 12000),        # few shares: a wavefront has four tiles and more in a row
])
@pytest.mark.parametrize("group", [9, 16, 17, 20, 24, 25])
def test_weights_of_every_group_size(group, heads, ctx, bound, d):
    """Scores leave the kernel in passes over the query heads: few, some empty, all of them; the tiles in hand have to have landed."""
    c = decode_case((group * heads, heads, d, 16), ctx)
    prior = np.random.default_rng(18).exponential(1e-3, (len(ctx), heads, bound)).astype(np.float32)
    want, tol, sums, sums_tol = ref.decode_weights(c, prior)
    weights = dev(prior)
    out = kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), dev(wide_table(c, bound)), dev(c.ctx), view_of(c), bound, weights)
    within(host(out), want, tol)
    assert (np.abs(host(weights).astype(np.float64) - sums) <= sums_tol).all()

"""GPU parity of the operators around the cache with their plain 64-bit forms: sizes, layouts, masks and strides where they can
go wrong.  Pools are poisoned with NaN wherever no valid token lies, and compared whole."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from operator_refs import DP, TP
from paper_2602_22593_amd import binding as kv
from paper_2602_22593_amd import workloads as wl

from helpers import bf16_bits_to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
G8B, G70B, TINY = (32, 8, 128, 16), (64, 8, 128, 16), (8, 2, 64, 16)


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16)).to(DEV).view(torch.bfloat16) if a.dtype == np.uint16 else torch.from_numpy(a).to(DEV)


def host(t):
    t = t.contiguous()
    return t.view(torch.int16).cpu().numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.cpu().numpy()


def view_of(c):
    i = c.view
    return kv.kv_view_create(c.w.n_q_heads, c.w.n_kv_heads, c.w.head_dim, c.w.base_block_size, i.layout, i.tp_degree, i.rank)


def within(got_bits, want, tol, what=""):
    got = bf16_bits_to_f64(got_bits)
    assert np.isfinite(got).all(), what
    bad = np.abs(got - want) > tol + 1e-30
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.abs(got - want).max():.3g}, first at {np.argwhere(bad)[0]}"


# ---- kv_rope_append ----------------------------------------------------------------------------------

def rope_inputs(c, axes, rot, rng, far=False):
    total = int(c.q_off[-1])
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], c.w.head_dim
    qkv = wl.randn_bf16((total, ql + 2 * hl, d), wl.generator(c.w.index, wl.SUB_MISC))
    positions = rng.integers(0, 2 ** 31 - 1 if far else 5000, (axes, total)).astype(np.int32)
    if far and total:
        positions[0, 0], positions[-1, -1] = 2 ** 31 - 1, -(2 ** 31) + 1
    half = rot // 2
    inv_freq = (1e4 ** (-np.arange(half) / max(half, 1))).astype(np.float32)
    return qkv, positions, inv_freq, [int(a) for a in rng.integers(0, axes, half)]


@pytest.mark.parametrize("geom,triple,ctx,q_lens,axes,adjacent,rot", [
    (TINY, (DP, 1, 0), [17, 1, 300, 64], [1, 1, 1, 1], 1, False, 64),
    (TINY, (TP, 2, 1), [40, 33, 5, 0, 64], [3, 33, 1, 0, 0], 2, True, 32),
    (G8B, (DP, 1, 0), [300, 1, 77], [129, 1, 40], 3, False, 128),
    (G8B, (TP, 4, 2), [2100], [2100], 4, True, 128),
    (G8B, (DP, 4, 3), [50, 61], [20, 7], 3, False, 64),
    (G70B, (TP, 8, 5), [16] * 70 + [1200], [2] * 70 + [1100], 1, False, 16),
    ((6, 2, 96, 5), (TP, 2, 1), [23, 9], [11, 9], 2, False, 48),
    (G8B, (DP, 1, 0), [5, 3], [2, 3], 1, False, 0),
])
def test_rope_append(geom, triple, ctx, q_lens, axes, adjacent, rot):
    c = ref.case(geom, triple, ctx, q_lens)
    rng = np.random.default_rng(5)
    qkv, positions, inv_freq, axis_of = rope_inputs(c, axes, rot, rng)
    hl, ql, total = c.info["n_kv_local"], c.info["n_q_local"], int(c.q_off[-1])
    x = bf16_bits_to_f64(qkv)
    want, tol = ref.rotated(x[:, :ql + hl], positions, inv_freq, axis_of, adjacent)
    # two rows more than the sequences have: they stay as they are
    parts = dev(np.concatenate([qkv, qkv[:1], qkv[:1]]))
    pos = np.concatenate([positions, positions[:, :1], positions[:, :1]], axis=1)
    out = torch.full((total + 2, ql, geom[2]), 7.0, dtype=torch.bfloat16, device=DEV)
    pool = dev(c.pool)
    token_pos = torch.full((len(ctx), hl, max(ctx) + 3), -5, dtype=torch.int32, device=DEV)
    kv.kv_rope_append(pool, view_of(c), parts[:, :ql], parts[:, ql:ql + hl], parts[:, ql + hl:], dev(pos), dev(inv_freq),
                      dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), axes=axis_of,
                      pairs=kv.KV_ROPE_ADJACENT if adjacent else kv.KV_ROPE_HALVES, out=out, token_pos=token_pos)
    got = host(out)
    assert (out[total:] == 7.0).all()
    within(got[:total], want[:, :ql], tol[:, :ql], "q")
    got_pool, want_pool = host(pool).reshape(c.pool.shape), c.pool.copy()
    rows, h0 = ref.view_rows(c, want_pool)
    got_rows, _ = ref.view_rows(c, got_pool)
    want_pos = np.full(token_pos.shape, -5, np.int32)
    for s in range(len(ctx)):
        new = np.arange(c.ctx[s] - c.q_lens[s], c.ctx[s])
        r = slice(int(c.q_off[s]), int(c.q_off[s + 1]))
        b, slot = ref.place(c, s, new)
        within(got_rows[b, 0, slot, h0:h0 + hl], want[r, ql:], tol[r, ql:], f"keys of {s}")
        rows[b, 1, slot, h0:h0 + hl] = qkv[r, ql + hl:]
        rows[b, 0, slot, h0:h0 + hl] = got_rows[b, 0, slot, h0:h0 + hl]
        want_pos[s, :, new] = positions[0, r][:, None]
    assert np.array_equal(got_pool, want_pool), "values, or bytes that are nobody's"
    assert np.array_equal(host(token_pos), want_pos)


def test_rope_of_far_positions_and_in_place():
    c = ref.case(G8B, (DP, 1, 0), [40, 9], [30, 9])
    qkv, positions, inv_freq, axis_of = rope_inputs(c, 2, 128, np.random.default_rng(6), far=True)
    x = bf16_bits_to_f64(qkv)
    want, tol = ref.rotated(x[:, :40], positions, inv_freq, axis_of, False)
    q, k, v = (dev(np.ascontiguousarray(a)) for a in (qkv[:, :32], qkv[:, 32:40], qkv[:, 40:]))
    out = kv.kv_rope_append(dev(c.pool), view_of(c), q, k, v, dev(positions), dev(inv_freq), dev(c.table), dev(c.ctx),
                            dev(c.q_off.astype(np.int32)), axes=axis_of, out=q)
    assert out.data_ptr() == q.data_ptr()
    within(host(q), want[:, :32], tol[:, :32])


def test_rope_skips_places_that_are_none():
    """A padded sequence (length 0), a block of -1 and one past the pool: queries turn, nothing is written."""
    c = ref.case(TINY, (DP, 1, 0), [20, 20, 20, 20], [1, 1, 1, 1])
    qkv, positions, inv_freq, axis_of = rope_inputs(c, 1, 64, np.random.default_rng(7))
    ctx, table = c.ctx.copy(), c.table.copy()
    ctx[0], table[1, 1], table[2, 1], ctx[3] = 0, -1, len(c.pool), 16 * table.shape[1] + 1
    pool = dev(c.pool)
    out = kv.kv_rope_append(pool, view_of(c), dev(qkv[:, :8]), dev(qkv[:, 8:10]), dev(qkv[:, 10:]), dev(positions),
                            dev(inv_freq), dev(table), dev(ctx), axes=axis_of)
    want, tol = ref.rotated(bf16_bits_to_f64(qkv)[:, :8], positions, inv_freq, axis_of, False)
    within(host(out), want, tol)
    assert np.array_equal(host(pool).reshape(c.pool.shape), c.pool)


# ---- paged_tree_attn ---------------------------------------------------------------------------------

def run_tree(c, words, **more):
    return kv.paged_tree_attn(dev(c.q), dev(c.pool), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), dev(words),
                              view_of(c), int(c.ctx.max()), int(c.q_lens.max()), **more)


@pytest.mark.parametrize("geom,triple,ctx,q_lens", [
    (TINY, (DP, 1, 0), [17, 1, 300, 64], [3, 1, 8, 5]),                       # up to 32 rows
    (G8B, (DP, 1, 0), [40, 31, 32, 33, 700], [8, 1, 2, 3, 4]),
    (G8B, (TP, 2, 1), [900, 64, 15, 0, 513], [16, 1, 15, 0, 9]),               # up to 64
    (G70B, (TP, 8, 3), [1200, 16, 130, 2], [16, 16, 7, 2]),                    # up to 128
    (G8B, (DP, 4, 2), [400, 333], [31, 32]),                                  # rank's heads in place
    (G8B, (TP, 4, 0), [600, 256, 1000, 64], [64, 256, 65, 1]),                 # several blocks of rows
    ((10, 2, 64, 32), (DP, 1, 0), [77, 500, 200], [13, 33, 200]),              # odd groups
    ((10, 2, 128, 48), (TP, 2, 0), [77, 500, 97], [13, 12, 1]),                # blocks of 96 tokens
    ((64, 2, 64, 16), (DP, 1, 0), [100, 20], [5, 20]),                        # 32 query heads on one
    (TINY, (DP, 1, 0), [9000], [256]),
    (G8B, (TP, 8, 7), [20000], [5]),                                          # one sequence over all workgroups
    (TINY, (TP, 2, 0), [3] * 400 + [2000], [2] * 400 + [9]),                   # more sequences than threads
])
def test_tree_attention(geom, triple, ctx, q_lens):
    c = ref.case(geom, triple, ctx, q_lens)
    seen, words = ref.tree_masks(c.q_lens, np.random.default_rng(8))
    want, tol = ref.tree_attention(c, seen)
    within(host(run_tree(c, words)), want, tol)


def test_tree_of_any_bits():
    """Masks that are no trees: rows that see nothing, everything, later nodes; bits past the draft; more words than needed."""
    c = ref.case(G8B, (TP, 2, 0), [70, 12, 40, 300], [70, 12, 1, 100])
    rng = np.random.default_rng(9)
    seen = rng.random((int(c.q_off[-1]), 256)) < 0.5
    seen[3], seen[75], seen[82] = False, False, False        # (rows of sequences with nothing before the draft: zeros)
    seen[5] = True
    want, tol = ref.tree_attention(c, seen)
    got = host(run_tree(c, ref.pack(seen), scale=0.11))
    want, tol = ref.tree_attention(c, seen, 0.11)
    within(got, want, tol)
    assert (got[3] == 0).all() and (got[75] == 0).all()


@pytest.mark.parametrize("d,bad", [(128, np.nan), (128, np.inf), (64, -np.inf)])
def test_tree_hides_what_is_not_finite(d, bad):
    """Infinities and NaN in keys and values of drafted tokens reach the rows that see them, and no others."""
    c = ref.case((8, 2, d, 16), (DP, 1, 0), [100, 45, 31], [20, 45, 7])
    seen, words = ref.tree_masks(c.q_lens, np.random.default_rng(10))
    bits = {True: 0x7FC0, False: 0x7F80 if bad > 0 else 0xFF80}[bool(np.isnan(bad))]
    rows, h0 = ref.view_rows(c, c.pool)
    victims = {0: (7, 0), 1: (11, 1), 2: (3, 1)}              # node, plane
    hit = np.zeros(len(seen), bool)
    for s, (node, plane) in victims.items():
        b, slot = ref.place(c, s, c.ctx[s] - c.q_lens[s] + node)
        rows[b, plane, slot, :, ::3] = bits
        hit[c.q_off[s]:c.q_off[s + 1]] = seen[c.q_off[s]:c.q_off[s + 1], node]
    want, tol = ref.tree_attention(c, seen)
    got = bf16_bits_to_f64(host(run_tree(c, words)))
    assert hit.any() and not hit.all()
    assert (np.abs(got[~hit] - want[~hit]) <= tol[~hit]).all()
    for s, (node, plane) in victims.items():
        if plane == 1:                                        # values: those elements and no others
            r = np.arange(c.q_off[s], c.q_off[s + 1])
            r = r[hit[r]]
            assert not np.isfinite(got[r][:, :, ::3]).any()
            keep = np.arange(d) % 3 != 0
            assert (np.abs(got[r] - want[r]) <= tol[r])[:, :, keep].all()


def test_tree_chain_is_causal_attention():
    c = ref.case(G8B, (TP, 2, 1), [3000, 200], [40, 64])
    chain = np.zeros((104, 64), bool)
    for s in range(2):
        for j in range(int(c.q_lens[s])):
            chain[int(c.q_off[s]) + j, :j + 1] = True
    got = bf16_bits_to_f64(host(run_tree(c, ref.pack(chain))))
    same = kv.paged_prefill_attn(dev(c.q), dev(c.pool), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), view_of(c), 3000, 64)
    _, tol = ref.tree_attention(c, chain)
    assert (np.abs(got - bf16_bits_to_f64(host(same))) <= 2 * tol).all()


def test_tree_bounds_larger_than_needed_and_rows_behind():
    c = ref.case(G8B, (TP, 4, 1), [90, 200], [5, 9])
    seen, words = ref.tree_masks(c.q_lens, np.random.default_rng(11), words=4)
    want, tol = ref.tree_attention(c, seen)
    pad = np.concatenate([c.q, c.q[:3]])
    table = np.pad(c.table, ((0, 0), (0, 60)), constant_values=-1)
    out = torch.full(pad.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    kv.paged_tree_attn(dev(pad), dev(c.pool), dev(table), dev(c.ctx), dev(c.q_off.astype(np.int32)),
                       dev(np.concatenate([words, words[:3]])), view_of(c), 4000, 256, out=out)
    within(host(out)[:14], want, tol)
    assert (out[14:] == 7.0).all()


@pytest.mark.parametrize("geom,triple,ctx,q_lens", [
    (G8B, (DP, 1, 0), [40, 31, 32, 33, 700, 1, 64], [8, 1, 2, 3, 4, 1, 8]),    # four heads a workgroup, 1 KiB a token
    (G8B, (TP, 2, 1), [900, 64, 15, 5], [8, 1, 7, 5]),
    (G8B, (DP, 2, 1), [300, 77], [3, 8]),                                     # the rank's half of a row
    ((16, 4, 64, 16), (DP, 1, 0), [500, 33, 8, 1000], [8, 1, 8, 2]),            # rows of 128 bytes
    ((24, 12, 64, 32), (TP, 3, 2), [130, 31], [16, 15]),
    (G8B, (DP, 1, 0), [5000], [8]),
])
def test_tree_and_weights_of_heads_side_by_side(geom, triple, ctx, q_lens):
    """Bounds of a large batch, for which several heads of a token are read together."""
    c = ref.case(geom, triple, ctx, q_lens)
    bound = 150000
    table = np.pad(c.table, ((0, 0), (0, -(-bound // c.info["block_tokens"]) - c.table.shape[1])), constant_values=-1)
    seen, words = ref.tree_masks(c.q_lens, np.random.default_rng(16))
    want, tol = ref.tree_attention(c, seen)
    off, view = c.q_off.astype(np.int32), view_of(c)
    got = kv.paged_tree_attn(dev(c.q), dev(c.pool), dev(table), dev(c.ctx), dev(off), dev(words), view, bound, max(q_lens))
    within(host(got), want, tol)
    c.q = wl.randn_bf16((len(ctx), c.info["n_q_local"], geom[2]), wl.generator(61, wl.SUB_QUERY))
    prior = np.random.default_rng(17).exponential(1e-3, (len(ctx), c.info["n_kv_local"], bound)).astype(np.float32)
    want, tol, sums, sums_tol = ref.decode_weights(c, prior)
    weights = dev(prior)
    within(host(kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), dev(table), dev(c.ctx), view, bound, weights)), want, tol)
    assert (np.abs(host(weights).astype(np.float64) - sums) <= sums_tol).all()


# ---- kv_accept ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("geom,triple,ctx,q_lens,counts", [
    (TINY, (DP, 1, 0), [17, 1, 300, 64], [3, 1, 8, 5], [2, 1, 0, 5]),
    (G8B, (DP, 1, 0), [700, 256, 40], [64, 256, 40], [7, 200, 39]),
    (G8B, (TP, 4, 3), [90, 0, 33], [33, 0, 17], [12, 0, 1]),
    (G8B, (DP, 2, 1), [300], [300], [270]),
    ((6, 2, 96, 5), (TP, 2, 1), [23, 9], [11, 9], [4, 6]),
])
def test_accept(geom, triple, ctx, q_lens, counts):
    c = ref.case(geom, triple, ctx, q_lens)
    rng = np.random.default_rng(12)
    nodes = np.full((len(ctx), max(counts) + 2), -1, np.int32)
    for s, k in enumerate(counts):
        nodes[s, :k] = np.sort(rng.permutation(int(c.q_lens[s]))[:k])
    want, lens = ref.accepted_pool(c, c.pool, nodes, counts)
    pool = dev(c.pool)
    got = kv.kv_accept(pool, view_of(c), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), dev(nodes), dev(np.asarray(counts, np.int32)))
    assert np.array_equal(host(pool).reshape(want.shape), want)
    assert np.array_equal(host(got), lens)


def test_accept_of_nodes_that_are_none():
    """Numbers outside the draft are skipped, counts are cut to the draft and the list."""
    c = ref.case(TINY, (DP, 1, 0), [40, 30], [6, 4])
    nodes = np.array([[1, 99, 5, -3], [2, 3, 3, 3]], np.int32)
    want, _ = ref.accepted_pool(c, c.pool, [[1, 1, 5], [2, 3]], [1, 2])
    rows, h0 = ref.view_rows(c, want)
    (tb, ts), (sb, ss) = ref.place(c, 0, 36), ref.place(c, 0, 39)
    rows[tb, :, ts] = ref.view_rows(c, c.pool)[0][sb, :, ss]
    pool = dev(c.pool)
    got = kv.kv_accept(pool, view_of(c), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), dev(nodes), dev(np.array([9, 2], np.int32)))
    assert np.array_equal(host(pool).reshape(want.shape), want)
    assert host(got).tolist() == [38, 28]


# ---- paged_decode_attn_weights -----------------------------------------------------------------------

@pytest.mark.parametrize("geom,triple,ctx", [
    (TINY, (DP, 1, 0), [17, 1, 300, 64]),
    (G8B, (DP, 1, 0), [1, 31, 32, 33, 0, 2100]),
    (G70B, (TP, 8, 3), [1200, 16, 130]),
    (G8B, (DP, 4, 2), [400, 0]),
    ((10, 2, 128, 48), (TP, 2, 0), [777, 97]),
    ((2, 2, 64, 16), (DP, 1, 0), [5000]),
    ((64, 2, 128, 16), (DP, 1, 0), [300, 1100]),
    (G8B, (TP, 8, 7), [30000]),
    (TINY, (TP, 2, 0), [3] * 300 + [4000]),
])
def test_decode_weights(geom, triple, ctx):
    c = ref.case(geom, triple, ctx, [min(n, 1) for n in ctx])
    c.q = wl.randn_bf16((len(ctx), c.info["n_q_local"], geom[2]), wl.generator(61, wl.SUB_QUERY))   # empty sequences have a row too
    rng = np.random.default_rng(13)
    prior = rng.exponential(3.0 / max(ctx), (len(ctx), c.info["n_kv_local"], max(ctx) + 5)).astype(np.float32)
    for s, n in enumerate(ctx):
        prior[s, :, max(n - 1, 0):] = np.nan      # the newest token's entry is set, later ones are left
    want, tol, sums, sums_tol = ref.decode_weights(c, prior)
    weights = dev(prior)
    out = kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), dev(c.table), dev(c.ctx), view_of(c), max(ctx), weights)
    within(host(out), want, tol)
    got = host(weights).astype(np.float64)
    for s, n in enumerate(ctx):
        assert np.isnan(got[s, :, n:]).all()
        off = np.abs(got[s, :, :n] - sums[s, :, :n])
        assert (off <= sums_tol[s, :, :n]).all(), (s, off.max(), sums_tol[s, :, :n].max())


# ---- kv_evict ----------------------------------------------------------------------------------------

def evict_inputs(c, rng, ties=True):
    shape = (len(c.ctx), c.info["n_kv_local"], int(c.ctx.max()) + 3)
    weights = rng.lognormal(0, 2, shape).astype(np.float32)
    if ties:
        weights[rng.random(shape) < 0.3] = 0.0
        weights = np.where(rng.random(shape) < 0.3, np.float32(0.25), weights)
    token_pos = rng.permuted(np.broadcast_to(np.arange(shape[2], dtype=np.int32), shape), axis=2)
    return weights, np.ascontiguousarray(token_pos)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("geom,triple,ctx,keep,sinks,recent", [
    (TINY, (DP, 1, 0), [17, 1, 300, 64], [8, 1, 100, 64], 0, 0),
    (TINY, (TP, 2, 1), [40, 41, 500, 0], [39, 1, 0, 5], 4, 10),
    (G8B, (DP, 1, 0), [700, 256, 2000], [512, 300, 64], 4, 32),
    (G8B, (TP, 4, 3), [90, 3000], [50, 2990], 0, 100),
    (G8B, (DP, 8, 6), [1500], [20], 16, 1000),                # more protected than the budget holds
    ((6, 2, 96, 5), (TP, 2, 1), [23, 77], [11, 33], 1, 3),
    (TINY, (DP, 1, 0), [20000], [9000], 4, 500),
    (TINY, (DP, 1, 0), [8192, 8191, 4097], [4096, 8190, 1], 0, 0),   # the most that one workgroup takes
    (TINY, (TP, 2, 0), [8193, 12288, 100, 0, 9000], [8192, 4096, 100, 5, 0], 4, 64),
    (TINY, (DP, 2, 1), [13000, 10000], [300, 4200], 16, 6000),      # long, and more protected than the budget holds in one
])
def test_evict(geom, triple, ctx, keep, sinks, recent, in_place):
    c = ref.case(geom, triple, ctx, [0] * len(ctx))
    weights, token_pos = evict_inputs(c, np.random.default_rng(14))
    next_pos = np.full(len(ctx), weights.shape[2], np.int32)
    want, w2, p2, lens = ref.evicted(c, c.pool, np.asarray(keep), weights, token_pos, next_pos, sinks, recent)
    pool, w, p = dev(c.pool), dev(weights), dev(token_pos)
    outs = {} if in_place else dict(weights_out=torch.full_like(w, -1.0), token_pos_out=torch.full_like(p, -1))
    got = kv.kv_evict(pool, view_of(c), dev(c.table), dev(c.ctx), dev(np.asarray(keep, np.int32)), w, p, dev(next_pos), max(ctx),
                      sinks=sinks, recent=recent, **outs)
    assert np.array_equal(host(got), lens)
    assert np.array_equal(host(pool).reshape(want.shape), want)
    got_w, got_p = (host(w), host(p)) if in_place else (host(outs["weights_out"]), host(outs["token_pos_out"]))
    for s, k in enumerate(lens):
        assert np.array_equal(got_w[s, :, :k], w2[s, :, :k]) and np.array_equal(got_p[s, :, :k], p2[s, :, :k])
        if in_place:
            assert np.array_equal(got_w[s, :, k:], weights[s, :, k:]) and np.array_equal(got_p[s, :, k:], token_pos[s, :, k:])
        else:
            assert (got_w[s, :, k:] == -1).all() and (got_p[s, :, k:] == -1).all()
            assert np.array_equal(host(w), weights) and np.array_equal(host(p), token_pos)


def test_evict_by_weights_of_all_kinds():
    """Equal, negative, infinite and NaN weights, both zeros: NaN leaves first, equals stay by place."""
    c = ref.case(TINY, (DP, 1, 0), [257] * 6, [0] * 6)
    weights, token_pos = evict_inputs(c, np.random.default_rng(15), ties=False)
    weights[0] = 1.5
    weights[1] = np.where(weights[1] > 1, np.float32(0.0), np.float32(-0.0))
    weights[2] = np.where(weights[2] > 2, np.float32(np.nan), -weights[2])
    weights[3] = np.where(weights[3] > 1, np.float32(np.inf), np.float32(-np.inf))
    weights[4] = np.nan
    weights[5] = np.arange(weights[5].size, dtype=np.float32).reshape(weights[5].shape) * np.float32(1e-45)
    keep, next_pos = np.array([100, 256, 180, 90, 13, 128]), np.full(6, 300, np.int32)
    want, w2, p2, lens = ref.evicted(c, c.pool, keep, weights, token_pos, next_pos, 2, 3)
    pool, w, p = dev(c.pool), dev(weights), dev(token_pos)
    kv.kv_evict(pool, view_of(c), dev(c.table), dev(c.ctx), dev(keep.astype(np.int32)), w, p, dev(next_pos), 257, sinks=2, recent=3)
    assert np.array_equal(host(pool).reshape(want.shape), want)
    for s, k in enumerate(lens):
        assert np.array_equal(host(w)[s, :, :k], w2[s, :, :k], equal_nan=True) and np.array_equal(host(p)[s, :, :k], p2[s, :, :k])

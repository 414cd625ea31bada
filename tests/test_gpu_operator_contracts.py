"""What the operators around the cache promise beyond the ordinary call: every group size of query heads, values that are no numbers, caches
whose places are used again, arrays that move along.  Against the plain 64-bit forms."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from operator_refs import DP
from paper_2602_22593_amd import binding as kv
from paper_2602_22593_amd import workloads as wl

from helpers import bf16_bits_to_f64
from test_gpu_operator_runs import read_back
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


def set_token(c, s, t, key=None, value=None):
    """Rows of token t of sequence s: a key of one element that counts, values of every third element; in the pool and in the logical arrays."""
    rows, _ = ref.view_rows(c, c.pool)
    b, slot = ref.place(c, s, t)
    a = int(c.seq_off[s]) + t
    if key is not None:
        for k in (rows[b, 0, slot], c.K[a]):
            k[...] = 0
            k[..., 0] = key
    if value is not None:
        for v in (rows[b, 1, slot], c.V[a]):
            v[..., ::3] = value


EIGHT, FAR, INF, NAN = 0x4100, 0xC40E, 0x7F80, 0x7FC0      # 8, -568: scores of -400 at 128 elements, -568 at 64


@pytest.mark.parametrize("bad", [INF, NAN])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bound,q_lens", [(100, [20, 45, 7]), (400000, [8, 3, 7]), (400000, [16, 1, 7]), (400000, [64, 45, 31])])
def test_a_tree_row_meets_what_it_sees(bound, q_lens, d, bad):
    """An infinity or NaN in the values of a drafted token reaches the rows that see it however little it weighs: a weight past the
    smallest number times infinity is no number.  Rows that do not see it are as without it."""
    ctx = [100, 45, 31]
    c = ref.case((16, 4, d, 16), (DP, 1, 0), ctx, q_lens, index=81)
    c.q[:, :, 0] = EIGHT
    seen = np.random.default_rng(38).random((len(c.q), 64)) < 0.5
    for s in range(3):
        node = int(c.q_lens[s]) // 2
        set_token(c, s, int(c.ctx[s] - c.q_lens[s]) + node, FAR, bad)
        if c.q_lens[s] > 1:
            seen[c.q_off[s]:c.q_off[s + 1], node - 1] = True      # (another one, of ordinary weight)
    hit = np.array([seen[r, int(c.q_lens[s]) // 2] for s in range(3) for r in range(int(c.q_off[s]), int(c.q_off[s + 1]))])
    want, tol = ref.tree_attention(c, seen)
    got = bf16_bits_to_f64(host(kv.paged_tree_attn(dev(c.q), dev(c.pool), dev(wide_table(c, bound)), dev(c.ctx),
                                                       dev(c.q_off.astype(np.int32)), dev(ref.pack(seen)), view_of(c), bound, max(q_lens))))
    assert hit.any() and not hit.all()
    keep = np.arange(d) % 3 != 0
    assert (np.abs(got[~hit] - want[~hit]) <= tol[~hit]).all()
    assert (np.abs(got[hit] - want[hit]) <= tol[hit])[:, :, keep].all() and not np.isfinite(got[hit][:, :, ::3]).any()


@pytest.mark.parametrize("bad", [INF, NAN])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,bound", [(2, 1000), (4, WIDE)])
@pytest.mark.parametrize("low", [32, 64, 256])
def test_a_decode_row_meets_every_value(low, heads, bound, d, bad):
    """The same with sums of weights: tokens that weigh nothing, a tile, a wavefront's share or a whole piece of them, one with such values."""
    c = decode_case((4 * heads, heads, d, 16), [1000, 400], index=82)
    c.q[:, :, 0] = EIGHT
    for t in range(low):
        set_token(c, 0, t, FAR)
    set_token(c, 0, 10, value=bad)
    prior = np.zeros((2, heads, bound), np.float32)
    want, tol, sums, sums_tol = ref.decode_weights(c, prior)
    weights = dev(prior)
    out = kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), dev(wide_table(c, bound)), dev(c.ctx), view_of(c), bound, weights)
    got, keep = bf16_bits_to_f64(host(out)), np.arange(d) % 3 != 0
    assert (np.abs(got - want) <= tol)[:, :, keep].all() and (np.abs(got[1] - want[1]) <= tol[1]).all()
    assert not np.isfinite(got[0][:, ::3]).any()
    assert (np.abs(host(weights).astype(np.float64) - sums) <= sums_tol).all()


def accepted_entries(c, nodes, counts, values):
    """Values per token [batch][heads][tokens] after acceptance."""
    out = values.copy()
    for s, k in enumerate(counts):
        first = int(c.ctx[s] - c.q_lens[s])
        for i in range(int(k)):
            if first + nodes[s][i] < values.shape[2]:
                out[s, :, first + i] = values[s, :, first + nodes[s][i]]
    return out


@pytest.mark.parametrize("through_c", [True, False])
@pytest.mark.parametrize("geom,triple,ctx,q_lens,counts", [
    ((8, 2, 64, 16), (DP, 1, 0), [17, 1, 300, 64], [3, 1, 8, 5], [2, 1, 0, 5]),
    ((32, 8, 128, 16), (DP, 1, 0), [700, 256, 40], [64, 256, 40], [7, 200, 39]),
    ((32, 8, 128, 16), (ref.TP, 4, 3), [90, 0, 33], [33, 0, 17], [12, 0, 1]),
    ((32, 8, 128, 16), (DP, 2, 1), [300], [300], [270]),
    ((6, 2, 96, 5), (ref.TP, 2, 1), [23, 9], [11, 9], [4, 6]),
    ((300, 300, 64, 16), (DP, 1, 0), [40], [20], [9]),              # values per token of many workgroups
])
def test_acceptance_moves_what_is_kept_per_token(geom, triple, ctx, q_lens, counts, through_c):
    c = ref.case(geom, triple, ctx, q_lens, index=83)
    rng, hl = np.random.default_rng(39), c.info["n_kv_local"]
    nodes = np.full((len(ctx), max(counts) + 2), -1, np.int32)
    for s, k in enumerate(counts):
        nodes[s, :k] = np.sort(rng.permutation(int(c.q_lens[s]))[:k])
    pos = rng.integers(0, 1 << 30, (len(ctx), hl, max(ctx) + 3)).astype(np.int32)
    w = rng.random((len(ctx), hl, max(max(ctx) - 6, 1))).astype(np.float32)       # (some places have no entry)
    want, lens = ref.accepted_pool(c, c.pool, nodes, counts)
    args = (view_of(c), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), dev(nodes), dev(np.asarray(counts, np.int32)))
    for token_pos, weights in ((pos, w), (pos, None), (None, w)):
        pool, kept = dev(c.pool), [None if x is None else dev(x) for x in (token_pos, weights)]
        new = torch.zeros(len(ctx), dtype=torch.int32, device=DEV) if through_c else None
        got = kv.kv_accept(pool, *args, new_lens=new, token_pos=kept[0], weights=kept[1])
        assert np.array_equal(host(pool).reshape(want.shape), want) and np.array_equal(host(got), lens)
        for x, y in zip(kept, (token_pos, weights)):
            if x is not None:
                assert np.array_equal(host(x), accepted_entries(c, nodes, counts, y))
    with pytest.raises(ValueError, match="token_pos"):
        kv.kv_accept(dev(c.pool), *args, new_lens=torch.zeros(len(ctx), dtype=torch.int32, device=DEV), token_pos=dev(pos).long())


def longest_path(seen):
    """Nodes of the deepest path of a tree: bool [nodes][nodes], a row for each."""
    return max((np.flatnonzero(row[:len(seen)]) for row in seen), key=len)


@pytest.mark.parametrize("through_c", [True, False])
@pytest.mark.parametrize("geom,triple", [((32, 8, 128, 16), (ref.TP, 2, 1)), ((8, 2, 64, 16), (DP, 1, 0))])
def test_drafts_on_a_budget(geom, triple, through_c):
    """Prompts, then steps that draft, verify, accept several tokens, decode one with sums of weights, and go back to the budget in place.
    Arrays per token start as they come: whatever was there, and whatever evicted tokens left, counts for nothing."""
    start, steps, q_lens = np.array([70, 41, 9], np.int32), 7, np.array([9, 14, 5], np.int32)
    budget, sinks, recent = np.array([60, 45, 30]), 2, 12
    c = ref.case(geom, triple, start + steps * (q_lens + 1), q_lens, index=84)
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], geom[2]
    view, most, rng, g = view_of(c), int(c.ctx.max()), np.random.default_rng(40), wl.generator(85, wl.SUB_MISC)
    pool, table, freq = dev(c.pool), dev(c.table), dev((1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32))
    weights = torch.full((3, hl, most), 1e6, device=DEV)
    token_pos = torch.full((3, hl, most), 1 << 29, dtype=torch.int32, device=DEV)
    model = host(weights)                       # of weights: verified values, zeros where tokens were written

    def append(lens, counts, positions):
        total = int(counts.sum())
        x = dev(wl.randn_bf16((total, ql + 2 * hl, d), g))
        out = torch.zeros((total, ql, d), dtype=torch.bfloat16, device=DEV) if through_c else None
        off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        for s in range(3):
            model[s, :, lens[s] - counts[s]:lens[s]] = 0
        return kv.kv_rope_append(pool, view, x[:, :ql], x[:, ql:ql + hl], x[:, ql + hl:], dev(positions.astype(np.int32)), freq, table,
                                 dev(lens.astype(np.int32)), dev(off), out=out, token_pos=token_pos, weights=weights)

    append(start, start, np.concatenate([np.arange(k) for k in start]))
    lens, next_pos, evictions = start.astype(np.int64), start.astype(np.int64), 0
    for step in range(steps):
        seen, words = ref.tree_masks(q_lens, rng)
        trees = [seen[a:a + k, :k] for a, k in zip(c.q_off, q_lens)]
        q = append(lens + q_lens, q_lens, np.concatenate([next_pos[s] + trees[s].sum(axis=1) - 1 for s in range(3)]))
        c.ctx, c.q = (lens + q_lens).astype(np.int32), host(q)
        read_back(c, pool)
        n, off = dev(c.ctx), dev(c.q_off.astype(np.int32))
        within(host(kv.paged_tree_attn(q, pool, table, n, off, dev(words), view, most, int(q_lens.max()))), *ref.tree_attention(c, seen), f"step {step}")
        paths = [longest_path(x) for x in trees]
        counts = np.array([len(x) for x in paths], np.int32)
        nodes = np.zeros((3, counts.max()), np.int32)
        for s, x in enumerate(paths):
            nodes[s, :len(x)] = x
        before = host(pool).reshape(c.pool.shape)
        new = kv.kv_accept(pool, view, table, n, off, dev(nodes), dev(counts), token_pos=token_pos, weights=weights,
                           new_lens=torch.zeros(3, dtype=torch.int32, device=DEV) if through_c else None)
        want_pool, want_lens = ref.accepted_pool(c, before, nodes, counts)
        assert np.array_equal(host(pool).reshape(before.shape), want_pool) and np.array_equal(host(new), want_lens)
        lens, next_pos = want_lens + 1, next_pos + counts + 1
        q = append(lens, np.ones(3, np.int32), next_pos - 1)
        c.ctx, c.q = lens.astype(np.int32), host(q)
        read_back(c, pool)
        kv.paged_decode_attn_weights(q, pool, table, dev(c.ctx), view, most, weights)
        _, _, sums, sums_tol = ref.decode_weights(c, model)
        model, pos = host(weights), host(token_pos)
        for s in range(3):
            here = slice(0, int(lens[s]))
            assert (np.abs(model[s, :, here].astype(np.float64) - sums[s, :, here]) <= sums_tol[s, :, here]).all(), (step, s)
            for h in range(hl):           # every token is there once, the recent ones and the first ones without a gap
                there = set(pos[s, h, here].tolist())
                assert len(there) == lens[s] and set(range(max(next_pos[s] - recent, 0), next_pos[s])) | set(range(sinks)) <= there
                assert max(there) == next_pos[s] - 1
        if (lens > budget).any():
            keep = np.minimum(lens, budget).astype(np.int32)
            kv.kv_evict(pool, view, table, dev(c.ctx), dev(keep), weights, token_pos, dev(next_pos.astype(np.int32)), most, sinks=sinks, recent=recent)
            _, w2, p2, _ = ref.evicted(c, host(pool).reshape(c.pool.shape), keep, model, pos, next_pos, sinks, recent)
            assert np.array_equal(host(weights), w2) and np.array_equal(host(token_pos), p2)
            model, lens, evictions = host(weights), keep.astype(np.int64), evictions + 1
    assert evictions >= 4


def test_append_clears_the_weights_of_what_it_writes():
    """Entries of other tokens stay, and those of tokens without a place in the pool or in the array."""
    c = ref.case((8, 2, 64, 16), (DP, 1, 0), [20, 20, 20, 40], [1, 1, 1, 30], index=86)
    ctx, table = c.ctx.copy(), c.table.copy()
    ctx[0], table[1, 1], table[2, 1] = 0, -1, len(c.pool)
    qkv = dev(wl.randn_bf16((33, 12, 64), wl.generator(87, wl.SUB_MISC)))
    weights = torch.full((4, 2, 25), 3.0, device=DEV)
    kv.kv_rope_append(dev(c.pool), view_of(c), qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], dev(np.arange(33, dtype=np.int32)),
                      dev(np.ones(32, np.float32)), dev(table), dev(ctx), dev(c.q_off.astype(np.int32)), weights=weights)
    want = np.full((4, 2, 25), 3.0, np.float32)
    want[3, :, 10:] = 0
    assert np.array_equal(host(weights), want)


@pytest.mark.parametrize("call", ["tree", "weights", "prefill"])
def test_workspace_of_a_graph_outlives_a_larger_one(call):
    """A call without a workspace is captured on a stream; then an eager call there needs more.  The graph still writes to its own."""
    c = ref.case((8, 2, 128, 16), (DP, 1, 0), [2000, 700], [9, 30], index=88)
    view, words = view_of(c), dev(ref.tree_masks(c.q_lens, np.random.default_rng(41))[1])
    q, pool, table, n, off = dev(c.q), dev(c.pool), dev(wide_table(c, WIDE)), dev(c.ctx), dev(c.q_off.astype(np.int32))
    weights, out = torch.zeros((2, 2, WIDE), device=DEV), torch.zeros_like(q)

    def run(bound, out):
        if call == "tree":
            return kv.paged_tree_attn(q, pool, table, n, off, words, view, bound, 30, out=out)
        if call == "prefill":
            return kv.paged_prefill_attn(q, pool, table, n, off, view, bound, 30, out=out)
        return kv.paged_decode_attn_weights(q[:2], pool, table, n, view, bound, weights, out=out[:2])

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    key = (0, side.cuda_stream, "scratch")
    kv._workspaces.pop(key, None)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        kv._workspace(q.device, 1 << 21)                # what an eager call before left, of an ordinary size
        run(2000, out)
        want = host(out)
        with torch.cuda.graph(graph, stream=side):
            run(2000, out)
        mine = kv._workspaces[key]
        address, size = mine.data_ptr(), mine.numel()
        del mine
        kv._workspace(q.device, size + (1 << 20))       # a larger call comes
        assert kv._workspaces[key].data_ptr() != address
        others = [torch.full((size,), 0x5a, dtype=torch.uint8, device=DEV) for _ in range(4)]
        assert all(not x.data_ptr() <= address < x.data_ptr() + size for x in others)
    torch.cuda.synchronize()
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(out), want) and all(bool((x == 0x5a).all()) for x in others)


@pytest.mark.parametrize("geom,ctx,bound", [
    ((8, 2, 64, 16), [17, 1, 300, 64], 300),
    ((10, 2, 128, 48), [777, 97], 777),
    ((32, 8, 128, 16), [700, 33, 2100], WIDE),
    ((48, 4, 64, 16), [513, 1100], WIDE),
    ((64, 2, 128, 16), [1100, 31], 1100),
])
def test_decode_with_sums_rounds_its_output_alone(geom, ctx, bound):
    """The weights that are handed out in 32 bits are those that the values are added up with: each enters the product in two parts of
    bf16, whose second is off by 2^-8 of the first's 2^-8.  So out is off by 2^-16 sum p |v|, and 2^-15 of it and of itself for sums, the
    quotient and exponentials in fp32 (as elsewhere), before its one rounding."""
    c = decode_case(geom, ctx, index=89)
    weights = torch.zeros((len(ctx), geom[1], bound), device=DEV)
    got = bf16_bits_to_f64(host(kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), dev(wide_table(c, bound)), dev(c.ctx), view_of(c), bound, weights)))
    G, q = geom[0] // geom[1], bf16_bits_to_f64(c.q)
    for s, n in enumerate(ctx):
        K, V = ref.heads_of(c, s)
        for i in range(geom[0]):
            want, _, p = ref.attend(q[s, i][None], K[:, i // G], V[:, i // G], np.ones((1, n), bool), geom[2] ** -0.5)
            off = (2.0 ** -15 + 2.0 ** -16) * (p @ np.abs(V[:, i // G]) + np.abs(want))
            assert (np.abs(got[s, i] - want[0]) <= ref.HALF_BF16 * (np.abs(want[0]) + off[0]) + off[0]).all(), (s, i)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,bound", [(2, 1000), (4, WIDE)])
@pytest.mark.parametrize("token", [3, 500, 999])
def test_infinite_values_in_decode_with_sums(token, heads, bound, d):
    """An infinity among the values is one in the output, with its sign, wherever it lies: no part of a weight turns it into NaN."""
    c = decode_case((4 * heads, heads, d, 16), [1000, 33, 1], index=90)
    set_token(c, 0, token, value=INF)
    set_token(c, 1, 32, value=INF | 0x8000)
    set_token(c, 2, 0, value=INF)                                   # of weight 1
    prior = np.zeros((3, heads, bound), np.float32)
    want, tol, sums, sums_tol = ref.decode_weights(c, prior)
    weights = dev(prior)
    out = kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), dev(wide_table(c, bound)), dev(c.ctx), view_of(c), bound, weights)
    got, keep = bf16_bits_to_f64(host(out)), np.arange(d) % 3 != 0
    assert (np.abs(got - want) <= tol)[:, :, keep].all()
    assert (got[[0, 2]][:, :, ::3] == np.inf).all() and (got[1][:, ::3] == -np.inf).all()
    assert (np.abs(host(weights).astype(np.float64) - sums) <= sums_tol).all()


def test_padded_batch():
    """A batch filled up with sequences of no tokens goes through every operator: their rows are zeros, nothing of theirs is written, and
    their lengths stay 0."""
    ctx, q_lens = [40, 0, 23, 0], [6, 1, 3, 4]
    c = ref.case((8, 2, 64, 16), (DP, 1, 0), ctx, np.minimum(ctx, q_lens), index=91)
    off = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    view, pool, table, n = view_of(c), dev(c.pool), dev(c.table), dev(c.ctx)
    qkv = dev(wl.randn_bf16((14, 12, 64), wl.generator(92, wl.SUB_MISC)))
    token_pos, weights = torch.full((4, 2, 48), -7, dtype=torch.int32, device=DEV), torch.full((4, 2, 48), 5.0, device=DEV)
    q = kv.kv_rope_append(pool, view, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], dev(np.arange(14, dtype=np.int32)), dev(np.ones(32, np.float32)),
                          table, n, dev(off), token_pos=token_pos, weights=weights)
    words = dev(np.concatenate([ref.tree_masks([k], np.random.default_rng(42))[1] for k in q_lens]))
    out = kv.paged_tree_attn(q, pool, table, n, dev(off), words, view, 48, 6)
    assert not out[6].any() and not out[10:].any() and out[:6].any() and out[7:10].any()
    for count in (0, 1):
        new = kv.kv_accept(pool, view, table, n, dev(off), dev(np.zeros((4, 2), np.int32)), dev(np.array([2, count, 1, count], np.int32)),
                           token_pos=token_pos, weights=weights)
        assert host(new).tolist() == [36, 0, 21, 0]
    got = kv.paged_decode_attn_weights(q[:4].contiguous(), pool, table, new, view, 48, weights)
    assert not got[1].any() and not got[3].any() and got[0].any()
    state = host(pool)
    new2 = kv.kv_evict(pool, view, table, new, dev(np.full(4, 30, np.int32)), weights, token_pos, n, 48, sinks=1, recent=5)
    assert host(new2).tolist() == [30, 0, 21, 0]
    for x, untouched in ((host(weights), 5.0), (host(token_pos), -7)):
        assert (x[[1, 3]] == untouched).all()
    moved = np.flatnonzero((host(pool) != state).reshape(len(state), -1).any(axis=1))
    assert len(moved) and set(moved) <= set(c.table[0][:3].tolist())


@pytest.mark.parametrize("batch", [3, 100])
def test_a_batch_of_nothing(batch):
    """Bounds of 0 and 1 where no sequence has a token."""
    view = kv.kv_view_create(8, 2, 64, 16, DP, 1, 0)
    pool = torch.full((4, 2 * 16 * 2 * 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    n, table = torch.zeros(batch, dtype=torch.int32, device=DEV), torch.full((batch, 1), -1, dtype=torch.int32, device=DEV)
    q = torch.ones((batch, 8, 64), dtype=torch.bfloat16, device=DEV)
    for bound in (0, 1):
        weights = torch.full((batch, 2, 3), 5.0, device=DEV)
        out = torch.ones_like(q)
        assert not kv.paged_decode_attn_weights(q, pool, table, n, view, bound, weights, out=out).any() and (weights == 5.0).all()
        pos = torch.zeros((batch, 2, 3), dtype=torch.int32, device=DEV)
        assert not kv.kv_evict(pool, view, table, n, n, weights, pos, n, bound).any() and (weights == 5.0).all()
    off = torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    out = torch.ones_like(q)
    assert not kv.paged_tree_attn(q, pool, table, n, off, torch.full((batch, 1), -1, dtype=torch.int64, device=DEV), view, 1, 1, out=out).any()
    assert pool.isnan().all()

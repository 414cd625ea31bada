"""The operators around the cache as an engine uses them together: a speculative step from rotated drafts to the accepted cache, a
cache held to its budget over decode steps, captured graphs, two streams, pools past 4 GiB.  Every stage is checked against the
plain 64-bit forms fed with what the stage before left on the GPU."""
import numpy as np
import pytest
import torch

import operator_refs as ref
from operator_refs import DP, TP
from paper_2602_22593_amd import binding as kv
from paper_2602_22593_amd import workloads as wl

from helpers import bf16_bits_to_f64
from test_gpu_operators import DEV, G8B, TINY, dev, host, view_of, within

pytestmark = pytest.mark.gpu
HALVES = kv.KV_ROPE_HALVES


def read_back(c, pool):
    """The case's logical K and V as the pool holds them now (of the exposed heads)."""
    rows, h0 = ref.view_rows(c, host(pool).reshape(c.pool.shape))
    hl, g0 = c.info["n_kv_local"], c.info["kv_head0"]
    for s in range(len(c.ctx)):
        b, slot = ref.place(c, s, np.arange(c.ctx[s]))
        a = int(c.seq_off[s])
        c.K[a:a + c.ctx[s], g0:g0 + hl] = rows[b, 0, slot, h0:h0 + hl]
        c.V[a:a + c.ctx[s], g0:g0 + hl] = rows[b, 1, slot, h0:h0 + hl]


@pytest.mark.parametrize("geom,triple", [(G8B, (DP, 1, 0)), (G8B, (TP, 4, 1)), (TINY, (TP, 2, 1))])
def test_speculative_step(geom, triple):
    ctx, q_lens = [130, 64, 37], [12, 33, 5]
    c = ref.case(geom, triple, ctx, q_lens)
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], geom[2]
    rng, view = np.random.default_rng(30), view_of(c)
    pool, table, n, off = dev(c.pool), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32))
    seen, words = ref.tree_masks(c.q_lens, rng)
    # a node's position is its depth behind the context
    depth = np.array([seen[r].sum() - 1 for r in range(len(seen))])
    first = np.repeat(c.ctx - c.q_lens, c.q_lens)
    qkv = wl.randn_bf16((len(seen), ql + 2 * hl, d), wl.generator(62, wl.SUB_MISC))
    freq = (1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    positions = (first + depth).astype(np.int32)
    parts = dev(qkv)
    q = kv.kv_rope_append(pool, view, parts[:, :ql], parts[:, ql:ql + hl], parts[:, ql + hl:], dev(positions), dev(freq), table, n, off)
    want, tol = ref.rotated(bf16_bits_to_f64(qkv)[:, :ql], positions[None], freq, [0] * (d // 2), False)
    within(host(q), want, tol, "queries")
    read_back(c, pool)
    c.q = host(q)
    out = kv.paged_tree_attn(q, pool, table, n, off, dev(words), view, max(ctx), max(q_lens))
    within(host(out), *ref.tree_attention(c, seen), "tree")
    # the longest path of every draft is accepted
    paths = [max((np.flatnonzero(seen[r, :q_lens[s]]) for r in range(int(c.q_off[s]), int(c.q_off[s + 1]))), key=len) for s in range(3)]
    counts = np.array([len(p) for p in paths], np.int32)
    nodes = np.zeros((3, counts.max()), np.int32)
    for s, p in enumerate(paths):
        nodes[s, :len(p)] = p
    before = host(pool).reshape(c.pool.shape)
    new = kv.kv_accept(pool, view, table, n, off, dev(nodes), dev(counts))
    want_pool, lens = ref.accepted_pool(c, before, nodes, counts)
    assert np.array_equal(host(pool).reshape(before.shape), want_pool) and np.array_equal(host(new), lens)
    # and the next token attends to what was kept: the accepted path, in order, behind the context
    keep = [np.concatenate([np.arange(ctx[s] - q_lens[s]), ctx[s] - q_lens[s] + paths[s]]) for s in range(3)]
    q1 = wl.randn_bf16((3, ql, d), wl.generator(63, wl.SUB_QUERY))
    got = kv.paged_decode_attn(dev(q1), pool, table, new, view, int(lens.max()))
    for s in range(3):
        K, V = ref.heads_of(c, s)
        for i in range(ql):
            g = i // (ql // hl)
            row, bound, _ = ref.attend(bf16_bits_to_f64(q1)[s, i][None], K[keep[s], g], V[keep[s], g], np.ones((1, len(keep[s])), bool), d ** -0.5)
            assert (np.abs(bf16_bits_to_f64(host(got)[s, i]) - row[0]) <= bound[0]).all(), (s, i)


@pytest.mark.parametrize("geom,triple", [(G8B, (TP, 2, 0)), (TINY, (DP, 1, 0))])
def test_cache_held_to_its_budget(geom, triple):
    """A prompt, then decode steps that append, attend and add up weights; every few steps the caches go back to their budgets."""
    start, steps, budget, slack = np.array([90, 41, 7], np.int32), 24, np.array([64, 48, 20], np.int32), 8
    c = ref.case(geom, triple, start + steps, [1, 1, 1])
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], geom[2]
    view, most = view_of(c), int(c.ctx.max())
    pool, table = dev(c.pool), dev(c.table)
    weights = torch.zeros((3, hl, most), device=DEV)
    token_pos = torch.full((3, hl, most), -9, dtype=torch.int32, device=DEV)
    freq = (1e4 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    g = wl.generator(64, wl.SUB_MISC)
    total, off = int(start.sum()), np.concatenate([[0], np.cumsum(start)]).astype(np.int32)
    qkv = dev(wl.randn_bf16((total, ql + 2 * hl, d), g))
    pos = np.concatenate([np.arange(k) for k in start]).astype(np.int32)
    kv.kv_rope_append(pool, view, qkv[:, :ql], qkv[:, ql:ql + hl], qkv[:, ql + hl:], dev(pos), dev(freq), table, dev(start), dev(off),
                      token_pos=token_pos)
    lens, next_pos = start.copy(), start.copy()
    evictions = 0
    for step in range(steps):
        lens, next_pos = lens + 1, next_pos + 1
        qkv = dev(wl.randn_bf16((3, ql + 2 * hl, d), g))
        q = kv.kv_rope_append(pool, view, qkv[:, :ql], qkv[:, ql:ql + hl], qkv[:, ql + hl:], dev(next_pos - 1), dev(freq), table, dev(lens),
                              token_pos=token_pos)
        c.ctx = lens.astype(np.int32)
        read_back(c, pool)
        c.q, prior = host(q), host(weights)
        out = kv.paged_decode_attn_weights(q, pool, table, dev(c.ctx), view, most, weights)
        want, tol, sums, sums_tol = ref.decode_weights(c, prior)
        within(host(out), want, tol, f"step {step}")
        got = host(weights).astype(np.float64)
        for s in range(3):
            assert (np.abs(got[s, :, :lens[s]] - sums[s, :, :lens[s]]) <= sums_tol[s, :, :lens[s]]).all(), (step, s)
            p = host(token_pos)[s]
            for h in range(hl):           # every token is there once, the newest at the end
                assert len(set(p[h, :lens[s]])) == lens[s] and p[h, lens[s] - 1] == next_pos[s] - 1
        if (lens > budget + slack).any():
            state = host(pool).reshape(c.pool.shape), host(weights), host(token_pos)
            keep = np.where(lens > budget + slack, budget, lens).astype(np.int32)
            new = kv.kv_evict(pool, view, table, dev(c.ctx), dev(keep), weights, token_pos, dev(next_pos.astype(np.int32)), most, sinks=2, recent=10)
            want_pool, w2, p2, want_lens = ref.evicted(c, state[0], keep, state[1], state[2], next_pos, 2, 10)
            assert np.array_equal(host(pool).reshape(c.pool.shape), want_pool) and np.array_equal(host(new), want_lens)
            assert np.array_equal(host(weights), w2) and np.array_equal(host(token_pos), p2)
            lens, evictions = want_lens.copy(), evictions + 1
            for s in range(3):
                for h in range(hl):
                    kept = set(p2[s, h, :lens[s]])
                    assert set(range(next_pos[s] - min(10, lens[s]), next_pos[s])) <= kept
    assert evictions >= 3


def test_calls_in_python_and_in_c_agree():
    """The four calls that csrc/binding_calls.c marshals, with and without it, with and without a stream."""
    c = ref.case(G8B, (TP, 2, 1), [90, 33, 64], [7, 1, 20])
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], 128
    view, seen_words = view_of(c), ref.tree_masks(c.q_lens, np.random.default_rng(31))[1]
    qkv, freq = dev(wl.randn_bf16((28, ql + 2 * hl, d), wl.generator(65, wl.SUB_MISC))), dev((1e4 ** (-np.arange(64) / 64)).astype(np.float32))
    pos, axes = dev(np.arange(84, dtype=np.int32).reshape(3, 28)), [i % 3 for i in range(64)]
    table, n, off = dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32))
    nodes, counts = dev(np.array([[1, 3, 6], [0, 0, 0], [2, 4, 19]], np.int32)), dev(np.array([3, 0, 3], np.int32))
    q1 = dev(wl.randn_bf16((3, ql, d), wl.generator(66, wl.SUB_QUERY)))

    def run(stream):
        pool, token_pos = dev(c.pool), torch.zeros((3, hl, 100), dtype=torch.int32, device=DEV)
        weights, new = torch.full((3, hl, 90), 0.25, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
        q, out, out1 = (torch.zeros((k, ql, d), dtype=torch.bfloat16, device=DEV) for k in (28, 28, 3))
        ws = torch.zeros(kv.paged_tree_attn_workspace_bytes(view, 3, 28, 90, 20), dtype=torch.uint8, device=DEV)
        ws1 = torch.zeros(kv.paged_decode_attn_weights_workspace_bytes(view, 3, 90), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        assert kv.kv_rope_append(pool, view, qkv[:, :ql], qkv[:, ql:ql + hl], qkv[:, ql + hl:], pos, freq, table, n, off, axes=axes, out=q,
                                 token_pos=token_pos, stream=stream) is q
        assert kv.paged_tree_attn(q, pool, table, n, off, dev(seen_words), view, 90, 20, out=out, workspace=ws, stream=stream) is out
        assert kv.kv_accept(pool, view, table, n, off, nodes, counts, new_lens=new, stream=stream) is new
        assert kv.paged_decode_attn_weights(q1, pool, table, new, view, 90, weights, out=out1, workspace=ws1, stream=stream) is out1
        torch.cuda.synchronize()
        return [host(x) for x in (pool, token_pos, q, out, new, weights, out1)]

    class Counting:
        def __init__(self, module):
            self.module, self.answered = module, 0

        def __getattr__(self, name):
            def call(*args):
                rc = getattr(self.module, name)(*args)
                self.answered += rc is not None
                return rc
            return call

    was, results = kv._calls(), []
    try:
        for module, stream in ((was, None), (was, torch.cuda.Stream()), (kv._InPython(), None), (kv._InPython(), torch.cuda.Stream())):
            kv._calls_module = count = Counting(module)
            results.append(run(stream))
            if not isinstance(was, kv._InPython):
                assert count.answered == (4 if module is was else 0)
        # what the checks refuse is refused in Python, with its message
        kv._calls_module = was
        pool, q, new = dev(c.pool), torch.zeros((28, ql, d), dtype=torch.bfloat16, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
        for bad, text in ((lambda: kv.kv_accept(pool, view, table, n, off[:3], nodes, counts, new_lens=new), "q_offsets"),
                          (lambda: kv.kv_accept(pool, view, table, n, off, nodes.long(), counts, new_lens=new), "accepted"),
                          (lambda: kv.kv_rope_append(pool, view, qkv[:, :ql], qkv[:, ql:ql + hl], qkv[:, ql + hl:], pos, freq, table, n, off,
                                                     axes=axes[:3], out=q), "axes"),
                          (lambda: kv.kv_rope_append(pool, view, qkv[:, :ql], qkv[:, ql:ql + hl], qkv[:, ql + hl:], pos, freq, table, n, off,
                                                     out=q), "axes"),
                          (lambda: kv.kv_rope_append(pool, view, qkv[:, 1:ql + 1].transpose(1, 2), qkv[:, ql:ql + hl], qkv[:, ql + hl:], pos[0],
                                                     freq, table, n, off, out=q), "q has shape"),
                          (lambda: kv.kv_accept(pool, view, table, n.cpu(), off, nodes, counts, new_lens=new), "one device")):
            with pytest.raises(ValueError, match=text):
                bad()
        with pytest.raises(kv.KVError) as e:
            kv.kv_rope_append(pool, view, qkv[:, :ql], qkv[:, ql:ql + hl], qkv[:, ql + hl:], pos, freq, table, n, off, axes=[3] * 64, out=q)
        assert e.value.status == kv.KV_ERR_INVALID_ARG
    finally:
        kv._calls_module = was
    for other in results[1:]:
        assert all(np.array_equal(x, y) for x, y in zip(results[0], other))


def test_captured_and_replayed():
    """A speculative step and a step of a budgeted cache in one graph, replayed between eager work on the same buffers."""
    c = ref.case(G8B, (TP, 4, 2), [200, 90], [17, 30])
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], 128
    view, rng = view_of(c), np.random.default_rng(32)
    words = dev(ref.tree_masks(c.q_lens, rng)[1])
    qkv, freq = dev(wl.randn_bf16((47, ql + 2 * hl, d), wl.generator(67, wl.SUB_MISC))), dev((1e4 ** (-np.arange(64) / 64)).astype(np.float32))
    pos, table, n, off = dev(np.arange(47, dtype=np.int32)), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32))
    nodes, counts = dev(np.array([[0, 2, 9], [1, 20, 0]], np.int32)), dev(np.array([3, 2], np.int32))
    q1, keep, next_pos = dev(wl.randn_bf16((2, ql, d), wl.generator(68, wl.SUB_QUERY))), dev(np.array([100, 64], np.int32)), dev(c.ctx)
    clean = dev(c.pool)
    start_w = torch.rand((2, hl, 200), device=DEV)
    start_p = torch.argsort(torch.rand((2, hl, 200), device=DEV), dim=2).to(torch.int32)
    pool, w, p = clean.clone(), start_w.clone(), start_p.clone()
    q, out, out1 = (torch.zeros((k, ql, d), dtype=torch.bfloat16, device=DEV) for k in (47, 47, 2))
    new, new2 = (torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(2))
    ws = [torch.zeros(k, dtype=torch.uint8, device=DEV) for k in (
        kv.paged_tree_attn_workspace_bytes(view, 2, 47, 200, 30), kv.paged_decode_attn_weights_workspace_bytes(view, 2, 200),
        kv.kv_evict_workspace_bytes(view, 2, 200))]

    def step():
        kv.kv_rope_append(pool, view, qkv[:, :ql], qkv[:, ql:ql + hl], qkv[:, ql + hl:], pos, freq, table, n, off, out=q, token_pos=p)
        kv.paged_tree_attn(q, pool, table, n, off, words, view, 200, 30, out=out, workspace=ws[0])
        kv.kv_accept(pool, view, table, n, off, nodes, counts, new_lens=new)
        kv.paged_decode_attn_weights(q1, pool, table, new, view, 200, w, out=out1, workspace=ws[1])
        kv.kv_evict(pool, view, table, new, keep, w, p, next_pos, 200, sinks=1, recent=8, new_lens=new2, workspace=ws[2])

    def reset():
        pool.copy_(clean)
        w.copy_(start_w)
        p.copy_(start_p)
        for x in (q, out, out1, new, new2):
            x.zero_()

    results = (pool, w, p, q, out, out1, new, new2)
    step()                     # (first launches outside the capture)
    reset()
    step()
    torch.cuda.synchronize()
    want = [host(x) for x in results]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for replay in range(4):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(host(x), y, equal_nan=True) if x.dtype == torch.float32 else np.array_equal(host(x), y)
                   for x, y in zip(results, want)), replay
        reset()
        step()                 # the same work eagerly in between
        torch.cuda.synchronize()
        assert np.array_equal(host(out), want[4]) and np.array_equal(host(pool), want[0])


def test_two_streams_at_once():
    """Two sequences' worth of work on two streams, each with the binding's own workspaces: results as one after the other."""
    cases = [ref.case(G8B, (TP, 2, r), [700 + 90 * r, 300], [16, 8], index=70 + r) for r in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    inputs = []
    for c in cases:
        words = ref.tree_masks(c.q_lens, np.random.default_rng(33))[1]
        inputs.append((view_of(c), dev(c.q), dev(c.pool), dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), dev(words),
                       torch.zeros((2, c.info["n_kv_local"], int(c.ctx.max())), device=DEV)))

    def run(k, stream):
        view, q, pool, table, n, off, words, w = inputs[k]
        most = w.shape[2]
        w.zero_()
        outs = []
        for _ in range(5):
            outs.append(kv.paged_tree_attn(q, pool, table, n, off, words, view, most, 16, stream=stream))
            outs.append(kv.paged_decode_attn_weights(q[:2], pool, table, n, view, most, w, stream=stream))
        return outs + [w]

    torch.cuda.synchronize()
    want = []
    for k in range(2):
        got = run(k, None)
        torch.cuda.synchronize()
        want.append([host(x) for x in got])
    both = []
    for k in range(2):
        streams[k].wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(streams[k]):
            both.append(run(k, None))
    torch.cuda.synchronize()
    for got, exp in zip(both, want):
        assert all(np.array_equal(host(x), y) for x, y in zip(got, exp))


def test_pools_past_4_gib():
    """Blocks whose bytes lie past 4 GiB of the pool: every operator reaches them, and nothing else changes."""
    c = ref.case(G8B, (DP, 1, 0), [100, 47], [12, 30])
    shift, n_own = 72000, len(c.pool)                  # blocks of 64 KiB: 4.4 GiB
    small = dev(c.pool).view(torch.int16)
    big = torch.zeros((shift + n_own, small.shape[1]), dtype=torch.int16, device=DEV)
    big[shift:] = small
    table = dev(np.where(c.table >= 0, c.table + shift, c.table).astype(np.int32))
    near, view = dev(c.table), view_of(c)
    words = dev(ref.tree_masks(c.q_lens, np.random.default_rng(34))[1])
    n, off = dev(c.ctx), dev(c.q_off.astype(np.int32))
    qkv, freq = dev(wl.randn_bf16((42, 48, 128), wl.generator(69, wl.SUB_MISC))), dev((1e4 ** (-np.arange(64) / 64)).astype(np.float32))
    w0 = torch.rand((2, 8, 100), device=DEV)
    p0 = torch.argsort(torch.rand((2, 8, 100), device=DEV), dim=2).to(torch.int32)

    def run(pool, tab):
        w, p = w0.clone(), p0.clone()
        q = kv.kv_rope_append(pool, view, qkv[:, :32], qkv[:, 32:40], qkv[:, 40:], dev(np.arange(42, dtype=np.int32)), freq, tab, n, off)
        out = kv.paged_tree_attn(q, pool, tab, n, off, words, view, 100, 30)
        new = kv.kv_accept(pool, view, tab, n, off, dev(np.array([[3, 7], [1, 29]], np.int32)), dev(np.array([2, 2], np.int32)))
        out1 = kv.paged_decode_attn_weights(q[:2].contiguous(), pool, tab, new, view, 100, w)
        new2 = kv.kv_evict(pool, view, tab, new, dev(np.array([50, 9], np.int32)), w, p, n, 100, sinks=2, recent=4)
        return [host(x) for x in (q, out, new, out1, w, p, new2)]

    want, got = run(small, near), run(big, table)
    assert all(np.array_equal(x, y) for x, y in zip(want, got))
    assert torch.equal(big[shift:], small) and not big[:shift].any()


def test_positions_only_of_what_is_written():
    """token_pos stays as it is where a token has no place in the pool."""
    c = ref.case(TINY, (DP, 1, 0), [20, 20, 20, 20], [1, 1, 1, 1])
    ctx, table = c.ctx.copy(), c.table.copy()
    ctx[0], table[1, 1], table[2, 1] = 0, -1, len(c.pool)
    qkv = dev(wl.randn_bf16((4, 12, 64), wl.generator(71, wl.SUB_MISC)))
    token_pos = torch.full((4, 2, 20), -5, dtype=torch.int32, device=DEV)
    kv.kv_rope_append(dev(c.pool), view_of(c), qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], dev(np.arange(4, dtype=np.int32)),
                      dev(np.ones(32, np.float32)), dev(table), dev(ctx), token_pos=token_pos)
    want = np.full((4, 2, 20), -5, np.int32)
    want[3, :, 19] = 3
    assert np.array_equal(host(token_pos), want)


@pytest.mark.parametrize("geom,q_len", [(G8B, 1), (G8B, 13), (TINY, 20), (G8B, 50)])
def test_scores_of_great_size(geom, q_len):
    """Scores of a hundred and more either way: the running reference moves many times, few tokens hold all the weight.

    A score is off by e = 4 sqrt(d) 2^-24 sum |q k| scale and its exponent by 1.45 |score| 2^-22 besides, above and below the
    fraction: weights move by 2 e of themselves, the output by 2 e (sum p |v| + |out|), 4 e max |v| at most.
    """
    ctx, scale, d = [700, 33], 2.0, geom[2]
    c = ref.case(geom, (DP, 1, 0), ctx, [q_len, min(q_len, 33)], index=72)
    group = geom[0] // geom[1]
    seen, words = ref.tree_masks(c.q_lens, np.random.default_rng(35))
    want, tol = ref.tree_attention(c, seen, scale)
    q = bf16_bits_to_f64(c.q)
    for s in range(2):
        K, V = ref.heads_of(c, s)
        for i in range(geom[0]):
            rows = slice(int(c.q_off[s]), int(c.q_off[s + 1]))
            e = 4 * np.sqrt(d) * 2.0 ** -24 * scale * (np.abs(q[rows, i]) @ np.abs(K[:, i // group]).T).max(axis=1)
            e += 1.45 * 2.0 ** -22 * scale * np.abs(q[rows, i] @ K[:, i // group].T).max(axis=1)
            tol[rows, i] += 4 * e[:, None] * np.abs(V[:, i // group]).max()
    view, table, n = view_of(c), dev(c.table), dev(c.ctx)
    got = kv.paged_tree_attn(dev(c.q), dev(c.pool), table, n, dev(c.q_off.astype(np.int32)), dev(words), view, 700, q_len, scale=scale)
    within(host(got), want, tol)
    if q_len == 1:      # (a draft of one token that sees itself is a decode step)
        weights = torch.zeros((2, geom[1], 700), device=DEV)
        got = kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), table, n, view, 700, weights, scale=scale)
        within(host(got), want, tol)
        total = host(weights).astype(np.float64).sum(axis=2)
        assert np.abs(total - group).max() <= group * 2.0 ** -18      # n terms and a quotient in fp32


@pytest.mark.parametrize("geom,triple,ctx,q_lens", [
    (G8B, (DP, 1, 0), [600, 256, 1000, 64], [64, 256, 65, 1]),
    (G8B, (TP, 2, 1), [300, 77, 2000], [256, 77, 1]),
    (G8B, (DP, 2, 1), [90], [50]),
    (TINY, (DP, 1, 0), [500, 33, 300, 8], [200, 33, 256, 8]),
    ((20, 4, 64, 32), (DP, 1, 0), [77, 500, 200], [40, 33, 200]),
    ((64, 4, 128, 48), (TP, 2, 0), [300, 97, 256, 16], [12, 97, 256, 1]),
])
def test_large_batches_of_many_rows(geom, triple, ctx, q_lens):
    """Bounds and numbers of drafts for which eight wavefronts share a tile; a workspace asked for with other numbers serves."""
    c = ref.case(geom, triple, ctx, q_lens)
    bound = 400000
    table = np.pad(c.table, ((0, 0), (0, -(-bound // c.info["block_tokens"]) - c.table.shape[1])), constant_values=-1)
    seen, words = ref.tree_masks(c.q_lens, np.random.default_rng(36))
    want, tol = ref.tree_attention(c, seen)
    view = view_of(c)
    sizes = {kv.paged_tree_attn_workspace_bytes(view, len(ctx), total, bound, max(q_lens)) for total in (1, len(c.q), len(ctx) * max(q_lens))}
    assert len(sizes) == 1
    workspace = torch.full((sizes.pop(),), 0xff, dtype=torch.uint8, device=DEV)
    got = kv.paged_tree_attn(dev(c.q), dev(c.pool), dev(table), dev(c.ctx), dev(c.q_off.astype(np.int32)), dev(words), view, bound,
                             max(q_lens), workspace=workspace)
    within(host(got), want, tol)


@pytest.mark.parametrize("d,bad", [(128, np.nan), (64, np.inf)])
@pytest.mark.parametrize("q_lens", [[8, 3, 7], [16, 1, 7], [64, 45, 31]])
def test_large_batches_hide_what_is_not_finite(d, bad, q_lens):
    """As in small batches: infinities and NaN in drafted tokens' values reach the rows that see them; any bits; rows that see nothing."""
    ctx = [100, 45, 31]
    c = ref.case((16, 4, d, 16), (DP, 1, 0), ctx, q_lens)
    bound = 400000
    table = np.pad(c.table, ((0, 0), (0, -(-bound // c.info["block_tokens"]) - c.table.shape[1])), constant_values=-1)
    seen = np.random.default_rng(37).random((len(c.q), 64)) < 0.5
    rows, h0 = ref.view_rows(c, c.pool)
    hit = np.zeros(len(seen), bool)
    for s in range(3):
        node = int(c.q_lens[s]) // 2
        b, slot = ref.place(c, s, c.ctx[s] - c.q_lens[s] + node)
        rows[b, 1, slot, :, ::3] = 0x7FC0 if np.isnan(bad) else 0x7F80
        hit[c.q_off[s]:c.q_off[s + 1]] = seen[c.q_off[s]:c.q_off[s + 1], node]
    want, tol = ref.tree_attention(c, seen)
    got = bf16_bits_to_f64(host(kv.paged_tree_attn(dev(c.q), dev(c.pool), dev(table), dev(c.ctx), dev(c.q_off.astype(np.int32)),
                                                   dev(ref.pack(seen)), view_of(c), bound, max(q_lens))))
    assert hit.any() and not hit.all()
    keep = np.arange(d) % 3 != 0
    assert (np.abs(got[~hit] - want[~hit]) <= tol[~hit]).all()
    assert (np.abs(got[hit] - want[hit]) <= tol[hit])[:, :, keep].all() and not np.isfinite(got[hit][:, :, ::3]).any()


@pytest.mark.parametrize("seed", range(10))
def test_random_batches(seed):
    """Ragged batches of 1 to 70 sequences and bounds at random: whatever the shares come to, every tile counts once."""
    rng = np.random.default_rng(100 + seed)
    geom = [TINY, (4, 1, 128, 16), (6, 3, 64, 32), G8B][seed % 4]
    batch = int(rng.integers(1, 9)) if geom is G8B else int(rng.integers(1, 71))
    most = int(rng.choice([40, 300, 1500]))
    ctx = rng.integers(0, most + 1, batch)
    ctx[rng.integers(0, batch)] = most
    q_lens = np.minimum(rng.integers(0, int(rng.choice([2, 9, 40, 100])), batch), ctx)
    q_lens[ctx.argmax()] = max(q_lens.max(), 1)
    c = ref.case(geom, (DP, 1, 0), ctx, q_lens, index=73)
    seen, words = ref.tree_masks(np.maximum(c.q_lens, 0), rng)
    want, tol = ref.tree_attention(c, seen)
    bound, q_bound = most + int(rng.integers(0, 200)), int(min(q_lens.max() + rng.integers(0, 3), most))
    table = np.pad(c.table, ((0, 0), (0, max(0, -(-bound // c.info["block_tokens"]) - c.table.shape[1]))), constant_values=-1)
    words = np.pad(words, ((0, 0), (0, max(0, -(-q_bound // 64) - words.shape[1]))))
    view, tab, n = view_of(c), dev(table), dev(c.ctx)
    got = kv.paged_tree_attn(dev(c.q), dev(c.pool), tab, n, dev(c.q_off.astype(np.int32)), dev(words), view, bound, q_bound)
    within(host(got), want, tol)
    c.q = wl.randn_bf16((batch, geom[0], geom[2]), wl.generator(74, wl.SUB_QUERY))
    prior = rng.exponential(1e-2, (batch, geom[1], bound)).astype(np.float32)
    want, tol, sums, sums_tol = ref.decode_weights(c, prior)
    weights = dev(prior)
    within(host(kv.paged_decode_attn_weights(dev(c.q), dev(c.pool), tab, n, view, bound, weights)), want, tol)
    assert (np.abs(host(weights).astype(np.float64) - sums) <= sums_tol).all()

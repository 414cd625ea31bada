"""Plain 64-bit implementations, in numpy on logical tensors, of the operators around the cache: rotary append, attention of
drafted trees, acceptance, decode with summed weights, eviction; and the bounds that their results are held to."""
from __future__ import annotations

import numpy as np

import oracle
from paper_2602_22593_amd import workloads as wl

from helpers import bf16_bits_to_f64, make_prefill_case

DP, TP = oracle.LAYOUT_DP, oracle.LAYOUT_TP
HALF_BF16 = 2.0 ** -8      # half a step of bf16, relative


def case(geom, triple, ctx, q_lens, index=60):
    """A NaN-poisoned pool with the caches of these lengths, and queries; geom = (q heads, kv heads, head_dim, block size)."""
    w = wl.Workload("operators", index, *geom, len(ctx), "x", ())
    return make_prefill_case(w, triple, np.asarray(ctx, np.int32), np.asarray(q_lens, np.int32))


def view_rows(c, pool):
    """The pool as [block][plane][slot][stored head][d] and the first exposed head in a row."""
    i = c.info
    return pool.reshape(len(pool), 2, i["block_tokens"], i["row_heads"], c.w.head_dim), i["row_head0"]


def place(c, s, t):
    t = np.asarray(t)
    return c.table[s][t // c.info["block_tokens"]], t % c.info["block_tokens"]


def heads_of(c, s):
    """K and V of the exposed heads of sequence s in float64, [tokens][heads][d]."""
    h0, hl = c.info["kv_head0"], c.info["n_kv_local"]
    a = int(c.seq_off[s])
    b = a + int(c.ctx[s])
    return bf16_bits_to_f64(c.K[a:b, h0:h0 + hl]), bf16_bits_to_f64(c.V[a:b, h0:h0 + hl])


def attend(q, K, V, seen, scale):
    """(out, bound on its error, weights) of one head: q [rows][d], seen [rows][tokens]; rows that see nothing are zeros.

    The bound: weights enter the second product in bf16, each off by half a step, above and below the fraction, so out moves by
    at most 2^-8 sum p |v - out| / (1 - 2^-8); then one rounding of out.  Sums in fp32 and the exponentials are worth 2^-15 of
    sum p |v| with much to spare (scores up to 30, 2^-24 relative each way).
    """
    a = np.where(seen, (q @ K.T) * scale, -np.inf)
    top = a.max(axis=1, keepdims=True, initial=-np.inf)
    p = np.exp(a - np.where(np.isinf(top), 0.0, top))
    total = p.sum(axis=1, keepdims=True)
    p = p / np.where(total == 0, 1.0, total)
    v = np.where(np.isfinite(V), V, 0.0)
    out = p @ v
    spread = p @ np.abs(v) + np.abs(out)
    return out, 1.01 * HALF_BF16 * (spread + np.abs(out)) + 2.0 ** -15 * spread, p


def tree_masks(q_lens, rng, words=None):
    """bool [rows][256] of random trees (a node sees its ancestors and itself), and the same packed as int64 words."""
    words = words or max(1, -(-int(max(q_lens)) // 64))
    seen = np.zeros((int(np.sum(q_lens)), 64 * words), dtype=bool)
    at = 0
    for k in q_lens:
        for j in range(int(k)):
            up = int(rng.integers(-1, j)) if j and rng.random() < 0.6 else j - 1
            if up >= 0:
                seen[at + j] = seen[at + up]
            seen[at + j, j] = True
        at += int(k)
    return seen, pack(seen)


def pack(seen):
    return np.packbits(seen, axis=1, bitorder="little").view(np.int64)


def tree_attention(c, seen, scale=None):
    """Expected rows and their bounds [total][n_q_local][d]."""
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], c.w.head_dim
    G, scale = ql // hl, 1.0 / np.sqrt(d) if scale is None else scale
    q = bf16_bits_to_f64(c.q)
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(len(c.ctx)):
        m, n = int(c.q_lens[s]), int(c.ctx[s])
        if m == 0:
            continue
        K, V = heads_of(c, s)
        rows = slice(int(c.q_off[s]), int(c.q_off[s]) + m)
        sees = np.concatenate([np.ones((m, n - m), bool), seen[rows, :m]], axis=1)
        for h in range(ql):
            out[rows, h], tol[rows, h], _ = attend(q[rows, h], K[:, h // G], V[:, h // G], sees, scale)
    return out, tol


def decode_weights(c, prior):
    """(out, bound, weights, bound) of one decode step with summed weights; prior [batch][heads][tokens].

    The weights' bound: a score is a sum of d exact products in fp32, off by 4 sqrt(d) 2^-24 sum |q k| with overwhelming
    probability, its exponent by 2^-22 of itself besides, and numerator and denominator carry both; the denominator adds
    n terms, 4 sqrt(n) 2^-24; the sum with the prior rounds once.
    """
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], c.w.head_dim
    G, scale = ql // hl, 1.0 / np.sqrt(d)
    q = bf16_bits_to_f64(c.q)
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    sums, sums_tol = prior.astype(np.float64), np.zeros(prior.shape)
    for s in range(len(c.ctx)):
        n = int(c.ctx[s])
        if n == 0:
            continue
        K, V = heads_of(c, s)
        for h in range(hl):
            w, off = np.zeros(n), np.zeros(n)
            for i in range(h * G, (h + 1) * G):
                out[s, i], tol[s, i], p = attend(q[s, i][None], K[:, h], V[:, h], np.ones((1, n), bool), scale)
                x = np.abs(q[s, i]) @ np.abs(K[:, h]).T * scale
                e = 4 * np.sqrt(d) * 2.0 ** -24 * x.max() + 2.0 ** -22 * np.abs(q[s, i] @ K[:, h].T * scale).max() * 1.45
                w += p[0]
                off += p[0] * (2 * e + 4 * np.sqrt(n) * 2.0 ** -24 + 2.0 ** -20)
            sums[s, h, :n - 1] += w[:n - 1]
            sums[s, h, n - 1] = w[n - 1]
            sums_tol[s, h, :n] = off + 2.0 ** -23 * np.abs(sums[s, h, :n]) + 1e-30
    return out, tol, sums, sums_tol


def evicted(c, pool, keep, weights, token_pos, next_pos, sinks, recent):
    """Pool, weights, token_pos (as they are afterwards, below the new lengths) and lengths after an eviction."""
    pool, w2, p2 = pool.copy(), weights.copy(), token_pos.copy()
    rows, h0 = view_rows(c, pool)
    old = rows.copy()
    lens = np.minimum(c.ctx, np.maximum(keep, 0)).astype(np.int32)
    for s in range(len(c.ctx)):
        n, k = int(c.ctx[s]), int(lens[s])
        for h in range(c.info["n_kv_local"]):
            w, pos = weights[s, h, :n].astype(np.float64), token_pos[s, h, :n].astype(np.int64)
            guarded = (pos < sinks) | (pos >= int(next_pos[s]) - recent)
            order = sorted(range(n), key=lambda t: (not guarded[t], np.isnan(w[t]), -w[t] if w[t] == w[t] else 0.0, t))
            kept = set(order[:k])
            holes = [t for t in range(k) if t not in kept]
            late = [t for t in range(k, n) if t in kept]
            assert len(holes) == len(late)
            for to, src in zip(holes, late):
                (tb, ts), (sb, ss) = place(c, s, to), place(c, s, src)
                rows[tb, :, ts, h0 + h] = old[sb, :, ss, h0 + h]
                w2[s, h, to], p2[s, h, to] = weights[s, h, src], token_pos[s, h, src]
    return pool, w2, p2, lens


def accepted_pool(c, pool, nodes, counts):
    pool = pool.copy()
    rows, h0 = view_rows(c, pool)
    old, hl = rows.copy(), c.info["n_kv_local"]
    lens = np.zeros(len(c.ctx), np.int32)
    for s in range(len(c.ctx)):
        first = int(c.ctx[s] - c.q_lens[s])
        lens[s] = first + counts[s]
        for i in range(int(counts[s])):
            (tb, ts), (sb, ss) = place(c, s, first + i), place(c, s, first + nodes[s][i])
            rows[tb, :, ts, h0:h0 + hl] = old[sb, :, ss, h0:h0 + hl]
    return pool, lens


def rotated(x, positions, inv_freq, axes, adjacent):
    """(rows, bound) of x [tokens][heads][d] in float64; the bound: one rounding to bf16, and cosines, sines and products in
    fp32 (2^-21 of the pair's size: a sine off by 2^-22 of a turn's error or its own, two products, a sum)."""
    y, tol = x.copy(), np.zeros(x.shape)
    half = len(inv_freq)
    for f in range(half):
        i, j = (2 * f, 2 * f + 1) if adjacent else (f, f + half)
        a = positions[axes[f]].astype(np.longdouble) * np.longdouble(inv_freq[f])
        cos, sin = (np.asarray(fn(a), np.float64)[:, None] for fn in (np.cos, np.sin))
        y[..., i], y[..., j] = x[..., i] * cos - x[..., j] * sin, x[..., j] * cos + x[..., i] * sin
        # (at a position p the 64-bit angle is off by p 2^-53 turns, 2^-22 at most)
        size = (np.abs(x[..., i]) + np.abs(x[..., j])) * 2.0 ** -19
        tol[..., i] = HALF_BF16 * np.abs(y[..., i]) + size
        tol[..., j] = HALF_BF16 * np.abs(y[..., j]) + size
    return y, tol

"""Plain 64-bit forms of the operators on a cache held in 8 bits, in numpy on logical tensors, and the bounds that results are held to."""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

import operator_refs as ref
from operator_refs import HALF_BF16, place
from paper_2602_22593_amd import workloads as wl

from helpers import bf16_bits_to_f64

E4M3, INT8 = "e4m3", "int8"
LARGEST = {E4M3: 448.0, INT8: 127.0}
POISON = {E4M3: 0x7F, INT8: 0x80}      # NaN; a code that the library never writes
LEAST_SCALE = 2.0 ** -120


def _e4m3_values():
    v = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v[b] = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if b & 128 else 1)
    v[[0x7F, 0xFF]] = np.nan
    return v


VALUES = {E4M3: _e4m3_values(), INT8: np.arange(256).astype(np.uint8).view(np.int8).astype(np.float64)}


def values(codes, fmt):
    return VALUES[fmt][codes]


def nearest(y, fmt):
    """The code nearest to y (ties to even), as a number; y no larger than the largest."""
    if fmt == INT8:
        return np.rint(y)
    e = np.frexp(np.where(y == 0, 1.0, y))[1] - 1
    step = 2.0 ** (np.maximum(e, -6) - 3.0)
    return np.rint(y / step) * step


def codes_of(numbers, fmt):
    """The bytes of numbers that are codes."""
    if fmt == E4M3:
        pos = VALUES[fmt][:127]
        at = np.searchsorted(pos, np.abs(numbers))
        assert (pos[at] == np.abs(numbers)).all()
        return (at + 128 * np.signbit(numbers)).astype(np.uint8)
    return numbers.astype(np.int8).view(np.uint8)


def half_step(y, fmt):
    """Half the distance of the codes around y (in units of the scale)."""
    if fmt == INT8:
        return np.full(np.shape(y), 0.5)
    e = np.frexp(np.where(y == 0, 1.0, y))[1] - 1
    return 2.0 ** (np.maximum(e, -6) - 4.0)


def scale_for(top, fmt):
    """The smallest power of two, at least 2^-120, that brings `top` down to the largest code."""
    m, e = np.frexp(np.asarray(top, np.float64) / LARGEST[fmt])
    s = np.ldexp(1.0, np.where(m == 0.5, e - 1, e))
    return np.where(np.asarray(top) == 0, LEAST_SCALE, np.maximum(s, LEAST_SCALE))


@dataclass
class Q8Case:
    c: object                  # the tables, lengths, queries and views of a bf16 case
    fmt: str
    codes: np.ndarray          # uint8 [blocks][2][slots][heads of a row][d], poisoned where no valid token of an exposed head lies
    scales: np.ndarray         # fp32 [blocks][2][groups][heads of a row], NaN likewise

    @property
    def base(self):
        return self.c.w.base_block_size

    def group_of(self, s, t):
        """Block and group of token t of sequence s."""
        b, slot = place(self.c, s, t)
        return b, slot // self.base

    def cached(self, s):
        """K and V of the exposed heads of sequence s in float64, [tokens][heads][d]."""
        h0, hl = self.c.info["row_head0"], self.c.info["n_kv_local"]
        t = np.arange(self.c.ctx[s])
        (b, slot), (_, g) = place(self.c, s, t), self.group_of(s, t)
        return [values(self.codes[b, p, slot, h0:h0 + hl], self.fmt) * self.scales[b, p, g, h0:h0 + hl].astype(np.float64)[..., None]
                for p in (0, 1)]


def case(geom, triple, ctx, q_lens, fmt, index=80, powers=True, size=1.0):
    """Caches of these lengths with normal values; powers: under scales that are powers of two, others otherwise."""
    c = ref.case(geom, triple, ctx, q_lens, index)
    i, d, B = c.info, geom[2], geom[3]
    n = len(c.pool)
    x = Q8Case(c, fmt, np.full((n, 2, i["block_tokens"], i["row_heads"], d), POISON[fmt], np.uint8),
               np.full((n, 2, i["block_tokens"] // B, i["row_heads"]), np.nan, np.float32))
    rng = np.random.default_rng(index)
    h0, hl = i["row_head0"], i["n_kv_local"]
    for s in range(len(c.ctx)):
        k = int(c.ctx[s])
        if k == 0:
            continue
        t = np.arange(k)
        b, slot = place(c, s, t)
        y = np.clip(rng.standard_normal((k, 2, hl, d)) * LARGEST[fmt] / 4.5, -LARGEST[fmt], LARGEST[fmt])
        x.codes[b, :, slot, h0:h0 + hl] = codes_of(nearest(y, fmt), fmt)
        b, g = x.group_of(s, np.arange(0, k, B))
        unit = size * 4.5 / LARGEST[fmt]
        some = rng.integers(0, 2, (len(b), 2, hl))
        x.scales[b, :, g, h0:h0 + hl] = (2.0 ** np.ceil(np.log2(unit)) / 2.0 ** some) if powers else unit * (0.6 + 0.5 * rng.random(some.shape))
    return x


def attention(x, causal, scale=None, rounded=False):
    """Expected rows of decode (one query a sequence) or of several causal ones, and their bounds.  rounded: keys and values enter the
    products as bf16, off by half a step each: that moves a score by 2^-8 scale |q| . |k| at most, a weight by e to twice that, and out by
    2^-8 sum p |v| more."""
    c = x.c
    hl, ql, d = c.info["n_kv_local"], c.info["n_q_local"], c.w.head_dim
    G, scale = ql // hl, 1.0 / np.sqrt(d) if scale is None else scale
    q = bf16_bits_to_f64(c.q)
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(len(c.ctx)):
        m, n = (int(c.q_lens[s]) if causal else 1), int(c.ctx[s])
        if n == 0 or m == 0:
            continue
        K, V = x.cached(s)
        rows = slice(int(c.q_off[s]), int(c.q_off[s]) + m) if causal else slice(s, s + 1)
        seen = np.arange(n)[None, :] <= np.arange(n - m, n)[:, None]
        for h in range(ql):
            k, v = K[:, h // G], V[:, h // G]
            out[rows, h], tol[rows, h], p = ref.attend(q[rows, h], k, v, seen, scale)
            if rounded:
                e = HALF_BF16 * scale * (np.abs(q[rows, h]) @ np.abs(k).T)
                moved = np.expm1(2 * np.where(seen, e, 0).max(axis=1, keepdims=True))
                spread = p @ np.abs(v)
                tol[rows, h] += moved * (spread + np.abs(out[rows, h])) + HALF_BF16 * spread * (1 + moved)
    return out, tol


def appended(x, rows, new_lens):
    """Codes (as numbers), scales and the rows' bounds after writing `rows` [tokens][2][heads][d] (float64, rotated): (numbers of the whole
    pool with NaN for poison, scales).  Older tokens are rounded again where their scale grows."""
    c, B, fmt = x.c, x.base, x.fmt
    h0, hl = c.info["row_head0"], c.info["n_kv_local"]
    numbers, scales = values(x.codes, fmt), x.scales.copy()
    at = 0
    for s in range(len(c.ctx)):
        n, k = int(c.ctx[s]), int(new_lens[s])
        first = n - k
        for g0 in range(first // B * B, n, B):
            t = np.arange(max(g0, first), min(g0 + B, n))
            if len(t) == 0:
                continue
            new = rows[at + t - first]
            (b, slot), (gb, g) = place(c, s, t), x.group_of(s, g0)
            scale = scale_for(np.abs(new).max(axis=(0, 3)), fmt)
            if g0 < first:
                was = scales[gb, :, g, h0:h0 + hl].astype(np.float64)
                scale = np.maximum(scale, was)
                ob, oslot = place(c, s, np.arange(g0, first))
                numbers[ob, :, oslot, h0:h0 + hl] = nearest(numbers[ob, :, oslot, h0:h0 + hl] * (was / scale)[..., None], fmt)
            numbers[b, :, slot, h0:h0 + hl] = nearest(new / scale[..., None], fmt)
            scales[gb, :, g, h0:h0 + hl] = scale
        at += k
    return numbers, scales


def repacked(src, dst_c, codes, scales):
    """The pool and the scales after moving the tokens of src's case under its view to dst_c's table and view."""
    codes, scales = codes.copy(), scales.copy()
    a, z = src.c.info, dst_c.info
    lo, hi = max(a["kv_head0"], z["kv_head0"]), min(a["kv_head0"] + a["n_kv_local"], z["kv_head0"] + z["n_kv_local"])
    B, d = src.base, src.c.w.head_dim

    def laid(arr, info, last):
        return arr.reshape(len(arr), 2, info["block_tokens"] // (1 if last else B), info["row_heads"], *([d] if last else []))
    for x, last in ((codes, True), (scales, False)):
        old = laid(x.copy(), a, last)
        new = laid(x, z, last)
        for s in range(len(src.c.ctx)):
            t = np.arange(0, src.c.ctx[s], 1 if last else B)
            sb, ss = src.c.table[s][t // a["block_tokens"]], t % a["block_tokens"] // (1 if last else B)
            db, ds = dst_c.table[s][t // z["block_tokens"]], t % z["block_tokens"] // (1 if last else B)
            f, o = lo - a["kv_head0"] + a["row_head0"], lo - z["kv_head0"] + z["row_head0"]
            new[db, :, ds, o:o + hi - lo] = old[sb, :, ss, f:f + hi - lo]
    return codes, scales


def normal_rows(total, ql, hl, d, index):
    qkv = wl.randn_bf16((total, ql + 2 * hl, d), wl.generator(index, wl.SUB_MISC))
    return qkv

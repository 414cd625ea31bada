"""CPU checks of the operators around the cache: what the entry points refuse, before anything is launched, and pins of the
plain forms that the GPU tests compare with."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import operator_refs as ref
from paper_2602_22593_amd import binding as kv

from helpers import bf16_bits_to_f64, textbook_causal_attention

FAKE = C.c_void_p(256)
INVALID, UNSUPPORTED, TOO_SMALL = kv.KV_ERR_INVALID_ARG, kv.KV_ERR_UNSUPPORTED, kv.KV_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built_library():
    from paper_2602_22593_amd.build import ensure_built
    ensure_built()
    return kv.lib()


def view(hq=32, hkv=8, d=128, bs=16, layout=kv.KV_LAYOUT_DP, p=1, r=0):
    return kv.kv_view_create(hq, hkv, d, bs, layout, p, r)


def call(name, **changed):
    """The entry point with arguments that it takes, except for the changed ones (nothing here may reach a launch)."""
    v = changed.pop("view", view())
    common = dict(kv_pool=FAKE, n_pool_blocks=10, view=getattr(v, "handle", v), block_table=FAKE, stride=64, ctx=FAKE, batch=2, st=None)
    args = {
        "kv_rope_append": dict(kv_pool=0, n_pool_blocks=0, view=0, q=FAKE, q_stride=6144, k=FAKE, k_stride=6144, v=FAKE, v_stride=6144,
                               q_out=C.c_void_p(512), positions=FAKE, position_stride=9, n_axes=2, inv_freq=FAKE, rotary_dim=128,
                               axes=(C.c_int32 * 64)(), pairs=0, block_table=0, stride=0, ctx=0, q_off=FAKE, batch=0, total=9,
                               token_pos=None, token_pos_stride=0, st=0),
        "paged_tree_attn": dict(q=FAKE, out=FAKE, kv_pool=0, n_pool_blocks=0, block_table=0, stride=0, ctx=0, q_off=FAKE, mask=FAKE,
                                words=1, batch=0, total=9, max_ctx=1024, max_q=64, view=0, scale=0.0, ws=FAKE, ws_bytes=1 << 40, st=0),
        "kv_accept": dict(kv_pool=0, n_pool_blocks=0, view=0, block_table=0, stride=0, ctx=0, q_off=FAKE, accepted=FAKE, acc_stride=4,
                          n_accepted=FAKE, batch=0, new_lens=C.c_void_p(512), st=0),
        "paged_decode_attn_weights": dict(q=FAKE, out=FAKE, kv_pool=0, n_pool_blocks=0, block_table=0, stride=0, ctx=0, batch=0,
                                          max_ctx=1024, view=0, scale=0.0, weights=FAKE, w_stride=1024, ws=FAKE, ws_bytes=1 << 40, st=0),
        "kv_evict": dict(kv_pool=0, n_pool_blocks=0, view=0, block_table=0, stride=0, ctx=0, keep=C.c_void_p(512), batch=0, max_ctx=1024,
                         weights=FAKE, token_pos=FAKE, w_stride=1024, next_pos=FAKE, sinks=0, recent=0, w_out=FAKE, p_out=FAKE,
                         out_stride=1024, new_lens=C.c_void_p(768), ws=FAKE, ws_bytes=1 << 40, st=0),
    }[name]
    args.update({k: v for k, v in common.items() if k in args})
    assert set(changed) <= set(args), changed
    args.update(changed)
    return getattr(kv.lib(), name)(*args.values())


@pytest.mark.parametrize("name,changed,status", [
    *[("kv_rope_append", {x: None}, INVALID) for x in ("kv_pool", "view", "q", "k", "v", "q_out", "positions", "inv_freq", "block_table", "ctx")],
    *[("kv_rope_append", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "total", "rotary_dim", "position_stride")],
    ("kv_rope_append", dict(q_stride=4095), INVALID),
    ("kv_rope_append", dict(k_stride=1023), INVALID),
    ("kv_rope_append", dict(v_stride=1016), INVALID),
    ("kv_rope_append", dict(q_out=FAKE), INVALID),                 # in place needs contiguous tokens
    ("kv_rope_append", dict(position_stride=8), INVALID),
    ("kv_rope_append", dict(axes=(C.c_int32 * 64)(*[2] * 64)), INVALID),
    ("kv_rope_append", dict(pairs=2), INVALID),
    ("kv_rope_append", dict(n_axes=0), INVALID),
    ("kv_rope_append", dict(rotary_dim=130), INVALID),
    ("kv_rope_append", dict(q_off=None), INVALID),                 # nine tokens of two sequences
    ("kv_rope_append", dict(rotary_dim=24), UNSUPPORTED),
    ("kv_rope_append", dict(q_stride=6148), UNSUPPORTED),
    ("kv_rope_append", dict(k=C.c_void_p(264)), UNSUPPORTED),
    ("kv_rope_append", dict(n_axes=5), UNSUPPORTED),
    ("kv_rope_append", dict(view=view(d=72), rotary_dim=64), UNSUPPORTED),
    ("kv_rope_append", dict(batch=0, total=0, q=None), kv.KV_OK),
    *[("paged_tree_attn", {x: None}, INVALID) for x in ("q", "out", "kv_pool", "block_table", "ctx", "q_off", "mask", "view", "ws")],
    *[("paged_tree_attn", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "total", "max_ctx", "max_q", "words")],
    ("paged_tree_attn", dict(n_pool_blocks=0), INVALID),
    ("paged_tree_attn", dict(max_q=65), INVALID),                  # two words are needed
    ("paged_tree_attn", dict(max_ctx=32), INVALID),                # more new tokens than cached ones
    ("paged_tree_attn", dict(stride=63), INVALID),
    ("paged_tree_attn", dict(ws=C.c_void_p(264)), INVALID),
    ("paged_tree_attn", dict(ws_bytes=1024), TOO_SMALL),
    ("paged_tree_attn", dict(max_q=257, words=5), UNSUPPORTED),
    ("paged_tree_attn", dict(view=view(d=96)), UNSUPPORTED),
    ("paged_tree_attn", dict(view=view(hq=8 * 33)), UNSUPPORTED),
    ("paged_tree_attn", dict(view=view(bs=24), stride=4096), UNSUPPORTED),
    ("paged_tree_attn", dict(batch=0, q=None), kv.KV_OK),
    ("paged_tree_attn", dict(total=0, q=None), kv.KV_OK),
    *[("kv_accept", {x: None}, INVALID) for x in ("kv_pool", "view", "block_table", "ctx", "q_off", "accepted", "n_accepted")],
    *[("kv_accept", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "acc_stride", "batch")],
    ("kv_accept", dict(new_lens=FAKE), INVALID),                   # the lengths themselves
    ("kv_accept", dict(batch=0, kv_pool=None), kv.KV_OK),
    *[("paged_decode_attn_weights", {x: None}, INVALID) for x in ("q", "out", "kv_pool", "block_table", "ctx", "weights", "view", "ws")],
    *[("paged_decode_attn_weights", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "max_ctx")],
    ("paged_decode_attn_weights", dict(w_stride=1023), INVALID),
    ("paged_decode_attn_weights", dict(stride=63), INVALID),
    ("paged_decode_attn_weights", dict(ws_bytes=1 << 10), TOO_SMALL),
    ("paged_decode_attn_weights", dict(view=view(d=256)), UNSUPPORTED),
    ("paged_decode_attn_weights", dict(batch=0, q=None), kv.KV_OK),
    *[("kv_evict", {x: None}, INVALID) for x in ("kv_pool", "view", "block_table", "ctx", "keep", "weights", "token_pos", "next_pos",
                                                 "w_out", "p_out", "ws")],
    *[("kv_evict", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "max_ctx", "sinks", "recent", "out_stride")],
    ("kv_evict", dict(w_stride=1023), INVALID),
    ("kv_evict", dict(out_stride=1025), INVALID),                  # in place, but other rows
    ("kv_evict", dict(stride=63), INVALID),
    ("kv_evict", dict(new_lens=FAKE), INVALID),
    ("kv_evict", dict(new_lens=C.c_void_p(512)), INVALID),
    ("kv_evict", dict(ws_bytes=64), TOO_SMALL),
    ("kv_evict", dict(max_ctx=(1 << 24) + 1, w_stride=1 << 25, out_stride=1 << 25, stride=1 << 21), UNSUPPORTED),
    ("kv_evict", dict(batch=0, kv_pool=None), kv.KV_OK),
])
def test_refusals(name, changed, status):
    assert call(name, **changed) == status


def test_workspace_sizes():
    v = view()
    assert kv.paged_tree_attn_workspace_bytes(v, 0, 0, 0, 0) == 0
    assert kv.paged_tree_attn_workspace_bytes(v, 1, 4, 100, 4) > 0
    assert kv.paged_decode_attn_weights_workspace_bytes(v, 3, 1000) >= 3 * 32 * 1000 * 4
    assert kv.kv_evict_workspace_bytes(v, 3, 1001) >= 3 * 8 * 2 * 501 * 4


def test_binding_refuses_before_the_library():
    """Shapes, types and places of tensors are checked in Python."""
    v = view(8, 2, 64)
    pool, table, ctx = torch.zeros(4, 2 * 16 * 2 * 64, dtype=torch.bfloat16), torch.zeros(1, 4, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    q, k = torch.zeros(1, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    pos, freq, mask, per = torch.zeros(1, dtype=torch.int32), torch.ones(32), torch.ones(1, 1, dtype=torch.int64), torch.zeros(1, 2, 64)
    off = torch.tensor([0, 1], dtype=torch.int32)
    for f in (lambda: kv.kv_rope_append(pool, v, q, k, k, pos, freq, table, ctx),
              lambda: kv.paged_tree_attn(q, pool, table, ctx, off, mask, v, 1, 1),
              lambda: kv.kv_accept(pool, v, table, ctx, off, pos[None], pos),
              lambda: kv.paged_decode_attn_weights(q, pool, table, ctx, v, 1, per),
              lambda: kv.kv_evict(pool, v, table, ctx, ctx, per, per.int(), ctx, 64)):
        with pytest.raises((ValueError, RuntimeError), match="device|cuda|CUDA|HIP"):
            f()
    with pytest.raises(ValueError, match="one shape"):
        kv.kv_evict(pool, v, table, ctx, ctx, per, per.int()[:, :, 1:], ctx, 64)
    with pytest.raises(ValueError, match="one device"):
        kv.kv_accept(pool, v, table, ctx.to("meta"), off, pos[None], pos)


# ---- pins of the plain forms -------------------------------------------------------------------------

def test_chain_masks_give_causal_attention():
    c = ref.case((8, 2, 64, 16), (ref.DP, 1, 0), [40, 17, 9], [12, 17, 1])
    seen = np.zeros((30, 64), bool)
    for s in range(3):
        for j in range(int(c.q_lens[s])):
            seen[int(c.q_off[s]) + j, :j + 1] = True
    got, tol = ref.tree_attention(c, seen)
    assert np.abs(got - textbook_causal_attention(c, 1 / 8.0)).max() < 1e-12
    assert (tol > 0).all() and tol.max() < 0.1


def test_rotation_keeps_lengths_and_depends_on_distance():
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((2, 1, 1, 64))
    freq = (1e4 ** (-np.arange(32) / 32)).astype(np.float32)

    def turn(x, p, adjacent):
        return ref.rotated(x, np.array([[p]], np.int32), freq, [0] * 32, adjacent)[0]
    for adjacent in (False, True):
        assert np.allclose(np.linalg.norm(turn(q, 12345, adjacent)), np.linalg.norm(q))
        assert np.allclose((turn(q, 700, adjacent) * turn(k, 650, adjacent)).sum(), (turn(q, 50, adjacent) * turn(k, 0, adjacent)).sum())
    assert np.array_equal(turn(q, 0, False), q)


def test_evicted_rows_are_moved_and_kept():
    c = ref.case((8, 2, 64, 16), (ref.DP, 1, 0), [50], [0])
    rng = np.random.default_rng(4)
    w = rng.random((1, 2, 50)).astype(np.float32)
    pos = np.tile(np.arange(50, dtype=np.int32), (1, 2, 1))
    pool, w2, p2, lens = ref.evicted(c, c.pool, np.array([20]), w, pos, np.array([50]), 2, 5)
    assert lens.tolist() == [20]
    old, _ = ref.view_rows(c, c.pool)
    new, _ = ref.view_rows(c, pool)
    for h in range(2):
        stay = set(p2[0, h, :20].tolist())
        assert {0, 1, 45, 46, 47, 48, 49} <= stay and len(stay) == 20
        others = np.sort(w[0, h, 2:45])[::-1][:13]
        assert np.array_equal(np.sort(w2[0, h, :20])[-20:], np.sort(np.concatenate([others, w[0, h, [0, 1, 45, 46, 47, 48, 49]]])))
        for t in range(20):
            (b, slot), (ob, oslot) = ref.place(c, 0, t), ref.place(c, 0, int(p2[0, h, t]))
            assert np.array_equal(new[b, :, slot, h], old[ob, :, oslot, h])


def test_names_in_the_binding_match_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "flying_kv.h")).read()
    assert "KV_ROPE_HALVES = 0, KV_ROPE_ADJACENT = 1" in text
    assert (kv.KV_ROPE_HALVES, kv.KV_ROPE_ADJACENT) == (0, 1)
    assert np.isfinite(bf16_bits_to_f64(np.array([0x3F80], np.uint16))).all()


@pytest.mark.parametrize("geom,p", [((32, 8, 128, 16), 1), ((32, 8, 128, 16), 2), ((64, 8, 128, 16), 8), ((8, 2, 64, 16), 1), ((20, 4, 64, 32), 1)])
def test_workspaces_for_larger_bounds_serve_smaller_calls(geom, p):
    view = kv.kv_view_create(*geom, kv.KV_LAYOUT_TP if p > 1 else kv.KV_LAYOUT_DP, p, 0)
    bounds = [(b, n) for b in (1, 3, 16, 64, 200) for n in (32, 256, 1000, 8192, 8193, 131072)]
    tree = {(b, n, q): kv.paged_tree_attn_workspace_bytes(view, b, b * q, n, q) for b, n in bounds for q in (1, 8, 9, 16, 17, 32, 33, 64, 256) if q <= n}
    weights = {x: kv.paged_decode_attn_weights_workspace_bytes(view, *x) for x in bounds}
    evict = {x: kv.kv_evict_workspace_bytes(view, *x) for x in bounds}
    for sizes in (tree, weights, evict):
        for x, need in sizes.items():
            assert all(given >= need for y, given in sizes.items() if all(j >= i for i, j in zip(x, y))), x

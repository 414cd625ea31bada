"""CPU checks of what the operators around the cache refuse or promise about arrays that meet, addresses and sizes."""
import ctypes as C

import pytest

from paper_2602_22593_amd import binding as kv

from test_operators_host import FAKE, INVALID, built_library, call, view  # noqa: F401  (the fixture builds)


def at(x):
    return C.c_void_p(x)


@pytest.mark.parametrize("name,changed", [
    ("kv_accept", dict(n_accepted=at(512))),                    # workgroups still read what another one overwrites
    ("kv_accept", dict(q_off=at(512))),
    ("kv_accept", dict(q_off=at(504))),                         # its last entry
    ("kv_accept", dict(n_accepted=at(516))),
    ("kv_accept", dict(accepted=at(512))),
    ("kv_accept", dict(accepted=at(512 - 28))),
    ("kv_accept", dict(ctx=at(508))),
    ("kv_evict", dict(next_pos=at(768))),
    ("kv_evict", dict(next_pos=at(764))),
    ("kv_evict", dict(keep=at(772))),
    ("kv_evict", dict(ctx=at(764))),
])
def test_new_lengths_meet_no_input(name, changed):
    assert call(name, **changed) == INVALID


@pytest.mark.parametrize("name,changed", [
    *[("paged_tree_attn", {x: at(256 + by)}) for x, by in (("kv_pool", 8), ("q", 8), ("q", 2), ("out", 4))],
    *[("paged_decode_attn_weights", {x: at(256 + by)}) for x, by in (("kv_pool", 8), ("kv_pool", 2), ("q", 8), ("out", 4))],
    ("kv_accept", dict(kv_pool=at(264))),
    ("kv_evict", dict(kv_pool=at(258))),
])
def test_addresses_are_those_of_whole_pieces(name, changed):
    """Rows are moved 16 bytes at a time and output 8."""
    assert call(name, **changed) == kv.KV_ERR_UNSUPPORTED


@pytest.mark.parametrize("heads", [1, 2, 3, 4, 5, 6, 7, 10, 12, 14, 18, 20, 22, 24, 36, 40, 52, 100, 300, 1030])
@pytest.mark.parametrize("d", [64, 128])
def test_workspaces_of_any_number_of_heads_serve_smaller_calls(heads, d):
    """The variants cut the work into numbers of shares that round differently: a larger bound never asks for less."""
    v = kv.kv_view_create(4 * heads, heads, d, 16, kv.KV_LAYOUT_DP, 1, 0)
    bounds = [(b, n) for b in (1, 3, 64, 65, 200) for n in (64, 1000, 8192, 131072)]
    tree = {(b, n, q): kv.paged_tree_attn_workspace_bytes(v, b, b * q, n, q) for b, n in bounds for q in (1, 8, 9, 16, 17, 32, 33, 64) if q <= n}
    weights = {x: kv.paged_decode_attn_weights_workspace_bytes(v, *x) for x in bounds}
    evict = {x: kv.kv_evict_workspace_bytes(v, *x) for x in bounds}
    for sizes in (tree, weights, evict):
        for x, need in sizes.items():
            assert all(given >= need for y, given in sizes.items() if all(j >= i for i, j in zip(x, y))), x


@pytest.mark.parametrize("d,status", [(1024, kv.KV_ERR_UNSUPPORTED), (4096, kv.KV_ERR_UNSUPPORTED), (512, kv.KV_ERR_WORKSPACE)])
def test_evictions_that_32_bits_count(d, status):
    """A head's rows that move are numbered by their 16-byte pieces in 32 bits; what passes that is refused."""
    assert call("kv_evict", view=view(8, 8, d), max_ctx=1 << 24, w_stride=1 << 24, out_stride=1 << 24, stride=1 << 20, ws_bytes=64) == status


@pytest.mark.parametrize("changed,status", [
    *[({x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "acc_stride", "batch", "pos_stride", "w_stride")],
    *[({x: None}, INVALID) for x in ("kv_pool", "view", "block_table", "ctx", "q_off", "accepted", "n_accepted")],
    (dict(n_accepted=at(512)), INVALID),
    (dict(batch=0, kv_pool=None), kv.KV_OK),
])
def test_accept_tracked_refusals(changed, status):
    v = view()
    args = dict(kv_pool=FAKE, n_pool_blocks=10, view=v.handle, block_table=FAKE, stride=64, ctx=FAKE, q_off=FAKE, accepted=FAKE, acc_stride=4,
                n_accepted=FAKE, batch=2, new_lens=at(512), token_pos=FAKE, pos_stride=100, weights=FAKE, w_stride=100, st=None)
    assert set(changed) <= set(args)
    args.update(changed)
    assert kv.lib().kv_accept_tracked(*args.values()) == status


@pytest.mark.parametrize("changed,status", [
    *[({x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "total", "pos_stride", "w_stride")],
    *[({x: None}, INVALID) for x in ("kv_pool", "view", "q", "ctx")],
    (dict(batch=0, total=0, q=None), kv.KV_OK),
])
def test_rope_append_tracked_refusals(changed, status):
    v = view()
    args = dict(kv_pool=FAKE, n_pool_blocks=10, view=v.handle, q=FAKE, q_stride=6144, k=FAKE, k_stride=6144, v=FAKE, v_stride=6144, q_out=at(512),
                positions=FAKE, position_stride=9, n_axes=1, inv_freq=FAKE, rotary_dim=128, axes=None, pairs=0, table=FAKE, stride=64, ctx=FAKE,
                q_off=FAKE, batch=2, total=9, token_pos=FAKE, pos_stride=100, weights=FAKE, w_stride=100, st=None)
    assert set(changed) <= set(args)
    args.update(changed)
    assert kv.lib().kv_rope_append_tracked(*args.values()) == status

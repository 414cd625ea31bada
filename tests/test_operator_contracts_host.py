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

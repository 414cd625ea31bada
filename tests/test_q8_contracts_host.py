"""CPU checks of the operators on a cache held in 8 bits at sizes that the header allows and few models have: the host code of a call has to come to
its end.  Nothing here reaches a launch."""
import ctypes as C

import pytest

from paper_2602_22593_amd import binding as kv

FAKE = C.c_void_p(256)


@pytest.fixture(scope="module", autouse=True)
def built_library():
    from paper_2602_22593_amd.build import ensure_built
    ensure_built()


@pytest.mark.parametrize("heads,d,tp", [(32, 128, 1), (33, 128, 1), (40, 128, 1), (64, 128, 2), (80, 128, 2), (65, 64, 1), (144, 64, 1), (512, 16, 1),
                                        (1, 16, 1), (1, 8192, 1)])
def test_moves_of_any_number_of_heads_are_laid_out(heads, d, tp):
    """More than 4096 elements of a token move at once, and fewer: more sequences than a grid has are refused after the grid is worked out."""
    src = kv.kv_view_create(heads, heads, d, 16, kv.KV_LAYOUT_DP, 1, 0)
    dst = kv.kv_view_create(heads, heads, d, 16, kv.KV_LAYOUT_TP if tp > 1 else kv.KV_LAYOUT_DP, tp, tp - 1)
    for a, b in ((src, dst), (dst, src)):
        assert kv.lib().kv_repack_q8(FAKE, FAKE, 10, a.handle, b.handle, FAKE, 64, FAKE, 64, FAKE, 65536, 1024, None) == kv.KV_ERR_INVALID_ARG

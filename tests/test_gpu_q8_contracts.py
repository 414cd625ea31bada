"""What the header promises of the operators on a cache held in 8 bits, where a call is easily answered wrongly: scales that are
infinite, moves of many heads."""
import numpy as np
import pytest

import q8_refs as q8
from operator_refs import DP, TP, place
from q8_refs import E4M3, INT8

from helpers import bf16_bits_to_f64
from test_gpu_operators import G8B, host
from test_gpu_q8 import decode, prefill, q_for, test_repack as check_repack

pytestmark = pytest.mark.gpu
FORMATS = [E4M3, INT8]


def make_infinite(x, s, at, plane, head, sign):
    """The scale of token `at`'s group becomes infinite.  Queries are positive and the keys' codes of the group's tokens negative, or the other
    way round with the scale's sign: each product of a score is -inf, where nothing makes it a NaN."""
    x.c.q &= np.uint16(0x7fff)
    first = at // x.base * x.base
    row = x.c.info["row_head0"] + head
    b, slot = place(x.c, s, np.arange(first, min(first + x.base, int(x.c.ctx[s]))))
    codes = x.codes[b, 0, slot, row]
    if x.fmt == E4M3:
        codes = codes & 0x7f | (0x80 if sign > 0 else 0)
        codes[(codes & 0x7f) == 0] += 8
    else:
        v = np.maximum(np.abs(codes.view(np.int8).astype(np.int32)), 1)
        codes = (-sign * v).astype(np.int8).view(np.uint8)
    x.codes[b, 0, slot, row] = codes
    b, g = x.group_of(s, at)
    x.scales[b, plane, g, row] = sign * np.inf


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("plane", [0, 1])
@pytest.mark.parametrize("triple,ctx,at", [
    ((DP, 1, 0), [300, 40], 100),       # a workgroup a pair
    ((DP, 1, 0), [289, 40], 288),       # a last group of one token
    ((TP, 4, 1), [1, 40], 0),           # nothing else
    ((DP, 1, 0), [3000, 40], 100),      # cut, eight heads side by side
    ((DP, 1, 0), [2993, 40], 2992),
    ((TP, 8, 5), [2993, 40], 2992),     # cut, one head
])
def test_decode_with_an_infinite_scale(fmt, sign, plane, triple, ctx, at):
    """Query heads of that KV head and sequence become NaN, all others keep their results."""
    x = q8.case(G8B, triple, ctx, [1, 1], fmt)
    x.c.q = q_for(x, 2)
    head, G = x.c.info["n_kv_local"] - 1, 4
    make_infinite(x, 0, at, plane, head, sign)
    out = bf16_bits_to_f64(host(decode(x)))
    with np.errstate(invalid="ignore"):
        want, tol = q8.attention(x, causal=False)
    hit = np.zeros(out.shape, bool)
    hit[0, G * head:] = True
    assert np.isnan(out[hit]).all() and (np.abs(out - want) <= tol)[~hit].all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("plane", [0, 1])
@pytest.mark.parametrize("ctx,q_lens,back", [
    ([200, 100], [200, 100], 40),       # not cut
    ([193, 100], [193, 100], 1),        # a last group of one token
    ([1500, 200], [60, 200], 40),       # cut
    ([1505, 200], [60, 200], 1),
])
def test_prefill_rows_see_infinite_scales_of_their_groups_only(fmt, sign, plane, ctx, q_lens, back):
    """Rows before the group keep their results, those that see a token of it are NaN."""
    x = q8.case(G8B, (TP, 8, 0), ctx, q_lens, fmt)
    x.c.q &= np.uint16(0x7fff)
    want, tol = q8.attention(x, causal=True)
    at = ctx[0] - back
    make_infinite(x, 0, at, plane, 0, sign)
    out = bf16_bits_to_f64(host(prefill(x)))
    hit = np.zeros(len(out), bool)
    hit[:q_lens[0]] = ctx[0] - q_lens[0] + np.arange(q_lens[0]) >= at // 16 * 16
    assert np.isnan(out[hit]).all() and (np.abs(out - want) <= tol)[~hit].all()


# ---- kv_repack_q8 ------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("geom,src,dst,ctx", [
    ((40, 40, 128, 16), (DP, 1, 0), (DP, 1, 0), [33, 5, 0, 100]),      # runs of 5120 elements, no power of two
    ((80, 80, 128, 16), (DP, 1, 0), (TP, 2, 1), [17, 64]),
    ((80, 80, 128, 16), (TP, 2, 1), (DP, 1, 0), [17, 64]),
    ((64, 64, 128, 16), (TP, 2, 0), (DP, 2, 0), [40, 1]),              # 4096: one token's run is the whole payload
    ((144, 144, 64, 16), (DP, 1, 0), (DP, 1, 0), [50, 16]),            # more scales of a group than a workgroup has threads
    ((136, 136, 64, 48), (DP, 1, 0), (TP, 4, 3), [100, 47, 0]),
    ((288, 288, 64, 32), (TP, 2, 0), (DP, 1, 0), [33]),
])
def test_repack_of_many_heads(fmt, geom, src, dst, ctx):
    check_repack(fmt, geom, src, dst, ctx)

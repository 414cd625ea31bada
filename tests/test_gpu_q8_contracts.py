"""What the header promises of the operators on a cache held in 8 bits, where a call is easily answered wrongly: scales that are
infinite, moves of many heads, the largest groups and batches; results that repeat themselves."""
import numpy as np
import pytest
import torch

import q8_refs as q8
from operator_refs import DP, TP, place
from paper_2602_22593_amd import binding as kv
from q8_refs import E4M3, INT8

from helpers import bf16_bits_to_f64
from test_gpu_operators import DEV, G8B, G70B, dev, host, view_of, within
from test_gpu_q8 import decode, pool_of, prefill, q_for
from test_gpu_q8 import test_append_one_token as check_append_one, test_append_several_tokens as check_append_several
from test_gpu_q8 import test_repack as check_repack

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


# ---- kv_rope_append_q8 -------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FORMATS)
def test_append_of_the_longest_groups_with_all_dims_turned(fmt):
    """Sines of 128 tokens and 64 pairs: all of the 64 KiB that a workgroup may have of LDS by default."""
    check_append_several(fmt, (4, 2, 128, 128), (DP, 1, 0), [300, 128, 129], [290, 1, 128], 1, False, 128)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_one_token_of_many_sequences(fmt):
    """From 512 on a sequence has one workgroup, which takes all of its rows."""
    check_append_one(fmt, G8B, (DP, 1, 0), [33 + i % 40 for i in range(530)], [1] * 530, 1, False, 128)


def test_append_several_tokens_of_thousands_of_sequences():
    """A group's sequence is found among 4200 in three steps."""
    check_append_several(E4M3, (2, 1, 64, 16), (DP, 1, 0), [3 + i % 31 for i in range(4200)], [i % 4 for i in range(4200)], 1, False, 64)


@pytest.mark.parametrize("one", [True, False])
def test_append_turns_queries_in_place(one):
    """The queries' own array as output, tokens that lie together: the bits that another array gets."""
    q_lens = [1, 1, 1] if one else [5, 40, 0]
    x = q8.case(G8B, (TP, 2, 1), [40, 90, 7], q_lens, E4M3)
    total, view = sum(q_lens), view_of(x.c)
    rows = dev(q8.normal_rows(total, 16, 4, 128, 131))
    q, k, v = (part.contiguous() for part in (rows[:, :16], rows[:, 16:20], rows[:, 20:]))
    positions, freq = dev(np.arange(total, dtype=np.int32) * 77), dev((1e4 ** (-np.arange(64) / 64)).astype(np.float32))
    off = None if one else dev(x.c.q_off.astype(np.int32))
    got = []
    for out in (torch.empty_like(q), q):
        pool, scales = pool_of(x)
        assert kv.kv_rope_append_q8(pool, scales, view, q, k, v, positions, freq, dev(x.c.table), dev(x.c.ctx), off, out=out) is out
        got.append(host(out))
    assert np.array_equal(got[0], got[1])


# ---- paged_prefill_attn_q8 ---------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("triple,ctx,q_lens", [
    ((DP, 1, 0), [300, 64], [20, 64]),                          # one workgroup a tile
    ((TP, 8, 3), [1200, 16, 130], [16, 16, 7]),                 # cut
    ((TP, 4, 0), [700] * 9, [200] * 9),                         # in the order of their lengths
])
def test_prefill_leaves_rows_behind_the_last_sequence(fmt, triple, ctx, q_lens):
    x = q8.case(G8B, triple, ctx, q_lens, fmt)
    c, pad = x.c, 300
    pool, scales = pool_of(x)
    q = torch.cat([dev(c.q), torch.full((pad,) + c.q.shape[1:], float("nan"), dtype=torch.bfloat16, device=DEV)])
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    kv.paged_prefill_attn_q8(q, pool, scales, dev(c.table), dev(c.ctx), dev(c.q_off.astype(np.int32)), view_of(c), max(ctx), max(q_lens), out=out)
    assert (out[-pad:] == 7.0).all()
    within(host(out[:-pad]), *q8.attention(x, causal=True))


# ---- every call again --------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("geom,triple,ctx,q_lens", [
    (G8B, (DP, 1, 0), [300, 17, 0, 64], [9, 17, 0, 1]),             # neither is cut
    (G8B, (TP, 4, 1), [5000, 2600, 33], [40, 3, 33]),               # both are
    (G70B, (TP, 8, 2), [2500] + [40] * 30, [16] + [5] * 30),
])
def test_attention_repeats_itself(fmt, geom, triple, ctx, q_lens):
    """Nothing depends on the order in which workgroups come to their ends, or on what a workspace held."""
    x = q8.case(geom, triple, ctx, q_lens, fmt)
    pool, scales = pool_of(x)
    several = [prefill(x, pool, scales).view(torch.int16).clone() for _ in range(4)]
    x.c.q = q_for(x, len(ctx))
    one = [decode(x, pool, scales).view(torch.int16).clone() for _ in range(4)]
    for got in (several, one):
        assert all(torch.equal(g, got[0]) for g in got[1:])

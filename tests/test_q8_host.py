"""CPU checks of the operators on a cache held in 8 bits: what the entry points refuse, before anything is launched, workspace sizes,
and pins of the plain forms that the GPU tests compare with."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import operator_refs as ref
import q8_refs as q8
from paper_2602_22593_amd import binding as kv

FAKE = C.c_void_p(256)
INVALID, UNSUPPORTED, TOO_SMALL, OK = kv.KV_ERR_INVALID_ARG, kv.KV_ERR_UNSUPPORTED, kv.KV_ERR_WORKSPACE, kv.KV_OK


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
    other = changed.pop("dst_view", view(layout=kv.KV_LAYOUT_TP, p=2))
    common = dict(kv_pool=FAKE, scales=FAKE, format=0, n_pool_blocks=10, view=getattr(v, "handle", v), block_table=FAKE, stride=64, ctx=FAKE,
                  batch=2, st=None)
    args = {
        "kv_rope_append_q8": dict(kv_pool=0, scales=0, format=0, n_pool_blocks=0, view=0, q=FAKE, q_stride=6144, k=FAKE, k_stride=6144, v=FAKE,
                                  v_stride=6144, q_out=C.c_void_p(512), positions=FAKE, position_stride=9, n_axes=2, inv_freq=FAKE,
                                  rotary_dim=128, axes=(C.c_int32 * 64)(), pairs=0, block_table=0, stride=0, ctx=0, q_off=FAKE, batch=0,
                                  total=9, st=0),
        "paged_decode_attn_q8": dict(q=FAKE, out=FAKE, kv_pool=0, scales=0, format=0, n_pool_blocks=0, block_table=0, stride=0, ctx=0, batch=0,
                                     max_ctx=1024, view=0, scale=0.0, ws=FAKE, ws_bytes=1 << 40, st=0),
        "paged_prefill_attn_q8": dict(q=FAKE, out=FAKE, kv_pool=0, scales=0, format=0, n_pool_blocks=0, block_table=0, stride=0, ctx=0,
                                      q_off=FAKE, batch=0, total=9, max_ctx=1024, max_q=64, view=0, scale=0.0, ws=FAKE, ws_bytes=1 << 40, st=0),
        "kv_repack_q8": dict(kv_pool=0, scales=0, n_pool_blocks=0, view=0, dst_view=getattr(other, "handle", other), block_table=0, stride=0,
                             dst_table=FAKE, dst_stride=32, n_tokens=FAKE, batch=0, max_tokens=1024, st=0),
    }[name]
    args.update({k: x for k, x in common.items() if k in args})
    assert set(changed) <= set(args), changed
    args.update(changed)
    return getattr(kv.lib(), name)(*args.values())


@pytest.mark.parametrize("name,changed,status", [
    *[("kv_rope_append_q8", {x: None}, INVALID) for x in ("kv_pool", "scales", "view", "q", "k", "v", "q_out", "positions", "inv_freq",
                                                          "block_table", "ctx")],
    *[("kv_rope_append_q8", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "total", "rotary_dim", "position_stride", "format")],
    ("kv_rope_append_q8", dict(format=2), INVALID),
    ("kv_rope_append_q8", dict(q_stride=4095), INVALID),
    ("kv_rope_append_q8", dict(k_stride=1023), INVALID),
    ("kv_rope_append_q8", dict(v_stride=1016), INVALID),
    ("kv_rope_append_q8", dict(q_out=FAKE), INVALID),                 # in place needs contiguous tokens
    ("kv_rope_append_q8", dict(position_stride=8), INVALID),
    ("kv_rope_append_q8", dict(axes=(C.c_int32 * 64)(*[2] * 64)), INVALID),
    ("kv_rope_append_q8", dict(pairs=2), INVALID),
    ("kv_rope_append_q8", dict(n_axes=0), INVALID),
    ("kv_rope_append_q8", dict(rotary_dim=130), INVALID),
    ("kv_rope_append_q8", dict(q_off=None), INVALID),                 # nine tokens of two sequences
    ("kv_rope_append_q8", dict(rotary_dim=24), UNSUPPORTED),
    ("kv_rope_append_q8", dict(q_stride=6148), UNSUPPORTED),
    ("kv_rope_append_q8", dict(k=C.c_void_p(264)), UNSUPPORTED),
    ("kv_rope_append_q8", dict(kv_pool=C.c_void_p(264)), UNSUPPORTED),
    ("kv_rope_append_q8", dict(scales=C.c_void_p(258)), UNSUPPORTED),
    ("kv_rope_append_q8", dict(n_axes=5), UNSUPPORTED),
    ("kv_rope_append_q8", dict(view=view(d=96), rotary_dim=64), UNSUPPORTED),
    ("kv_rope_append_q8", dict(view=view(bs=24), stride=4096), UNSUPPORTED),
    ("kv_rope_append_q8", dict(view=view(bs=144), stride=4096), UNSUPPORTED),
    ("kv_rope_append_q8", dict(batch=0, total=0, q=None, q_out=None), OK),
    *[("paged_decode_attn_q8", {x: None}, INVALID) for x in ("q", "out", "kv_pool", "scales", "block_table", "ctx", "view", "ws")],
    *[("paged_decode_attn_q8", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "max_ctx", "format")],
    ("paged_decode_attn_q8", dict(format=2), INVALID),
    ("paged_decode_attn_q8", dict(stride=63), INVALID),
    ("paged_decode_attn_q8", dict(ws=C.c_void_p(264)), INVALID),
    ("paged_decode_attn_q8", dict(ws_bytes=1024), TOO_SMALL),
    ("paged_decode_attn_q8", dict(view=view(d=96)), UNSUPPORTED),
    ("paged_decode_attn_q8", dict(view=view(hq=8 * 17)), UNSUPPORTED),
    ("paged_decode_attn_q8", dict(view=view(bs=24), stride=4096), UNSUPPORTED),
    ("paged_decode_attn_q8", dict(view=view(bs=8, layout=kv.KV_LAYOUT_TP, p=2), stride=4096), UNSUPPORTED),   # groups of 8 tokens
    ("paged_decode_attn_q8", dict(q=C.c_void_p(264)), UNSUPPORTED),
    ("paged_decode_attn_q8", dict(kv_pool=C.c_void_p(264)), UNSUPPORTED),
    ("paged_decode_attn_q8", dict(batch=0, q=None), OK),
    *[("paged_prefill_attn_q8", {x: None}, INVALID) for x in ("q", "out", "kv_pool", "scales", "block_table", "ctx", "q_off", "view")],
    *[("paged_prefill_attn_q8", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "batch", "total", "max_ctx", "max_q", "format")],
    ("paged_prefill_attn_q8", dict(format=2), INVALID),
    ("paged_prefill_attn_q8", dict(max_ctx=32), INVALID),             # more new tokens than cached ones
    ("paged_prefill_attn_q8", dict(stride=63), INVALID),
    ("paged_prefill_attn_q8", dict(view=view(d=64)), UNSUPPORTED),
    ("paged_prefill_attn_q8", dict(view=view(hq=8 * 17)), UNSUPPORTED),
    ("paged_prefill_attn_q8", dict(view=view(bs=8, layout=kv.KV_LAYOUT_TP, p=2), stride=4096), UNSUPPORTED),
    ("paged_prefill_attn_q8", dict(out=C.c_void_p(264)), UNSUPPORTED),
    ("paged_prefill_attn_q8", dict(scales=C.c_void_p(258)), UNSUPPORTED),
    ("paged_prefill_attn_q8", dict(batch=0, q=None), OK),
    ("paged_prefill_attn_q8", dict(total=0, q=None), OK),
    *[("kv_repack_q8", {x: None}, INVALID) for x in ("kv_pool", "scales", "view", "dst_view", "block_table", "dst_table", "n_tokens")],
    *[("kv_repack_q8", {x: -1}, INVALID) for x in ("n_pool_blocks", "stride", "dst_stride", "batch", "max_tokens")],
    ("kv_repack_q8", dict(dst_stride=31), INVALID),
    ("kv_repack_q8", dict(dst_view=view(hkv=4, hq=32)), INVALID),
    ("kv_repack_q8", dict(view=view(d=72), dst_view=view(d=72, layout=kv.KV_LAYOUT_TP, p=2)), UNSUPPORTED),
    ("kv_repack_q8", dict(kv_pool=C.c_void_p(264)), UNSUPPORTED),
    ("kv_repack_q8", dict(view=view(bs=24), dst_view=view(bs=24, layout=kv.KV_LAYOUT_TP, p=2), stride=4096, dst_stride=4096), UNSUPPORTED),
    ("kv_repack_q8", dict(view=view(layout=kv.KV_LAYOUT_TP, p=2, r=1)), OK),   # no head in common
    ("kv_repack_q8", dict(batch=0, kv_pool=None), OK),
])
def test_refusals(name, changed, status):
    assert call(name, **changed) == status


def test_binding_refuses_before_the_library():
    v = view(8, 2, 64)
    pool, scales = torch.zeros(4, 2 * 16 * 2 * 64, dtype=torch.int8), torch.zeros(4, 2, 2)
    table, ctx, off = torch.zeros(1, 4, dtype=torch.int32), torch.ones(1, dtype=torch.int32), torch.tensor([0, 1], dtype=torch.int32)
    q, k = torch.zeros(1, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    for f in (lambda: kv.kv_rope_append_q8(pool, scales, v, None, k, k, None, None, table, ctx),
              lambda: kv.paged_decode_attn_q8(q, pool, scales, table, ctx, v, 1),
              lambda: kv.paged_prefill_attn_q8(q, pool, scales, table, ctx, off, v, 1, 1),
              lambda: kv.kv_repack_q8(pool, scales, v, v, table, table, ctx, 1)):
        with pytest.raises((ValueError, RuntimeError), match="device|cuda|CUDA|HIP"):
            f()
    with pytest.raises(ValueError, match="one device"):
        kv.paged_decode_attn_q8(q, pool, scales.to("meta"), table, ctx, v, 1)
    with pytest.raises(ValueError, match="without q"):
        kv.kv_rope_append_q8(pool, scales, v, None, k, k, None, None, table, ctx, out=q)
    with pytest.raises(ValueError, match="without positions"):
        kv.kv_rope_append_q8(pool, scales, v, None, k, k, None, torch.ones(32), table, ctx)


@pytest.mark.parametrize("geom,p", [((32, 8, 128, 16), 1), ((32, 8, 128, 16), 2), ((32, 8, 128, 16), 4), ((64, 8, 128, 16), 8), ((8, 2, 64, 16), 1),
                                    ((20, 4, 64, 32), 1), ((12, 6, 128, 16), 1)])
def test_workspaces_for_larger_bounds_serve_smaller_calls(geom, p):
    v = kv.kv_view_create(*geom, kv.KV_LAYOUT_TP if p > 1 else kv.KV_LAYOUT_DP, p, 0)
    sizes = {(b, n): kv.paged_decode_attn_q8_workspace_bytes(v, b, n)
             for b in (0, 1, 3, 16, 64, 200, 1000) for n in (0, 32, 256, 512, 513, 1000, 8192, 8193, 131072)}
    for x, need in sizes.items():
        assert all(given >= need for y, given in sizes.items() if all(j >= i for i, j in zip(x, y))), x
        assert (need == 0) == (x[0] == 0 or x[1] <= 256)   # (no pair is cut up to there, whatever the batch)


def test_names_in_the_binding_match_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "flying_kv.h")).read()
    assert "KV_Q8_E4M3 = 0, KV_Q8_INT8 = 1" in text
    assert (kv.KV_Q8_E4M3, kv.KV_Q8_INT8) == (0, 1)


# ---- pins of the plain forms -------------------------------------------------------------------------

def test_e4m3_values_and_rounding_against_torch():
    b = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(b).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(q8.VALUES[q8.E4M3], want, equal_nan=True)
    y = np.concatenate([np.random.default_rng(1).standard_normal(5000) * s for s in (300, 10, 0.05, 0.003)])
    y = np.clip(np.concatenate([y, [0.0, -0.0, 448, -448, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0]]), -448, 448)
    # (through fp32, which holds these exactly or far more finely than the codes)
    got, cast = q8.nearest(y.astype(np.float32).astype(np.float64), q8.E4M3), torch.from_numpy(y).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, cast)
    assert np.array_equal(q8.values(q8.codes_of(got, q8.E4M3), q8.E4M3), got)


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.INT8])
def test_scales_are_the_least_that_hold(fmt):
    top = np.concatenate([[0.0, q8.LARGEST[fmt], 3.5, 1.984375, 1.75, 2.0 ** -140], np.abs(np.random.default_rng(2).standard_normal(1000))])
    s = q8.scale_for(top, fmt)
    assert (top <= s * q8.LARGEST[fmt]).all() and (np.frexp(s)[0] == 0.5).all()
    assert ((top > s / 2 * q8.LARGEST[fmt]) | (s == q8.LEAST_SCALE)).all()


@pytest.mark.parametrize("fmt", [q8.E4M3, q8.INT8])
def test_appended_rows_are_near_and_older_ones_stay_near(fmt):
    x = q8.case((8, 2, 64, 16), (ref.DP, 1, 0), [21, 40], [5, 40], fmt)
    rows = np.random.default_rng(3).standard_normal((45, 2, 2, 64)) * 3
    before = x.cached(0)[0][:16]
    numbers, scales = q8.appended(x, rows, [5, 40])
    after = q8.Q8Case(x.c, fmt, q8.codes_of(np.where(np.isnan(numbers), 0, numbers), fmt), scales)
    for p in (0, 1):
        assert np.array_equal(after.cached(0)[p][:16], q8.Q8Case(x.c, fmt, x.codes, x.scales).cached(0)[p][:16])
        got = np.concatenate([after.cached(0)[p][16:], after.cached(1)[p]])
        top = np.abs(rows[:, p]).max()
        assert np.abs(got - rows[:, p]).max() <= top * (2.0 ** -4 if fmt == q8.E4M3 else 2 / 127 / 2)
    assert np.array_equal(before, after.cached(0)[0][:16])


def test_attention_of_a_single_token_is_its_value():
    x = q8.case((8, 2, 64, 16), (ref.DP, 1, 0), [1, 300], [1, 1], q8.INT8)
    out, tol = q8.attention(x, causal=False)
    assert np.allclose(out[0], np.repeat(x.cached(0)[1][0], 4, axis=0), rtol=0, atol=1e-12)
    assert np.allclose(out, q8.attention(x, causal=True)[0]) and (tol > 0).all() and tol.max() < 0.1

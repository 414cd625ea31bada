"""The calls on an 8-bit cache that csrc/binding_calls.c marshals answer as the Python code they stand in for."""
import pytest
import torch

from paper_2602_22593_amd import binding as kv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ("append", "keys", "decode", "prefill", "repack")


class _Nothing:
    """Answers every call with None: the Python code marshals it."""

    def __getattr__(self, name):
        return lambda *a: None


class _Counting:
    def __init__(self, m):
        self.m, self.made = m, 0

    def __getattr__(self, name):
        def call(*a):
            rc = getattr(self.m, name)(*a)
            self.made += rc is not None
            return rc
        return call


def _bf(*shape):
    g = torch.Generator(device=DEV).manual_seed(sum(shape))
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _calls(bad):
    """name -> call; `bad` swaps one argument of each for something (name -> value)."""
    view = kv.kv_view_create(8, 2, 128, 16, kv.KV_LAYOUT_DP)
    tp = kv.kv_view_create(8, 2, 128, 16, kv.KV_LAYOUT_TP, 2, 1)
    g = torch.Generator(device=DEV).manual_seed(5)
    codes = torch.randint(-100, 101, (16, 2 * 16 * 2 * 128), dtype=torch.int8, device=DEV, generator=g)
    a = dict(pool=codes, scales=torch.full((16, 2, 2), 2.0 ** -6, device=DEV), table=_i32(1, 2, 3, 4).view(2, 2), lens=_i32(20, 9),
             q=_bf(2, 8, 128), k=_bf(2, 2, 128), v=_bf(2, 2, 128), out=torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=DEV),
             q_off=_i32(0, 1, 2), pos=_i32(19, 8), freq=torch.ones(64, device=DEV), axes=None, pairs=kv.KV_ROPE_HALVES, max=32,
             ws=torch.zeros(1 << 24, dtype=torch.uint8, device=DEV), dst=_i32(8, 9).view(2, 1), scale=0.0, stream=None)
    a.update(bad)
    return a, {
        "append": lambda: kv.kv_rope_append_q8(a["pool"], a["scales"], view, a["q"], a["k"], a["v"], a["pos"], a["freq"], a["table"],
                                               a["lens"], a["q_off"], a["axes"], a["pairs"], out=a["out"], stream=a["stream"]),
        "keys": lambda: kv.kv_rope_append_q8(a["pool"], a["scales"], view, None, a["k"], a["v"], None, None, a["table"], a["lens"],
                                             stream=a["stream"]),
        "decode": lambda: kv.paged_decode_attn_q8(a["q"], a["pool"], a["scales"], a["table"], a["lens"], view, a["max"], out=a["out"],
                                                  scale=a["scale"], workspace=a["ws"], stream=a["stream"]),
        "prefill": lambda: kv.paged_prefill_attn_q8(a["q"], a["pool"], a["scales"], a["table"], a["lens"], a["q_off"], view, a["max"], 1,
                                                    out=a["out"], scale=a["scale"], workspace=a["ws"], stream=a["stream"]),
        "repack": lambda: kv.kv_repack_q8(a["pool"], a["scales"], view, tp, a["table"], a["dst"], a["lens"], a["max"], stream=a["stream"]),
    }


def _outcome(name, bad, module):
    a, calls = _calls(bad)
    was, kv._calls_module = kv._calls_module, module
    torch.cuda.synchronize()   # (the call may be on a stream of its own)
    try:
        calls[name]()
    except Exception as e:   # noqa: BLE001 (the same one is wanted from both)
        return type(e), str(e)
    finally:
        kv._calls_module = was
    torch.cuda.synchronize()
    return [a[k].view(torch.uint8).cpu() for k in ("out", "pool", "scales") if isinstance(a[k], torch.Tensor) and a[k].is_cuda]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("stream", [False, True])
@pytest.mark.parametrize("what", ["int8", "e4m3", "parameter", "axes", "plain", "own"])
def test_calls_in_c(name, stream, what):
    """Either format, several axes of positions, nothing rotated, buffers given or the binding's: the same bytes as through Python."""
    def bad():
        b = {"stream": torch.cuda.Stream()} if stream else {}
        if what in ("e4m3", "parameter"):
            b["pool"] = _calls({})[0]["pool"].bitwise_and(0x5f).view(torch.float8_e4m3fn)
        if what == "parameter":
            b["scales"] = torch.nn.Parameter(torch.full((16, 2, 2), 2.0 ** -6, device=DEV), requires_grad=False)
        if what == "axes":
            b.update(pos=_i32(19, 8, 3, 4, 5, 6).view(3, 2), axes=[i % 3 for i in range(64)], pairs=kv.KV_ROPE_ADJACENT)
        if what == "plain":
            b.update(pos=None, freq=None)
        if what == "own":
            b.update(ws=None, out=None)
        return b

    count = _Counting(kv._calls())
    got, want = _outcome(name, bad(), count), _outcome(name, bad(), _Nothing())
    assert isinstance(got, list), got
    assert len(got) == len(want) and all(torch.equal(g, w) for g, w in zip(got, want))
    assert count.made == (0 if what == "own" and name in ("decode", "prefill") else 1)


# What each call takes of the arguments below
TAKES = {"append": ("pool", "scales", "q", "k", "v", "out", "pos", "freq", "axes", "table", "lens", "q_off"),
         "keys": ("pool", "scales", "k", "v", "table", "lens"),
         "decode": ("pool", "scales", "q", "out", "table", "lens", "ws", "scale"),
         "prefill": ("pool", "scales", "q", "out", "table", "lens", "q_off", "ws", "scale"),
         "repack": ("pool", "scales", "table", "dst", "lens")}
# Swaps that are no reason to refuse
TAKEN = {("decode", "scale", 1), ("prefill", "scale", 1), ("append", "axes", (0,) * 64), ("decode", "ws", "small"),
         ("prefill", "ws", "small")}


@pytest.mark.parametrize("name,arg,what", [(n, arg, what) for arg, what in [
    ("pool", "ragged"), ("pool", "bf16"), ("pool", "host"), ("pool", "strided"), ("scales", "short"), ("scales", "half"), ("scales", "host"),
    ("q", "host"), ("q", "half"), ("q", "rows"), ("q", "strided"), ("out", "strided"), ("out", "rows"), ("k", "rows"), ("v", "half"),
    ("pos", "long"), ("pos", "short"), ("freq", "half"), ("freq", "long"), ("axes", (0,) * 63), ("axes", (0,) * 64), ("axes", (7,) * 64),
    ("table", "long"), ("table", "flat"), ("lens", "short"), ("q_off", "short"), ("ws", "small"), ("ws", "half"), ("dst", "long"),
    ("dst", "flat"), ("scale", 1), ("scale", "text"),
] for n, takes in TAKES.items() if arg in takes])
def test_refusals_are_the_same(name, arg, what):
    """Arguments that the binding or the library refuses, or that only Python takes: the same error, or the same bytes."""
    make = {"host": lambda t: t.cpu(), "half": lambda t: t.half() if t.dtype != torch.uint8 else t.view(torch.float16),
            "long": lambda t: t.long(), "rows": lambda t: t[:1], "short": lambda t: t[:1], "flat": lambda t: t.flatten(),
            "strided": lambda t: torch.zeros(t.shape + (2,), dtype=t.dtype, device=DEV)[..., 0],
            "ragged": lambda t: t.flatten()[:-5000].contiguous(), "bf16": lambda t: t.view(torch.bfloat16), "small": lambda t: t[:256],
            "text": lambda t: "much"}
    base, _ = _calls({})
    outcomes = [_outcome(name, {arg: make[what](base[arg].clone() if isinstance(base[arg], torch.Tensor) else base[arg])
                                if isinstance(what, str) else what}, module) for module in (kv._calls(), _Nothing())]
    got, want = outcomes
    assert isinstance(want, tuple) == ((name, arg, what) not in TAKEN), want
    if isinstance(want, tuple):
        assert got == want
    else:
        assert all(torch.equal(g, w) for g, w in zip(got, want))

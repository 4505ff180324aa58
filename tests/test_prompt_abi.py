"""The prompt pass's C ABI on the CPU: every host-detectable error returns its
code before a launch.  The pointers are made up; a call whose arguments are in
order is stopped by a misaligned one, which is checked last."""
import ctypes

import pytest

from paper_2607_16673_amd import binding as B

GIB = 1 << 30
NAMES = {"prefill": "state q k v alpha beta start out state_out ws status".split(),
         "conv": "state x weight bias start y state_out status".split(),
         "inputs": "q k a b a_log dt_bias q_out k_out alpha beta".split(),
         "norm": "x z weight y".split()}
OPTIONAL = {"prefill": {"state", "status"}, "conv": {"state", "bias", "status"}, "inputs": {"dt_bias"}, "norm": {"weight"}}
WRITES = {"prefill": "out state_out ws status".split(), "conv": "y state_out status".split(),
          "inputs": "q_out k_out alpha beta".split(), "norm": ["y"]}
SHAPES = {"prefill": (B.SlaPrefillShape, dict(tokens=1000, batch=3, heads=8, k_heads=4, d_k=128, d_v=64,
                                              qkv_dtype=B.SLA_DTYPE_BF16, family=B.SLA_FAMILY_GDN)),
          "conv": (B.SlaConvPrefillShape, dict(tokens=1000, batch=3, channels=1024, kernel_size=4,
                                               x_dtype=B.SLA_DTYPE_BF16, activation=B.SLA_ACT_SILU)),
          "inputs": (B.SlaInputsShape, dict(rows=1000, heads=8, k_heads=4, repeat=2, d_k=128, dtype=B.SLA_DTYPE_BF16,
                                            q_scale=0.1, eps=1e-6)),
          "norm": (B.SlaNormShape, dict(rows=1000, heads=8, d_v=64, x_dtype=B.SLA_DTYPE_F32, dtype=B.SLA_DTYPE_BF16,
                                        gate=B.SLA_GATE_SILU, eps=1e-6))}
ROW = {"prefill": ("tokens", "q k v alpha beta out".split()), "conv": ("tokens", "x y".split()),
       "inputs": ("rows", "q k a b q_out k_out alpha beta a_log".split()), "norm": ("rows", "x z y".split())}


def shape(name, **o):
    cls, f = SHAPES[name]
    return cls(**{**f, **o})


def call(name, s=None, *, strides=None, ws_bytes=None, null_shape=False, **at):
    """The call with made-up buffers 64 GiB apart; `at` moves or drops some."""
    s = shape(name) if s is None else s
    ref = None if null_shape else ctypes.byref(s)
    p = {k: (i + 1) * 64 * GIB for i, k in enumerate(NAMES[name])}
    p.update(at)
    L = B.lib()
    if name == "prefill":
        n = L.sla_prefill_workspace_bytes(ref) if ws_bytes is None and ref is not None else ws_bytes or 0
        q, k, v = strides or (4 * 128, 4 * 128, 8 * 64)
        return L.sla_prefill(ref, p["state"], p["q"], q, p["k"], k, p["v"], v, p["alpha"], p["beta"], p["start"], p["out"],
                             p["state_out"], p["ws"], n, p["status"], None)
    if name == "conv":
        return L.sla_conv_prefill(ref, p["state"], p["x"], (strides or (1024,))[0], p["weight"], p["bias"], p["start"], p["y"],
                                  p["state_out"], p["status"], None)
    if name == "inputs":
        q, k, a, b = strides or (4 * 128, 4 * 128, 8, 8)
        return L.sla_recurrent_inputs(ref, p["q"], q, p["k"], k, p["a"], a, p["b"], b, p["a_log"], p["dt_bias"], p["q_out"],
                                      p["k_out"], p["alpha"], p["beta"], None)
    return L.sla_gated_norm(ref, p["x"], p["z"], (strides or (8 * 64,))[0], p["weight"], p["y"], None)


def odd(name):
    """An output that is no multiple of 16 bytes: where a call that is otherwise in order ends."""
    key = {"prefill": "out", "conv": "y", "inputs": "q_out", "norm": "y"}[name]
    return {key: 64 * GIB * (NAMES[name].index(key) + 1) + 4}


@pytest.mark.parametrize("name", list(NAMES))
def test_in_order_until_the_misaligned_output(name):
    assert call(name, **odd(name)) == B.SLA_ERR_UNSUPPORTED
    for field in OPTIONAL[name]:
        assert call(name, **{**odd(name), field: None}) == B.SLA_ERR_UNSUPPORTED


@pytest.mark.parametrize("name", list(NAMES))
def test_nulls(name):
    assert call(name, null_shape=True) == B.SLA_ERR_NULL
    for field in set(NAMES[name]) - OPTIONAL[name]:
        if name == "inputs" and field in ("alpha", "beta", "a", "b", "a_log"):
            continue
        assert call(name, **{field: None}) == B.SLA_ERR_NULL, field


def test_nulls_of_what_a_family_or_a_gate_reads():
    o = odd("prefill")
    assert call("prefill", shape("prefill", family=B.SLA_FAMILY_DELTANET), **o, alpha=None) == B.SLA_ERR_UNSUPPORTED
    assert call("prefill", shape("prefill", family=B.SLA_FAMILY_DELTANET), **o, beta=None) == B.SLA_ERR_NULL
    assert call("prefill", shape("prefill", family=B.SLA_FAMILY_DECAY), **o, beta=None) == B.SLA_ERR_UNSUPPORTED
    assert call("prefill", shape("prefill", family=B.SLA_FAMILY_DECAY), **o, alpha=None) == B.SLA_ERR_NULL
    for lost in (dict(a=None), dict(a_log=None), dict(alpha=None), dict(b=None), dict(beta=None)):
        assert call("inputs", **lost) == B.SLA_ERR_NULL, lost
    o = odd("inputs")
    for gone in (dict(a=None, alpha=None), dict(a=None, alpha=None, a_log=None), dict(b=None, beta=None)):
        assert call("inputs", **o, **gone) == B.SLA_ERR_UNSUPPORTED
    assert call("norm", shape("norm", gate=B.SLA_GATE_NONE), **odd("norm"), z=None) == B.SLA_ERR_UNSUPPORTED
    assert call("conv", shape("conv", kernel_size=1), **odd("conv"), state_out=None) == B.SLA_ERR_UNSUPPORTED


@pytest.mark.parametrize("name", list(NAMES))
def test_no_rows_need_no_pointers_to_rows(name):
    count, rows = ROW[name]
    s = shape(name, **{count: 0})
    gone = {k: None for k in rows}
    if name in ("inputs", "norm"):  # nothing to do
        assert call(name, s, **gone) == B.SLA_OK
    else:  # states are passed on: a misaligned one is told
        assert call(name, s, **gone, state_out=64 * GIB * 20 + 4) == B.SLA_ERR_UNSUPPORTED


BAD = {"prefill": [(dict(tokens=-1), "SHAPE"), (dict(tokens=(1 << 30) + 1), "SHAPE"), (dict(batch=0), "SHAPE"),
                   (dict(batch=65536), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(heads=7), "SHAPE"), (dict(k_heads=0), "SHAPE"),
                   (dict(heads=1 << 17, k_heads=1), "SHAPE"), (dict(d_v=8), "SHAPE"), (dict(d_v=72), "SHAPE"),
                   (dict(d_v=1040), "SHAPE"), (dict(d_k=0), "SHAPE"), (dict(d_k=96), "UNSUPPORTED"), (dict(qkv_dtype=2), "DTYPE"),
                   (dict(family=-1), "SHAPE"), (dict(family=4), "SHAPE"), (dict(family=B.SLA_FAMILY_GLA), "UNSUPPORTED"),
                   (dict(heads=1 << 16, k_heads=1, d_v=1024), "SHAPE"), (dict(tokens=1 << 30, heads=4096), "SHAPE"),
                   (dict(batch=65535, heads=4096, d_v=1024), "SHAPE")],
       "conv": [(dict(tokens=-5), "SHAPE"), (dict(tokens=(1 << 30) + 1), "SHAPE"), (dict(batch=0), "SHAPE"),
                (dict(batch=65536), "SHAPE"), (dict(channels=0), "SHAPE"), (dict(channels=12), "SHAPE"),
                (dict(channels=(1 << 20) + 8), "SHAPE"), (dict(kernel_size=0), "SHAPE"), (dict(kernel_size=5), "SHAPE"),
                (dict(x_dtype=-1), "DTYPE"), (dict(activation=2), "SHAPE"), (dict(tokens=1 << 30, channels=1 << 20), "SHAPE")],
       "inputs": [(dict(rows=-1), "SHAPE"), (dict(rows=(1 << 30) + 1), "SHAPE"), (dict(heads=0), "SHAPE"),
                  (dict(k_heads=0), "SHAPE"), (dict(repeat=0), "SHAPE"), (dict(repeat=65), "SHAPE"), (dict(d_k=80), "UNSUPPORTED"),
                  (dict(d_k=0), "SHAPE"), (dict(dtype=3), "DTYPE"), (dict(q_scale=float("inf")), "SHAPE"),
                  (dict(q_scale=float("nan")), "SHAPE"), (dict(eps=-1.0), "SHAPE"), (dict(eps=float("nan")), "SHAPE"),
                  (dict(eps=float("inf")), "SHAPE"), (dict(rows=1 << 30, k_heads=1 << 14), "SHAPE")],
       "norm": [(dict(rows=-1), "SHAPE"), (dict(rows=(1 << 30) + 1), "SHAPE"), (dict(heads=0), "SHAPE"), (dict(d_v=0), "SHAPE"),
                (dict(d_v=24), "SHAPE"), (dict(d_v=1040), "SHAPE"), (dict(x_dtype=2), "DTYPE"), (dict(dtype=-1), "DTYPE"),
                (dict(gate=3), "SHAPE"), (dict(gate=-1), "SHAPE"), (dict(eps=-1e-9), "SHAPE"), (dict(eps=float("nan")), "SHAPE"),
                (dict(rows=1 << 30, heads=1 << 10), "SHAPE")]}


@pytest.mark.parametrize("name", list(NAMES))
def test_shapes(name):
    for change, want in BAD[name]:
        assert call(name, shape(name, **change)) == getattr(B, "SLA_ERR_" + want), change


@pytest.mark.parametrize("name", list(NAMES))
def test_strides(name):
    good = {"prefill": [512, 512, 512], "conv": [1024], "inputs": [512, 512, 8, 8], "norm": [512]}[name]
    for i, g in enumerate(good):
        for bad, want in ((g - 1, "SHAPE"), (0, "SHAPE"), (-g, "SHAPE"), (g + 4, "UNSUPPORTED"), ((1 << 22) + 8, "UNSUPPORTED")):
            if name == "inputs" and i >= 2 and bad == g + 4:
                continue  # gates lie as they like
            s = list(good)
            s[i] = bad
            assert call(name, strides=s) == getattr(B, "SLA_ERR_" + want), (i, bad)


def test_workspace():
    L = B.lib()
    s = shape("prefill")
    need = L.sla_prefill_workspace_bytes(ctypes.byref(s))
    assert need > 0
    assert call("prefill", s, ws=None) == B.SLA_ERR_NULL
    assert call("prefill", s, ws_bytes=need - 1) == B.SLA_ERR_SHAPE
    assert call("prefill", s, **odd("prefill"), ws_bytes=need) == B.SLA_ERR_UNSUPPORTED
    assert L.sla_prefill_workspace_bytes(ctypes.byref(shape("prefill", tokens=6))) == 0  # as few as go token by token
    for change, _ in BAD["prefill"]:
        assert L.sla_prefill_workspace_bytes(ctypes.byref(shape("prefill", **change))) == 0
    more = L.sla_prefill_workspace_bytes(ctypes.byref(shape("prefill", tokens=2000)))
    assert need < more < 2 * need + need


@pytest.mark.parametrize("name", list(NAMES))
def test_outputs_overlap_nothing(name):
    at = {k: (i + 1) * 64 * GIB for i, k in enumerate(NAMES[name])}
    for w in WRITES[name]:
        for other in NAMES[name]:
            if other == w or (w, other) == ("state_out", "state") or (name == "norm" and other == "z"):
                continue
            assert call(name, **{w: at[other]}) == B.SLA_ERR_ALIAS, (w, other)


def test_in_place():
    for name in ("prefill", "conv"):
        at = 64 * GIB * (NAMES[name].index("state") + 1)
        assert call(name, state_out=at, **odd(name)) == B.SLA_ERR_UNSUPPORTED   # in place: in order
        assert call(name, state_out=at + 16) == B.SLA_ERR_ALIAS
        assert call(name, state_out=at - 16) == B.SLA_ERR_ALIAS
    x = 64 * GIB
    assert call("norm", y=x) == B.SLA_ERR_ALIAS                                   # fp32 x, bf16 y
    same = shape("norm", x_dtype=B.SLA_DTYPE_BF16)
    assert call("norm", same, y=x + 16) == B.SLA_ERR_ALIAS
    assert call("norm", same, y=x + 4, x=x + 4) == B.SLA_ERR_UNSUPPORTED           # in place: in order but misaligned
    assert call("norm", y=2 * x, strides=[520]) == B.SLA_ERR_ALIAS                # over a z with gaps
    assert call("norm", y=2 * x + 4, z=2 * x + 4) == B.SLA_ERR_UNSUPPORTED


def test_constants():
    assert (B.SLA_GATE_NONE, B.SLA_GATE_SILU, B.SLA_GATE_SIGMOID) == (0, 1, 2) and B.sla_version() >= 20200

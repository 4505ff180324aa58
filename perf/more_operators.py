"""Performance cases of a recurrent layer's prompt pass: whole prompts, ragged
over a batch, through the layer's short convolution, its norms and gates, the
gated delta rule and the gated norm of its output.

A serving engine packs the tokens of a batch's sequences into rows, one behind
the other: sequence b has the rows seq_start[b] .. seq_start[b + 1] - 1.  The
layer's fused projection is convolved along each sequence behind its committed
inputs (``conv``); queries and keys are normalised over the head and the raw
gates turned into decays and strengths (``inputs``); the recurrence runs over
the tokens from each sequence's state to its next one (``prefill``); its output
is normalised head by head and gated (``norm``).

A case is a dict of plain values: ``listed`` gives the fixed ones, ``draw`` one
more of the same ranges, ``prepare`` the device tensors of a case, ``run`` one
pass, ``work`` the bytes and operations a pass cannot do without, and ``exact``
the same outputs in 64 bits.

Layout.  q, k [T][key heads][d_k], v, out [T][heads][d_v]; value head h reads
key head h // (heads / key heads).  A state is [B][heads][d_k][d_v] in fp32, a
convolution's state [B][K - 1][channels] in fp32, oldest row first.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
CHUNK = 64


# ------------------------------------------------------------------- cases
def _named(name, case):
    return dict(name=name, **case) if name else case


def _prefill(name, batch, lo, hi, *, heads=16, k_heads=16, d_k=128, d_v=128, dtype="bf16", family="gdn", fused=True,
             fresh=False):
    return _named(name, dict(op="prefill", batch=batch, lo=lo, hi=hi, heads=heads, k_heads=k_heads, d_k=d_k, d_v=d_v,
                             dtype=dtype, family=family, fused=fused, fresh=fresh))


def _conv(name, batch, lo, hi, *, channels=6144, kernel=4, dtype="bf16", bias=False, silu=True):
    return _named(name, dict(op="conv", batch=batch, lo=lo, hi=hi, channels=channels, kernel=kernel, dtype=dtype,
                             bias=bias, silu=silu))


def _inputs(name, rows, *, heads=16, k_heads=16, repeat=1, d_k=128, dtype="bf16"):
    return _named(name, dict(op="inputs", rows=rows, heads=heads, k_heads=k_heads, repeat=repeat, d_k=d_k, dtype=dtype))


def _norm(name, rows, *, heads=16, d_v=128, dtype="bf16", x32=False, gate="silu"):
    return _named(name, dict(op="norm", rows=rows, heads=heads, d_v=d_v, dtype=dtype, x32=x32, gate=gate))


def listed():
    return [
        # one short interactive prompt: latency only
        _prefill("prefill_short", 1, 40, 40, fresh=True),
        # one long document: all of the work lies along the sequence
        _prefill("prefill_long", 1, 32768, 32768, fresh=True),
        # a prompt batch of mixed lengths, every two value heads sharing a key head
        _prefill("prefill_batch", 32, 1, 2048, heads=32),
        # a decode step next to prompts: many sequences of one token
        _prefill("prefill_tokens", 256, 1, 1, d_v=256, fused=False),
        # the largest heads, chunks of prompts that go on behind a state
        _prefill("prefill_wide", 16, 512, 1024, heads=8, k_heads=8, d_k=256, d_v=256),
        # fp32 activations, no decay, sizes that fit no tile, empty sequences among them
        _prefill("prefill_ragged_f32", 23, 0, 777, heads=12, k_heads=4, d_k=64, d_v=80, dtype="f32", family="deltanet",
                 fused=False),
        # the convolution of a mixed prompt batch
        _conv("conv_prompt", 16, 100, 2000),
        # fp32, few and nearly empty sequences, odd channel count
        _conv("conv_ragged_f32", 7, 0, 65, channels=1000, kernel=3, dtype="f32", bias=True, silu=False),
        # a verification round's rows: 64 sequences of 16 nodes, keys written for every value head
        _inputs("inputs_round", 1024, k_heads=8, repeat=2),
        # a prompt batch's rows
        _inputs("inputs_prompt", 32768, heads=32),
        # a verification's fp32 outputs
        _norm("norm_round", 1024, x32=True),
        # a prompt batch's outputs
        _norm("norm_prompt", 32768, heads=32),
    ]


MAX_FLOPS = 1e11
MAX_BYTES = 8e8


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choices(["prefill", "conv", "inputs", "norm"], [6, 2, 1, 1])[0]
    while True:
        dtype = rng.choices(["bf16", "f32"], [3, 1])[0]
        if op in ("prefill", "conv"):
            batch = _log_int(rng, 1, 256)
            hi = _log_int(rng, 1, 32768)
            lo = hi if batch == 1 or rng.random() < 0.2 else rng.randint(0, hi)
        if op == "prefill":
            k_heads = rng.choice([1, 2, 3, 4, 8, 16])
            case = _prefill(None, batch, lo, hi, heads=k_heads * rng.choice([1, 1, 2, 3, 4]), k_heads=k_heads,
                            d_k=rng.choice([64, 128, 128, 256]), d_v=16 * _log_int(rng, 1, 16), dtype=dtype,
                            family=rng.choice(["gdn", "gdn", "deltanet", "decay"]), fused=rng.random() < 0.5,
                            fresh=rng.random() < 0.3)
        elif op == "conv":
            case = _conv(None, batch, lo, hi, channels=8 * _log_int(rng, 1, 1024), kernel=rng.randint(2, 4),
                         dtype=dtype, bias=rng.random() < 0.5, silu=rng.random() < 0.7)
        elif op == "inputs":
            k_heads, repeat = rng.choice([1, 2, 4, 6, 8, 16]), rng.choice([1, 2, 3])
            case = _inputs(None, _log_int(rng, 1, 32768), heads=k_heads * rng.choice([1, 2, 3]), k_heads=k_heads,
                           repeat=repeat, d_k=rng.choice([64, 128, 256]), dtype=dtype)
        else:
            case = _norm(None, _log_int(rng, 1, 32768), heads=rng.choice([1, 3, 4, 8, 16, 32]),
                         d_v=16 * _log_int(rng, 1, 16), dtype=dtype, x32=rng.random() < 0.5,
                         gate=rng.choice(["silu", "sigmoid", "none"]))
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS and _rows(case) > 0 and _plain_bytes(case) <= 1.5e10:
            return case


def _plain_bytes(case):
    """The padded fp32 rows and 64 x 64 matrices of the plain form."""
    if case["op"] != "prefill":
        return 0
    rows = case["batch"] * -(-max(_lens(case)) // CHUNK) * CHUNK
    return 4 * rows * case["heads"] * (4 * case["d_k"] + 4 * case["d_v"] + 5 * CHUNK)


# ------------------------------------------------------------------ shapes
def _lens(case):
    """Tokens of each sequence: spread evenly over [lo, hi]."""
    lo, hi = case["lo"], case["hi"]
    return [lo + int((hi - lo + 1) * (((b + 1) * 0.6180339887498949) % 1.0)) for b in range(case["batch"])]


def _rows(case):
    return case["rows"] if "rows" in case else sum(_lens(case))


def work(case):
    w = 2 if case["dtype"] == "bf16" else 4
    T = _rows(case)
    if case["op"] == "prefill":
        H, kh, dk, dv = case["heads"], case["k_heads"], case["d_k"], case["d_v"]
        gates = {"gdn": 2, "deltanet": 1, "decay": 1}[case["family"]]
        state = 4 * case["batch"] * H * dk * dv
        return dict(bytes=2 * T * (kh * dk + H * dv) * w + 4 * gates * T * H + state * (1 if case["fresh"] else 2),
                    flops=(4 if case["family"] == "decay" else 6) * T * H * dk * dv)
    if case["op"] == "conv":
        D, K = case["channels"], case["kernel"]
        return dict(bytes=2 * T * D * w + 8 * case["batch"] * (K - 1) * D + 4 * D * K, flops=2 * T * D * K)
    if case["op"] == "inputs":
        kh, dk, H = case["k_heads"], case["d_k"], case["heads"]
        return dict(bytes=T * (2 * kh * dk * w * (1 + case["repeat"]) + H * (2 * w + 8)), flops=8 * T * kh * dk)
    n = T * case["heads"] * case["d_v"]
    return dict(bytes=n * ((4 if case["x32"] else w) + w + (w if case["gate"] != "none" else 0)), flops=8 * n)


# ------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _parts(T, widths, fused, make):
    """Row blocks [T][width]: parts of one row, as a fused projection leaves them, or tensors of their own."""
    if fused:
        return list(make(T, sum(widths)).split(widths, 1))
    return [make(T, w) for w in widths]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(case)
    T = _rows(case)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    uniform = lambda *s: torch.rand(*s, generator=g, device="cuda")
    st = dict(case=case)
    if case["op"] in ("prefill", "conv"):
        B, lens = case["batch"], _lens(case)
        starts = torch.tensor([0] + lens).cumsum(0)
        st.update(seq_start=starts.int().cuda(), longest=max(lens), status=torch.zeros(B, dtype=torch.int32, device="cuda"))
    if case["op"] == "prefill":
        H, kh, dk, dv = case["heads"], case["k_heads"], case["d_k"], case["d_v"]
        q, k, v = _parts(T, [kh * dk, kh * dk, H * dv], case["fused"], lambda *s: torch.empty(*s, dtype=dt, device="cuda"))
        st["q"], st["k"], st["v"] = q.unflatten(1, (kh, dk)), k.unflatten(1, (kh, dk)), v.unflatten(1, (H, dv))
        for x in (st["q"], st["k"]):
            x.copy_(torch.nn.functional.normalize(normal(T, kh, dk), dim=-1))
        st["v"].copy_(normal(T, H, dv))
        st["alpha"] = torch.sigmoid(2 + 3 * uniform(T, H)) if case["family"] != "deltanet" else None
        st["beta"] = torch.sigmoid(normal(T, H)) if case["family"] != "decay" else None
        st["state"] = None if case["fresh"] else 0.1 * normal(B, H, dk, dv)
        st["state_out"] = torch.empty(B, H, dk, dv, device="cuda")
        st["out"] = torch.empty(T, H, dv, dtype=dt, device="cuda")
        if own:
            from paper_2607_16673_amd import binding
            st["workspace"] = binding.prefill_workspace(st["q"], st["v"], B)
    elif case["op"] == "conv":
        D, K = case["channels"], case["kernel"]
        st["x"] = normal(T, D).to(dt)
        st["weight"] = (2 * uniform(D, K) - 1) * K ** -0.5
        st["bias"] = 0.1 * normal(D) if case["bias"] else None
        st["state"] = normal(B, K - 1, D)
        st["state_out"] = torch.empty(B, K - 1, D, device="cuda")
        st["y"] = torch.empty(T, D, dtype=dt, device="cuda")
    elif case["op"] == "inputs":
        H, kh, dk, r = case["heads"], case["k_heads"], case["d_k"], case["repeat"]
        q, k, _ = normal(T, 2 * kh * dk + H * 16).to(dt).split([kh * dk, kh * dk, H * 16], 1)
        st["q"], st["k"] = q.unflatten(1, (kh, dk)), k.unflatten(1, (kh, dk))
        st["a"], st["b"] = (2 * normal(T, 2 * H)).to(dt).split(H, 1)
        st["a_log"], st["dt_bias"] = torch.log(1 + 15 * uniform(H)), normal(H)
        st["q_out"], st["k_out"] = (torch.empty(T, kh * r, dk, dtype=dt, device="cuda") for _ in "qk")
        st["alpha"], st["beta"] = (torch.empty(T, H, device="cuda") for _ in "ab")
    else:
        H, dv = case["heads"], case["d_v"]
        st["x"] = 0.3 * normal(T, H, dv)
        if not case["x32"]:
            st["x"] = st["x"].to(dt)
        st["z"] = normal(T, H, dv).to(dt) if case["gate"] != "none" else None
        st["weight"] = 1 + 0.1 * normal(dv)
        st["y"] = torch.empty(T, H, dv, dtype=dt, device="cuda")
    return st


# -------------------------------------------------------------- plain forms
def _padded(st, width):
    """Row numbers [B][width] of every sequence's tokens, and which of them exist."""
    starts = st["seq_start"].long()
    at = starts[:-1, None] + torch.arange(width, device="cuda")
    live = at < starts[1:, None]
    return at.masked_fill(~live, 0), live


def _plain_prefill(st):
    case = st["case"]
    B, H, dk, dv = case["batch"], case["heads"], case["d_k"], case["d_v"]
    n = -(-st["longest"] // CHUNK)
    at, live = _padded(st, n * CHUNK)

    def rows(x, heads):  # [B][heads][chunks][64][d], zeros past a sequence's end
        x = x[at].float() * live[:, :, None, None]
        x = x.view(B, n, CHUNK, x.shape[2], x.shape[3]).permute(0, 3, 1, 2, 4)
        return x.repeat_interleave(heads // x.shape[1], 1).contiguous()

    def gate(x, fill):  # [B][heads][chunks][64]
        if x is None:
            return torch.ones(B, H, n, CHUNK, device="cuda").masked_fill_(
                ~live.view(B, 1, n, CHUNK).expand(B, H, n, CHUNK), fill)
        return torch.where(live[:, :, None], x[at], fill).view(B, n, CHUNK, H).permute(0, 3, 1, 2)

    q, k, v = rows(st["q"], H), rows(st["k"], H), rows(st["v"], H)
    beta = gate(st["beta"], 0.0)
    log = gate(st["alpha"], 1.0).double().log().cumsum(3)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device="cuda").tril()
    decay = (log[..., :, None] - log[..., None, :]).masked_fill_(~lower, -math.inf).exp_().float()
    since = log.exp().float()[..., None]  # from the chunk's start
    until = decay[..., -1, :, None]       # to its end
    mix = (q @ k.transpose(3, 4).contiguous()) * decay
    solve = None
    if case["family"] != "decay":
        low = (k @ k.transpose(3, 4).contiguous()) * decay * beta[..., None]
        solve = torch.eye(CHUNK, device="cuda").repeat(B, H, n, 1, 1)
        for i in range(1, CHUNK):  # forward substitution, row by row
            solve[..., i, :] -= (low[..., i, None, :i] @ solve[..., :i, :])[..., 0, :]
        solve = solve * beta[..., None, :]
    S = torch.zeros(B, H, dk, dv, device="cuda") if st["state"] is None else st["state"]
    out = torch.empty(B, H, n, CHUNK, dv, device="cuda")
    for c in range(n):
        u = v[:, :, c]
        if solve is not None:
            u = solve[:, :, c] @ (u - since[:, :, c] * (k[:, :, c] @ S))
        out[:, :, c] = since[:, :, c] * (q[:, :, c] @ S) + mix[:, :, c] @ u
        S = since[:, :, c, -1:] * S + (k[:, :, c] * until[:, :, c]).transpose(2, 3).contiguous() @ u
    st["out"][at[live]] = out.permute(0, 2, 3, 1, 4).flatten(1, 2)[live].to(st["out"].dtype)
    st["state_out"].copy_(S)
    return st["out"], st["state_out"]


def _plain_conv(st):
    case = st["case"]
    K = case["kernel"]
    starts = st["seq_start"].long()
    rows = torch.arange(st["x"].shape[0], device="cuda")
    seq = torch.bucketize(rows, starts[1:], right=True)
    place = rows - starts[seq]
    y = torch.zeros(st["x"].shape, device="cuda") if st["bias"] is None else st["bias"].expand(st["x"].shape)
    for i in range(K):  # the input K - 1 - i tokens earlier
        back = place - (K - 1 - i)
        z = torch.where((back >= 0)[:, None], st["x"][(rows - (K - 1 - i)).clamp(min=0)].float(),
                        st["state"][seq, (K - 1 + back).clamp(0, K - 2)])
        y = y + st["weight"][:, i] * z
    if case["silu"]:
        y = y / (1 + torch.exp(-y))
    st["y"].copy_(y)
    lens = (starts[1:] - starts[:-1])[:, None]
    step = lens - (K - 1) + torch.arange(K - 1, device="cuda")  # tokens of the next state, below 0 the old one's
    old = st["state"].gather(1, (K - 1 + step).clamp(0, K - 2)[..., None].expand_as(st["state"]))
    new = st["x"][(starts[:-1, None] + step).clamp(0, len(rows) - 1)].float()
    torch.where((step >= 0)[..., None], new, old, out=st["state_out"])
    return st["y"], st["state_out"]


def _plain_inputs(st):
    case = st["case"]
    res = []
    for x, scale in ((st["q"], case["d_k"] ** -0.5), (st["k"], 1.0)):
        y = x.float()
        y = y * torch.rsqrt((y * y).sum(-1, keepdim=True) + EPS) * scale
        res.append(y.repeat_interleave(case["repeat"], 1).to(x.dtype))
    x = st["a"].double() + st["dt_bias"]
    soft = torch.where(x > 0, x, 0.0) + torch.log1p(torch.exp(-x.abs()))
    alpha = torch.exp(-torch.exp(st["a_log"].double()) * soft).float()
    beta = (1 / (1 + torch.exp(-st["b"].double()))).float()
    return res[0], res[1], alpha, beta


def _plain_norm(st):
    x = st["x"].float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * st["weight"]
    if st["z"] is not None:
        z = st["z"].float()
        y = y * (z if st["case"]["gate"] == "silu" else 1.0) / (1 + torch.exp(-z))
    return y.to(st["y"].dtype)


# --------------------------------------------------------------------- run
def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return dict(prefill=_plain_prefill, conv=_plain_conv, inputs=_plain_inputs, norm=_plain_norm)[op](st)
    from paper_2607_16673_amd import binding as B
    if op == "prefill":
        B.sla_prefill(st["q"], st["k"], st["v"], st["alpha"], st["beta"], st["seq_start"], st["out"], st["state_out"],
                      state=st["state"], workspace=st["workspace"], status=st["status"], family=case["family"])
        return st["out"], st["state_out"]
    if op == "conv":
        B.sla_conv_prefill(st["x"], st["weight"], st["seq_start"], st["y"], st["state_out"], conv_state=st["state"],
                           bias=st["bias"], status=st["status"], activation=case["silu"])
        return st["y"], st["state_out"]
    if op == "inputs":
        B.sla_recurrent_inputs(st["q"], st["k"], st["a"], st["b"], st["a_log"], st["dt_bias"], st["q_out"], st["k_out"],
                               st["alpha"], st["beta"], q_scale=case["d_k"] ** -0.5, eps=EPS)
        return st["q_out"], st["k_out"], st["alpha"], st["beta"]
    B.sla_gated_norm(st["x"], st["z"], st["weight"], st["y"], eps=EPS, gate=case["gate"])
    return st["y"]


# ------------------------------------------------------------------- exact
def _exact_prefill(st, case):
    """Token by token, from the recurrence itself."""
    B, H, dk, dv, kh = case["batch"], case["heads"], case["d_k"], case["d_v"], case["k_heads"]
    lens = _lens(case)
    if 48.0 * B * H * dk * dv * max(lens) > 2e13:
        return None
    begin = torch.tensor([0] + lens).cumsum(0)[:-1].cuda()
    count = torch.tensor(lens).cuda()
    S = torch.zeros(B, H, dk, dv, dtype=torch.float64, device="cuda")
    if st["state"] is not None:
        S += st["state"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    heads = torch.arange(H, device="cuda") // (H // kh)
    order = sorted(range(B), key=lambda b: -lens[b])  # the longest first: a step's sequences are the first ones
    order_t = torch.tensor(order).cuda()
    S, begin = S[order_t], begin[order_t]
    active, t = B, 0
    ranked = [lens[b] for b in order]
    del count
    while t < ranked[0]:
        while ranked[active - 1] <= t:
            active -= 1
        r = begin[:active] + t
        k, q, v = st["k"][r][:, heads].double(), st["q"][r][:, heads].double(), st["v"][r].double()
        s = S[:active]
        if st["alpha"] is not None:
            s *= st["alpha"][r].double()[..., None, None]
        if st["beta"] is not None:
            v = st["beta"][r].double()[..., None] * (v - (k[..., None] * s).sum(2))
        s += k[..., None] * v[..., None, :]
        out[r] = (q[..., None] * s).sum(2)
        t += 1
    final = torch.empty_like(S)
    final[order_t] = S
    return out, final


def _exact_conv(st, case):
    """One sequence at a time: its rows behind its state's, every window as it lies."""
    K, D = case["kernel"], case["channels"]
    y, last, at = [], [], 0
    w = st["weight"].double()
    for b, n in enumerate(_lens(case)):
        line = torch.cat([st["state"][b].double(), st["x"][at:at + n].double()])
        at += n
        last.append(line[n:])
        if n:
            s = (line.unfold(0, K, 1) * w).sum(-1)
            if case["bias"]:
                s = s + st["bias"].double()
            y.append(s * torch.sigmoid(s) if case["silu"] else s)
    return torch.cat(y), torch.stack(last)


def _exact_inputs(st, case):
    unit = lambda x: x.double() / torch.sqrt(x.double().pow(2).sum(-1, keepdim=True) + EPS)
    spread = lambda x: torch.stack([x] * case["repeat"], 2).flatten(1, 2)
    rate = st["a_log"].double().exp() * torch.nn.functional.softplus(st["a"].double() + st["dt_bias"].double(), threshold=60.0)
    return (spread(unit(st["q"]) / math.sqrt(case["d_k"])), spread(unit(st["k"])), torch.exp(-rate),
            torch.sigmoid(st["b"].double()))


def _exact_norm(st, case):
    x = st["x"].double()
    y = st["weight"].double() * x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / case["d_v"] + EPS)
    if case["gate"] == "silu":
        y = y * torch.nn.functional.silu(st["z"].double())
    elif case["gate"] == "sigmoid":
        y = y * torch.sigmoid(st["z"].double())
    return y


def exact(case, seed):
    st = prepare(case, seed)
    return dict(prefill=_exact_prefill, conv=_exact_conv, inputs=_exact_inputs, norm=_exact_norm)[case["op"]](st, case)

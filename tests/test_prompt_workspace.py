"""The size of sla_prefill's workspace, on the CPU: a serving loop sizes one for its
largest call, and every smaller call has to take it."""
import ctypes
import random

import pytest

from paper_2607_16673_amd import binding as B


def need(tokens, batch, heads=4, k_heads=None, d_k=128, d_v=64, dtype=B.SLA_DTYPE_BF16, family=B.SLA_FAMILY_GDN):
    s = B.SlaPrefillShape(tokens, batch, heads, k_heads or heads, d_k, d_v, dtype, family)
    return B.lib().sla_prefill_workspace_bytes(ctypes.byref(s))


@pytest.mark.parametrize("heads,d_v", [(1, 16), (4, 64), (16, 128), (65, 16), (1100, 64)])
@pytest.mark.parametrize("dtype", [B.SLA_DTYPE_BF16, B.SLA_DTYPE_F32])
def test_it_grows_with_tokens_and_sequences(heads, d_v, dtype):
    """Both limits of the division (how many workgroups, how many tokens to a sequence) lie in these ranges."""
    tokens = sorted({0, 1, *range(5, 30), 63, 64, 65, 127, 200, 400, 1000, 2000, 16384, 16385, 20000, 100000})
    batch = sorted({*range(1, 34), 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300, 1023, 1024, 1025, 5000, 65535})
    table = [[need(t, b, heads=heads, d_v=d_v, dtype=dtype) for b in batch] for t in tokens]
    for row in table:
        assert all(x <= y for x, y in zip(row, row[1:]))
    for a, b in zip(table, table[1:]):
        assert all(x <= y for x, y in zip(a, b))
    assert not any(table[tokens.index(6)]) and table[-1][0] > 0


def test_it_grows_in_random_shapes():
    rng = random.Random(1)
    for _ in range(3000):
        kh, d_k, d_v = rng.choice([1, 2, 4, 16]), rng.choice([64, 128, 256]), 16 * rng.randint(1, 16)
        shape = dict(heads=kh * rng.choice([1, 2, 3]), k_heads=kh, d_k=d_k, d_v=d_v, dtype=rng.randint(0, 1),
                     family=rng.randint(0, 2))
        t, b = int(2 ** rng.uniform(0, 21)), int(2 ** rng.uniform(0, 15.99))
        whole = need(t, b, **shape)
        assert need(rng.randint(0, t), rng.randint(1, b), **shape) <= whole


def test_it_is_refused_when_too_small():
    """A call takes what the size of its own shape says, whichever way its sequences go."""
    L = B.lib()
    for tokens, batch in ((20, 256), (20, 2), (2000, 255), (2000, 256), (40, 40)):
        s = B.SlaPrefillShape(tokens, batch, 4, 4, 128, 64, B.SLA_DTYPE_BF16, B.SLA_FAMILY_GDN)
        n = need(tokens, batch)
        at = [(i + 1) << 36 for i in range(10)]
        call = lambda ws, size, out: L.sla_prefill(ctypes.byref(s), at[0], at[1], 512, at[2], 512, at[3], 256, at[4], at[5],
                                                   at[6], out, at[8], ws, size, None, None)
        assert n > 0
        assert call(None, n, at[7]) == B.SLA_ERR_NULL and call(at[9], n - 1, at[7]) == B.SLA_ERR_SHAPE
        assert call(at[9], n, at[7] + 4) == B.SLA_ERR_UNSUPPORTED  # in order but for a misaligned output


@pytest.mark.gpu
def test_one_workspace_for_a_loop_whose_sequences_leave():
    from prompt_util import Prompt

    largest = Prompt([7] * 255 + [215], heads=4, dk=64, dv=32)
    ws = largest.workspace()
    largest.check(largest.run(workspace=ws))
    for lens in ([7] * 254 + [215], [7] * 30 + [215], [215], [1900], [3] * 200, [20], [1] * 256):
        p = Prompt(lens, heads=4, dk=64, dv=32, seed=len(lens))
        p.check(p.run(workspace=ws))


def test_it_stays_within_two_gib_or_eight_times_the_states():
    for tokens in (1 << 17, 1 << 20, 1 << 26, 1 << 30):
        for batch in (1, 8, 512):
            if (tokens // 64 + batch) * 32 >= 1 << 31:
                continue
            states = batch * 32 * 128 * 128 * 4
            assert 1 << 29 < need(tokens, batch, heads=32, k_heads=16, d_v=128) <= max(2 << 30, 8 * states) + (1 << 20)


def packed(lens, heads, dk, dv, dtype, family="gdn", fresh=False):
    """Inputs too large to be made on the host."""
    import torch

    g = torch.Generator(device="cuda").manual_seed(sum(lens))
    T, dt = sum(lens), torch.bfloat16 if dtype == "bf16" else torch.float32
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
    unit = lambda: torch.nn.functional.normalize(rand(T, heads, dk), dim=-1).to(dt)
    return dict(q=unit(), k=unit(), v=rand(T, heads, dv).to(dt), beta=None if family == "decay" else torch.sigmoid(rand(T, heads)),
                alpha=None if family == "deltanet" else torch.sigmoid(3 + rand(T, heads)),
                state=None if fresh else 0.1 * rand(len(lens), heads, dk, dv))


def run(p, lens, family="gdn", state="own", first=0, in_place=False):
    """The call on the rows of `lens` from row `first` on."""
    import torch

    T, H, dv = sum(lens), p["v"].shape[1], p["v"].shape[2]
    part = lambda name: None if p[name] is None else p[name][first:first + T]
    q, v = part("q"), part("v")
    state = p["state"] if isinstance(state, str) else state
    out = torch.full((T, H, dv), 7.0, dtype=v.dtype, device="cuda")
    into = state if in_place else torch.full((len(lens), H, q.shape[2], dv), 7.0, device="cuda")
    status = torch.full((len(lens),), 9, dtype=torch.int32, device="cuda")
    start = torch.tensor([0, *lens], device="cuda").cumsum(0).int()
    ws = B.prefill_workspace(q, v, len(lens), family=family)
    B.sla_prefill(q, part("k"), v, part("alpha"), part("beta"), start, out, into, state=state, workspace=ws, status=status,
                  family=family)
    torch.cuda.synchronize()
    assert status.eq(0).all()
    return out, into, 0 if ws is None else ws.numel()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,fresh", [("bf16", True), ("f32", False)])
def test_a_prompt_in_several_passes_is_the_prompt_in_parts(dtype, fresh):
    """A long sequence, its rows at multiples of 64 handed over in calls of one pass: the same chunks, equal bits."""
    import torch

    n, part = (28000, 9600) if dtype == "bf16" else (22000, 8960)
    p = packed([n], 64, 256, 48, dtype, fresh=fresh)
    out, state, ws = run(p, [n])
    assert ws <= (2 << 30) + (1 << 20)
    carried, at = "own", 0
    while at < n:
        rows = min(part, n - at)
        o, carried, small = run(p, [rows], state=carried, first=at)
        assert small < ws * 1.01 and torch.equal(o, out[at:at + rows])
        at += rows
    assert torch.equal(carried, state)


@pytest.mark.gpu
@pytest.mark.parametrize("family,lens", [("gdn", [6000, 0, 65, 16000, 3]), ("decay", [1, 24000, 500]), ("deltanet", [9000] * 3)])
def test_batches_in_several_passes(family, lens):
    """Each sequence alone, in parts of one pass, gives the same bits: 32 columns to a workgroup either way."""
    import torch

    p = packed(lens, 64, 256, 80, "f32", family=family)
    out, state, ws = run(p, lens, family=family)
    assert ws <= (2 << 30) + (1 << 20)
    first = 0
    for b, n in enumerate(lens):
        carried, at = p["state"][b:b + 1], 0
        while at < n:
            rows = min(8960, n - at)
            o, carried, _ = run(p, [rows], family=family, state=carried, first=first + at)
            if n > 6:
                assert torch.equal(o, out[first + at:first + at + rows])
            else:  # alone it goes token by token
                assert (o - out[first + at:first + at + rows]).abs().max() <= 2e-5 * o.abs().max()
            at += rows
        if n > 6 or n == 0:
            assert torch.equal(carried, state[b:b + 1])
        first += n
    again = {**p, "state": p["state"].clone()}
    o, s, _ = run(again, lens, family=family, in_place=True)
    assert torch.equal(o, out) and torch.equal(s, state) and s.data_ptr() == again["state"].data_ptr()


@pytest.mark.gpu
def test_many_sequences_in_several_passes():
    """More sequences than a pass has slots for two chunks of each, most of them token by token."""
    import torch

    lens = [int(x) for x in torch.randint(1, 25, (396,), generator=torch.Generator().manual_seed(1))] + [9000, 64, 65, 7000]
    p = packed(lens, 64, 256, 16, "f32")
    assert sum(lens) <= 64 * len(lens)
    out, state, ws = run(p, lens)
    first = 0
    for b, n in enumerate(lens):
        if n > 24 or b % 40 == 0:
            o, s, _ = run(p, [n], state=p["state"][b:b + 1], first=first)
            for x, y in ((o, out[first:first + n]), (s, state[b:b + 1])):
                assert (x - y).float().abs().max() <= 2e-5 * y.float().abs().max()
        first += n


@pytest.mark.gpu
def test_several_passes_in_a_replayed_graph_and_bad_starts():
    import torch

    lens = [15000, 4000]
    p = packed(lens, 64, 256, 16, "f32")
    want = run(p, lens)
    start = torch.tensor([0, 15000, 19000], dtype=torch.int32, device="cuda")
    out, state = torch.empty_like(want[0]), torch.empty_like(want[1])
    status = torch.empty(2, dtype=torch.int32, device="cuda")
    ws = B.prefill_workspace(p["q"], p["v"], 2)
    call = lambda: B.sla_prefill(p["q"], p["k"], p["v"], p["alpha"], p["beta"], start, out, state, state=p["state"],
                                 workspace=ws, status=status)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in (out, state, status):
            t.fill_(7)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(state, want[1]) and status.eq(0).all()
    start[1] = 20000
    out.fill_(7.0)
    state.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert status.eq(B.SLA_ERR_LENGTH).all() and out.eq(7).all() and state.eq(7).all()

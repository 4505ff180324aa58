"""The recurrence over packed sequences (sla_prefill) on the GPU, against the
fp64 oracle: families, types, head layouts, lengths from none to several chunks,
strides, states, gates; streams, graphs, errors; equality with verification."""
import numpy as np
import pytest
import torch

from paper_2607_16673_amd import binding as B
from prompt_util import Prompt, close, f64, starts_of

pytestmark = pytest.mark.gpu

LENS = [1, 0, 63, 64, 65, 2, 130, 0, 257]


@pytest.mark.parametrize("family", ["gdn", "deltanet", "decay"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk", [64, 128, 256])
def test_families_types_and_heads(family, dtype, dk):
    p = Prompt(LENS, dk=dk, dv=64, dtype=dtype, family=family, seed=dk)
    p.check(p.run())


@pytest.mark.parametrize("dv", [16, 32, 48, 80, 112, 128, 208, 256, 1024])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_value_widths(dtype, dv):
    p = Prompt([70, 3, 128], heads=1, dk=64, dv=dv, dtype=dtype, seed=dv)
    p.check(p.run())


@pytest.mark.parametrize("heads,k_heads", [(1, 1), (4, 2), (6, 2), (8, 1), (3, 3), (12, 4)])
@pytest.mark.parametrize("fused", [False, True])
def test_grouped_heads_and_strides(heads, k_heads, fused):
    p = Prompt([33, 100], heads=heads, k_heads=k_heads, dv=32, fused=fused, seed=heads)
    p.check(p.run())
    p = Prompt([33, 100], heads=heads, k_heads=k_heads, dk=64, dv=32, fused=fused, dtype="f32", seed=heads)
    p.check(p.run())


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 127, 128, 129, 191, 192, 193, 640, 1000])
def test_lengths(n):
    p = Prompt([n], heads=2, seed=n, fresh=n % 2 == 0)
    p.check(p.run())


@pytest.mark.parametrize("lens", [[0], [0, 0, 0], [1] * 130, [0, 1] * 40, [200, 1, 0, 0, 1], [64] * 5, [63, 1, 64, 128]])
@pytest.mark.parametrize("fresh", [False, True])
def test_batches(lens, fresh):
    p = Prompt(lens, heads=2, dk=64, dv=48, fresh=fresh, seed=len(lens))
    p.check(p.run())


@pytest.mark.parametrize("before,behind", [(0, 5), (7, 0), (129, 200)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_sequence_are_neither_read_nor_written(before, behind, dtype):
    p = Prompt([40, 70], before=before, behind=behind, dtype=dtype, dv=32)
    want = p.exact()
    for t in (p.q, p.k, p.v, p.alpha, p.beta):
        t[:before] = float("nan")
        t[before + 110:] = float("nan")
    p.check(p.run(), want)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("what", ["q", "k", "v", "beta"])
def test_neighbours_are_untouched_by_bad_values(what, bad):
    """A bad value spoils its sequence from its chunk of 64 tokens on, and nothing else."""
    p = Prompt([37, 170, 90], dv=32)
    clean = p.run()
    want = p.exact()
    getattr(p, what)[p.starts[1] + 70] = bad
    out, state, status = p.run()
    torch.cuda.synchronize()
    assert status.eq(0).all()
    for b in (0, 2):
        rows = slice(p.starts[b], p.starts[b + 1])
        assert torch.equal(out[rows], clean[0][rows]) and torch.equal(state[b], clean[1][b])
    first = slice(p.starts[1], p.starts[1] + 64)
    close(out[first], want[0][first])


def test_the_past_does_not_see_the_future():
    p = Prompt([150], dv=32)
    first = p.run()[0].clone()
    p.v[100:] = 50.0
    p.beta[100:] = 0.9
    assert torch.equal(p.run()[0][:100], first[:100])


def strong(T, H, g):
    a = 1e-3 + 0.3 * torch.rand(T, H, generator=g)
    r = torch.rand(T, H, generator=g)
    a[r < 0.05] = 1e-20
    a[(r >= 0.05) & (r < 0.1)] = 1e-38
    a[r > 0.6] = 0.999
    return a


GATES = {"strong": (strong, None), "none": (lambda T, H, g: torch.ones(T, H), None),
         "no_update": (None, lambda T, H, g: torch.zeros(T, H)),
         "full_update": (lambda T, H, g: torch.ones(T, H), lambda T, H, g: torch.ones(T, H)),
         "twice": (None, lambda T, H, g: torch.full((T, H), 1.9))}


@pytest.mark.parametrize("name", list(GATES))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates(name, dtype):
    alpha, beta = GATES[name]
    p = Prompt([200, 64, 17], dv=32, dtype=dtype, alpha=alpha, beta=beta)
    p.check(p.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_keys(dtype):
    """Every token with the same key: each overwrites what the last one wrote."""
    p = Prompt([128, 77], dv=32, dtype=dtype, beta=lambda T, H, g: torch.full((T, H), 0.97))
    p.k[:] = p.k[0]
    p.check(p.run())


@pytest.mark.parametrize("lens", [[1] * 40 + [500] + [2] * 30, [7, 6, 5, 8, 0, 24, 25, 26, 23], [1] * 100 + [30] * 3 + [0] * 20,
                                  [25] * 70 + [24] * 70, [0, 0, 300, 0, 0]])
@pytest.mark.parametrize("heads", [2, 12])
def test_short_and_long_sequences_together(lens, heads):
    """Batches of which some sequences go token by token and some in chunks, with many and few workgroups."""
    p = Prompt(lens, heads=heads, dk=64, dv=48, seed=heads)
    p.check(p.run())


@pytest.mark.parametrize("lens", [[100, 3, 0, 64], [1, 1, 0, 1]])
def test_in_place_is_the_same(lens):
    p = Prompt(lens, dv=48)
    out, state, _ = p.run()
    mine = p.state.clone()
    again, _, status = p.run(state_out=mine, state=mine)
    assert torch.equal(out, again) and torch.equal(state, mine) and status.eq(0).all()


def test_no_state_is_a_state_of_zeros():
    p = Prompt([70, 0, 1, 129], dv=32, fresh=True)
    out, state, _ = p.run()
    zero, zstate, _ = p.run(state=torch.zeros_like(state))
    assert torch.equal(out, zero) and torch.equal(state, zstate)


@pytest.mark.parametrize("cut", [1, 64, 100])
def test_a_prompt_in_two_parts(cut):
    whole = Prompt([200], dv=64, seed=3)
    want = whole.exact()
    out, state, status = whole.outputs()
    mid = torch.empty_like(state)
    for first, last, into, state_in in ((0, cut, mid, whole.state), (cut, 200, state, mid)):
        start = torch.tensor([0, last - first], dtype=torch.int32, device="cuda")
        part = lambda t: t[first:last]
        B.sla_prefill(part(whole.q), part(whole.k), part(whole.v), part(whole.alpha), part(whole.beta), start,
                      part(out), into, state=state_in, status=status,
                      workspace=B.prefill_workspace(part(whole.q), part(whole.v), 1))
    whole.check((out, state, status), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("family", ["gdn", "deltanet", "decay"])
def test_chains_verified_and_committed_give_the_same(dtype, family):
    """A prompt of 64 tokens a sequence against one chain draft: outputs, and states after a full commit."""
    n, H = 64, 3
    p = Prompt([n] * 4, heads=H, dv=64, dtype=dtype, family=family)
    out, state, _ = p.run()
    four = lambda t: None if t is None else t.reshape(4, n, *t.shape[1:]).contiguous()
    parent = torch.arange(-1, n - 1, dtype=torch.int32, device="cuda").repeat(4, 1)
    o = torch.empty(4, n, H, 64, device="cuda")
    factors = B.Factors.empty(4, n, H, p.dk, 64, p.dt, family=family)
    mine = p.state.clone()
    B.sla_verify(mine, four(p.q), four(p.k), four(p.v), four(p.alpha), four(p.beta), parent, o, factors, family=family,
                 topology="chain")
    B.sla_commit(mine, factors, parent + 1, torch.full((4,), n, dtype=torch.int32, device="cuda"), family=family)
    close(state, f64(mine))
    close(out.view(4, n, H, 64), f64(o))


BAD = [[0, 10, 5, 20], [-1, 5, 6, 20], [0, 5, 10, 21], [5, 4, 4, 4], [0, 1 << 30, 3, 4], [-(1 << 31), 0, 0, 0],
       [0, 0, 0, (1 << 31) - 1]]


@pytest.mark.parametrize("starts", BAD)
def test_bad_starts_are_told_of_every_sequence(starts):
    p = Prompt([5, 5, 10], dv=32)
    p.start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    out, state, status = p.run()
    torch.cuda.synchronize()
    assert status.tolist() == [B.SLA_ERR_LENGTH] * 3
    assert out.eq(7).all() and state.eq(7).all()


def test_bad_starts_far_back_in_a_large_batch():
    p = Prompt([3] * 300, heads=1, dk=64, dv=16)
    p.start[290] = 1000
    out, state, status = p.run()
    torch.cuda.synchronize()
    assert status.eq(B.SLA_ERR_LENGTH).all() and out.eq(7).all() and state.eq(7).all()


@pytest.mark.parametrize("lens", [[300, 5, 64, 1], [1] * 9])
def test_equal_calls_give_equal_bits_in_any_batch(lens):
    p = Prompt(lens, heads=2, dv=48)
    out, state, _ = p.run()
    again = p.run()
    assert torch.equal(out, again[0]) and torch.equal(state, again[1])
    want = p.exact()
    for b, n in enumerate(lens):  # the same number of rows, the others of no sequence
        one = Prompt(lens, heads=2, dv=48)
        one.B, one.state = 1, p.state[b:b + 1].clone()
        one.start = torch.tensor(p.starts[b:b + 2].tolist(), dtype=torch.int32, device="cuda")
        o, s, _ = one.run()
        rows = slice(p.starts[b], p.starts[b + 1])
        if n > 24:
            assert torch.equal(o[rows], out[rows]) and torch.equal(s, state[b:b + 1])
        else:  # alone it may go another way, in a chunk or by itself: each is a rounding from the exact value
            close(o[rows], want[0][rows])
            close(s, want[1][b:b + 1])


@pytest.mark.parametrize("lens", [[100, 64, 3], [1] * 20])
def test_another_stream_and_a_replayed_graph(lens):
    p = Prompt(lens, dv=32)
    want = p.exact()
    out, state, status = p.outputs()
    ws = p.workspace()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.run(out, state, status, workspace=ws)
    side.synchronize()
    p.check((out, state, status), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(out, state, status, workspace=ws)
    for i in range(4):
        p.v.mul_(-1)  # new inputs in the same places: the outputs follow
        out.fill_(7.0)
        state.fill_(7.0)
        ws is None or ws.fill_(255)
        graph.replay()
        p.check((out, state, status))
        other = Prompt([80, 2], heads=1, dv=16, seed=i)  # the program's own work between replays
        other.check(other.run())


def test_two_graphs_share_a_workspace():
    ps = [Prompt([130, 70], dv=32, seed=s) for s in (1, 2)]
    ws = ps[0].workspace()
    made = [p.outputs() for p in ps]
    graphs = []
    for p, m in zip(ps, made):
        p.run(*m, workspace=ws)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            p.run(*m, workspace=ws)
    for _ in range(3):
        for m in made:
            m[0].fill_(7.0)
            m[1].fill_(7.0)
        for g in graphs:
            g.replay()
        for p, m in zip(ps, made):
            p.check(m)


def test_guard_bands():
    """Nothing in front of or behind the outputs and the workspace is written."""
    p = Prompt([65, 3, 0, 130], heads=3, dv=48, dk=64)
    band = 4096
    bufs = []
    for t in (*p.outputs(), p.workspace()):
        if t is None:
            bufs.append((None, None))
            continue
        n = t.numel() * t.element_size()
        raw = torch.full((n + 2 * band,), 0x5A, dtype=torch.uint8, device="cuda")
        raw[band:band + n] = t.contiguous().view(-1).view(torch.uint8)
        bufs.append((raw, raw[band:band + n].view(t.dtype).view(t.shape)))
    got = [b[1] for b in bufs[:3]]
    p.run(*got, workspace=bufs[3][1])
    p.check(got)
    for raw, _ in bufs:
        if raw is not None:
            assert raw[:band].eq(0x5A).all() and raw[-band:].eq(0x5A).all()


@pytest.mark.parametrize("seed", range(12))
def test_random(seed):
    r = np.random.default_rng(seed)
    lens = [int(x) for x in r.integers(0, r.choice([3, 40, 300]), r.integers(1, 12))]
    kh = int(r.choice([1, 2, 3]))
    p = Prompt(lens, heads=kh * int(r.choice([1, 2, 3])), k_heads=kh, dk=int(r.choice([64, 128, 256])),
               dv=16 * int(r.integers(1, 10)), dtype=str(r.choice(["bf16", "f32"])),
               family=str(r.choice(["gdn", "deltanet", "decay"])), fused=bool(r.integers(2)), fresh=bool(r.integers(2)),
               before=int(r.integers(0, 70)), behind=int(r.integers(0, 70)), seed=seed)
    p.check(p.run())


def test_long_sequences():
    """Thousands of tokens of many heads, the values of two heads against the oracle."""
    p = Prompt([5000, 1, 3333], heads=8, k_heads=4, dk=64, dv=32, seed=11)
    out, state, status = p.run()
    torch.cuda.synchronize()
    assert status.eq(0).all()
    q = Prompt([1], heads=2, k_heads=1, dk=64, dv=32)
    q.lens, q.starts, q.T, q.B, q.family = p.lens, p.starts, p.T, p.B, p.family
    q.q, q.k, q.v = p.q[:, 2:3], p.k[:, 2:3], p.v[:, 4:6]
    q.alpha, q.beta, q.state = p.alpha[:, 4:6], p.beta[:, 4:6], p.state[:, 4:6]
    o, s = q.exact()
    close(out[:, 4:6], o)
    close(state[:, 4:6], s)


def test_starts_of():
    assert starts_of([2, 0, 3], 4).tolist() == [4, 6, 6, 9]

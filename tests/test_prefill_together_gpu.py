"""sla_prefill where one call takes both ways (short sequences token by token, long
ones in chunks), and calls that run at the same time."""
import pytest
import torch

from prompt_util import Prompt

pytestmark = pytest.mark.gpu

MIXED = [1] * 30 + [40, 0, 7, 6]  # 83 tokens of 34 sequences: few to a sequence, some in chunks


def test_a_batch_of_both_ways_in_a_replayed_graph():
    p = Prompt(MIXED, dv=48)
    out, state, status = p.outputs()
    ws = p.workspace()
    assert ws is not None
    p.run(out, state, status, workspace=ws)
    p.check((out, state, status))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(out, state, status, workspace=ws)
    for i in range(4):
        p.v.mul_(-1)
        for t in (out, state):
            t.fill_(7.0)
        status.fill_(99)
        ws.fill_(255)
        graph.replay()
        p.check((out, state, status))
        other = Prompt([3, 90], heads=1, dv=16, seed=i)
        other.check(other.run())


@pytest.mark.parametrize("after", [[34] + [1] * 33, [2] * 34, [0] * 33 + [60]])
def test_a_graph_replayed_with_other_lengths(after):
    """The lengths are on the device: a replay goes by what they are then."""
    p = Prompt(MIXED, dv=32)
    made, ws = p.outputs(), p.workspace()
    p.run(*made, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(*made, workspace=ws)
    other = Prompt(after, dv=32, behind=p.T - sum(after), seed=1)
    for name in ("q", "k", "v", "alpha", "beta", "state", "start"):
        getattr(p, name).copy_(getattr(other, name))
    for _ in range(3):
        for t in made[:2]:
            t.fill_(7.0)
        graph.replay()
        other.check(made)


@pytest.mark.parametrize("lens", [MIXED, [700, 90], [1] * 40])
def test_calls_on_two_streams_at_once(lens):
    ps = [Prompt(lens, heads=4, seed=s) for s in (1, 2)]
    want = [p.exact() for p in ps]
    made, ws = [p.outputs() for p in ps], [p.workspace() for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, m, w, s in zip(ps, made, ws, streams):
            with torch.cuda.stream(s):
                p.run(*m, workspace=w)
    torch.cuda.synchronize()
    for p, m, w in zip(ps, made, want):
        p.check(m, w)


@pytest.mark.parametrize("lens", [MIXED, [1, 0, 5]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_guard_bands(lens, dtype):
    p = Prompt(lens, heads=3, dk=64, dv=48, dtype=dtype, before=2, behind=3)
    band, bufs = 4096, []
    for t in (*p.outputs(), p.workspace()):
        n = 0 if t is None else t.numel() * t.element_size()
        raw = torch.full((n + 2 * band,), 0x5A, dtype=torch.uint8, device="cuda")
        mine = None
        if t is not None:
            raw[band:band + n] = t.contiguous().view(-1).view(torch.uint8)
            mine = raw[band:band + n].view(t.dtype).view(t.shape)
        bufs.append((raw, mine))
    got = [mine for _, mine in bufs[:3]]
    p.run(*got, workspace=bufs[3][1])
    p.check(got)
    for raw, _ in bufs:
        assert raw[:band].eq(0x5A).all() and raw[-band:].eq(0x5A).all()


@pytest.mark.parametrize("value", [0.0, 1e-30, 1e15])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_of_any_size(value, dtype):
    """Outputs scale with the values where the state begins at zero."""
    p = Prompt([130, 64], dk=64, dv=32, dtype=dtype, fresh=True)
    p.v.mul_(value)
    p.check(p.run())

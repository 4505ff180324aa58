"""How far a bad value reaches in sla_prefill, gates included, in both forms; and gates
of zero, which sla_recurrent_inputs gives where a decay underflows."""
import pytest
import torch

from paper_2607_16673_amd import binding as B
from prompt_util import Prompt, close, f64

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), -float("inf")]


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("what", ["alpha", "beta", "v"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_bad_value_of_a_head_stays_in_its_sequence_and_head(what, bad, dtype):
    p = Prompt([37, 170, 90], heads=3, dk=64, dv=32, dtype=dtype)
    clean, want = p.run(), p.exact()
    getattr(p, what)[p.starts[1] + 70, 1] = bad
    out, state, status = p.run()
    torch.cuda.synchronize()
    assert status.eq(0).all()
    mine = slice(p.starts[1], p.starts[2])
    keep = torch.ones(p.T, 3, dtype=torch.bool, device="cuda")
    keep[mine, 1] = False
    assert torch.equal(out[keep], clean[0][keep])
    keep = torch.ones(3, 3, dtype=torch.bool, device="cuda")
    keep[1, 1] = False
    assert torch.equal(state[keep], clean[1][keep])
    first = slice(p.starts[1], p.starts[1] + 64)
    close(out[first], want[0][first])
    assert not state[1, 1].isfinite().all()


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("what", ["alpha", "beta", "q", "k", "v"])
def test_token_by_token(what, bad):
    """Outputs in front of the bad token are right, and so are the other sequences'."""
    p = Prompt([1, 6, 3] + [1] * 20, heads=2, dk=64, dv=32)
    clean, want = p.run(), p.exact()
    at = p.starts[1] + 3
    getattr(p, what)[at] = bad
    out, state, status = p.run()
    torch.cuda.synchronize()
    assert status.eq(0).all() and p.workspace() is not None
    other = torch.ones(p.T, dtype=torch.bool, device="cuda")
    other[at:p.starts[2]] = False
    assert torch.equal(out[other], clean[0][other])
    for b in (0, 2, 5):
        assert torch.equal(state[b], clean[1][b])
    close(out[:at], want[0][:at])


@pytest.mark.parametrize("lens", [[200, 64, 17], [1] * 20 + [5]])
@pytest.mark.parametrize("family", ["gdn", "decay"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gates_of_zero_forget_everything(lens, family, dtype):
    def gates(T, H, g):
        a = torch.rand(T, H, generator=g)
        a[torch.rand(T, H, generator=g) < 0.2] = 0.0
        return a

    p = Prompt(lens, heads=2, dk=64, dv=32, dtype=dtype, family=family, alpha=gates)
    p.check(p.run())


def test_gates_that_underflow_go_through_inputs_and_recurrence():
    n, H = 130, 2
    p = Prompt([n], heads=H, dk=64, dv=32)
    a = torch.full((n, H), 12.0, dtype=torch.bfloat16, device="cuda")
    a[::3] = -3.0
    b, log = torch.zeros_like(a), torch.full((H,), 3.0, device="cuda")
    q, k = torch.empty_like(p.q), torch.empty_like(p.k)
    alpha, beta = torch.empty(n, H, device="cuda"), torch.empty(n, H, device="cuda")
    B.sla_recurrent_inputs(p.q, p.k, a, b, log, None, q, k, alpha, beta)
    assert alpha[1].eq(0).all() and alpha[0].gt(0).all()
    p.q, p.k, p.alpha, p.beta = q, k, alpha, beta
    p.check(p.run())
    # the same rows as a chain draft
    parent = torch.arange(-1, 63, dtype=torch.int32, device="cuda")[None]
    o = torch.empty(1, 64, H, 32, device="cuda")
    row = lambda t: t[None, :64].contiguous()
    B.sla_verify(p.state.clone(), row(q), row(k), row(p.v), row(alpha), row(beta), parent, o,
                 B.Factors.empty(1, 64, H, 64, 32, torch.bfloat16), topology="chain")
    close(o[0], f64(torch.from_numpy(p.exact()[0][:64])))

"""The prompt pass where offsets pass 32 bits and launches 2^32 work-items."""
import pytest
import torch

from paper_2607_16673_amd import binding as B
from prompt_util import Prompt, close, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_prefill_of_rows_behind_4_gib():
    """Two sequences at the end of 600000 rows of 8 KB each."""
    T, step = 600000, 4096
    p = Prompt([70, 130], heads=1, dk=64, dv=32, seed=3)
    row = torch.empty(T, step, dtype=torch.bfloat16, device="cuda")
    row[-200:] = 0
    want = p.exact()
    big = lambda x, at: row[:, at:at + x.shape[1] * x.shape[2]].unflatten(1, x.shape[1:])
    q, k, v = big(p.q, 0), big(p.k, 64), big(p.v, 128)
    for x, y in ((q, p.q), (k, p.k), (v, p.v)):
        x[-200:] = y
    gate = lambda g: torch.cat([torch.full((T - 200, 1), float("nan"), device="cuda"), g])
    start = (p.start + (T - 200)).int()
    out, state = torch.full((T, 1, 32), 7.0, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 1, 64, 32, device="cuda")
    status = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    B.sla_prefill(q, k, v, gate(p.alpha), gate(p.beta), start, out, state, state=p.state, status=status,
                  workspace=B.prefill_workspace(q, v, 2))
    torch.cuda.synchronize()
    assert status.eq(0).all() and out[:-200].eq(7).all()
    close(out[-200:], want[0])
    close(state, want[1])
    # the convolution over the same rows
    x, w = row[:, :256], torch.randn(256, 4, device="cuda")
    y = torch.zeros(T, 256, dtype=torch.bfloat16, device="cuda")
    one = torch.tensor([0, 70, 200], dtype=torch.int32, device="cuda")
    small, new, mine = torch.empty(200, 256, dtype=torch.bfloat16, device="cuda"), *torch.empty(2, 2, 3, 256, device="cuda")
    B.sla_conv_prefill(x, w, start, y, new)
    B.sla_conv_prefill(x[-200:].contiguous(), w, one, small, mine)
    assert torch.equal(y[-200:], small) and torch.equal(new, mine) and y[:-200].eq(0).all()


def test_single_tokens_of_a_large_batch():
    """65535 sequences of a token, 65 heads: more workgroups than one dimension of a launch holds."""
    n, H = 65535, 65
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")
    q, v = z(n, H, 64), z(n, H, 16)
    state = z(n, H, 64, 16, dt=torch.float32)
    p = Prompt([1] * 3, heads=H, dk=64, dv=16, seed=2)
    k = q.clone()
    alpha, beta = torch.ones(n, H, device="cuda"), torch.zeros(n, H, device="cuda")
    for big, small in ((q, p.q), (k, p.k), (v, p.v), (state, p.state), (alpha, p.alpha), (beta, p.beta)):
        big[-3:] = small
    out, status = torch.full_like(v, 7.0), torch.full((n,), 9, dtype=torch.int32, device="cuda")
    ws = B.prefill_workspace(q, v, n)  # for the few sequences that could have more than 24 tokens
    assert ws.numel() < 65 * 4000 * (1 << 17)
    B.sla_prefill(q, k, v, alpha, beta, torch.arange(n + 1, dtype=torch.int32, device="cuda"), out, state, state=state,
                  status=status, workspace=ws)
    torch.cuda.synchronize()
    want = p.exact()
    assert status.eq(0).all() and out[:-3].eq(0).all()
    close(out[-3:], want[0])
    close(state[-3:], want[1])


def test_norm_of_many_rows():
    """2^22 + 5 rows of 4 heads of 1024: four heads to a workgroup, 2^33 bytes and more, in place."""
    n = (1 << 22) + 5
    x = torch.zeros(n, 4, 1024, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, 4, 1024, device="cuda")
    last = x[-3:].clone()
    B.sla_gated_norm(x, None, None, x, gate="none")
    want = last.double() / torch.sqrt(last.double().pow(2).mean(-1, keepdim=True) + 1e-6)
    assert ((x[-3:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()
    assert x[:-3].eq(0).all()


def test_inputs_of_many_rows():
    """2^24 rows of 8 + 8 heads of 64: 32 heads to a workgroup, more of them than one dimension holds."""
    n = 1 << 24
    q = torch.zeros(n, 8, 64, dtype=torch.bfloat16, device="cuda")
    q[-3:] = torch.randn(3, 8, 64, device="cuda")
    a = torch.zeros(n, 1, dtype=torch.bfloat16, device="cuda")
    a[-3:] = 2.0
    out, kout = torch.empty_like(q), torch.empty_like(q)
    beta = torch.empty(n, 1, device="cuda")
    B.sla_recurrent_inputs(q, q, None, a, None, None, out, kout, None, beta)
    want = f64(q[-3:]) / (f64(q[-3:].double().pow(2).sum(-1, keepdim=True)) + 1e-6) ** 0.5
    assert (abs(f64(out[-3:]) * 8 - want) <= 2.0 ** -8 * abs(want) + 1e-6).all()
    assert (abs(f64(kout[-3:]) - want) <= 2.0 ** -8 * abs(want) + 1e-6).all()
    assert out[:-3].eq(0).all() and kout[:-3].eq(0).all()
    assert beta[:-3].eq(0.5).all() and (beta[-3:] - 0.8807971).abs().max() < 1e-5

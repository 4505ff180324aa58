"""The steps around a recurrent layer's core on the GPU, against the fp64
oracle: the convolution along packed sequences, the recurrence's inputs, and the
gated norm; then all four together as a layer, whole and in parts."""
import numpy as np
import pytest
import torch

from oracle import prompt as O
from paper_2607_16673_amd import binding as B
from prompt_util import DT, close, f64, starts_of

pytestmark = pytest.mark.gpu


def rounds_to(got, want, slack):
    """Within half a step of got's type and `slack` of the value (fp32 arithmetic)."""
    x = f64(got)
    bound = (torch.finfo(got.dtype).eps / 2 + slack) * np.abs(want) + 1e-37
    assert (np.abs(x - want) <= bound).all(), float(np.max(np.abs(x - want) / bound))


class Conv:
    def __init__(self, lens, D=64, K=4, dtype="bf16", bias=True, fresh=False, before=0, behind=0, pad=0, seed=0):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g)
        self.starts = starts_of(lens, before)
        self.T, self.B, self.D, self.K = int(self.starts[-1]) + behind, len(lens), D, K
        self.x = rand(self.T, D + pad).to(DT[dtype]).cuda()[:, :D]
        self.w = rand(D, K).cuda()
        self.bias = rand(D).cuda() if bias else None
        self.state = None if fresh or K == 1 else rand(len(lens), K - 1, D).cuda()
        self.start = torch.from_numpy(self.starts).cuda()

    def run(self, silu=True, in_place=False, **over):
        y = torch.full((self.T, self.D), 7.0, dtype=self.x.dtype, device="cuda")
        new = self.state.clone() if in_place else torch.full((self.B, self.K - 1, self.D), 7.0, device="cuda")
        status = torch.full((self.B,), 99, dtype=torch.int32, device="cuda")
        B.sla_conv_prefill(self.x, self.w, self.start, y, new if self.K > 1 else None,
                           conv_state=new if in_place else self.state, bias=self.bias, status=status, activation=silu)
        return y, new, status

    def check(self, got, silu=True):
        """y: sums of K + 1 products, off by (K + 2) 2^-24 of the sum of their sizes, and SiLU by 2e-6
        of its value (and its slope, at most 1.1, of the sum's error); states are copies."""
        y, new, status = got
        want, state = O.conv(f64(self.state), f64(self.x), f64(self.w), f64(self.bias), self.starts, silu)
        torch.cuda.synchronize()
        assert status.eq(0).all()
        if self.K > 1:
            assert np.array_equal(f64(new), state)
        inside = ~np.isnan(want).all(1)
        assert (f64(y)[~inside] == 7).all()
        size = O.conv(None if self.state is None else abs(f64(self.state)), abs(f64(self.x)), abs(f64(self.w)),
                      None if self.bias is None else abs(f64(self.bias)), self.starts, False)[0][inside]
        bound = (torch.finfo(y.dtype).eps / 2 + 2e-6) * abs(want[inside]) + 1.1 * (self.K + 2) * 2.0 ** -24 * size
        assert (abs(f64(y)[inside] - want[inside]) <= bound).all()


@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("silu", [False, True])
def test_conv_kernels_and_types(K, dtype, silu):
    c = Conv([1, 0, 2, 3, 31, 32, 33, 100], K=K, dtype=dtype, seed=K)
    c.check(c.run(silu), silu)


@pytest.mark.parametrize("D", [8, 40, 504, 512, 520, 1000, 1536])
def test_conv_channels(D):
    c = Conv([5, 70, 1], D=D, seed=D, pad=16)
    c.check(c.run())


@pytest.mark.parametrize("lens", [[0], [0, 0], [1] * 100, [2, 2, 2], [64, 64], [1000], [7, 8, 9, 15, 16, 17]])
@pytest.mark.parametrize("fresh", [False, True])
def test_conv_batches(lens, fresh):
    c = Conv(lens, fresh=fresh, bias=False)
    c.check(c.run())


@pytest.mark.parametrize("before,behind", [(0, 9), (33, 0), (40, 50)])
def test_conv_rows_of_no_sequence(before, behind):
    c = Conv([10, 0, 40], before=before, behind=behind)
    want = c.run()
    c.x[:before] = float("nan")
    c.x[before + 50:] = float("nan")
    got = c.run()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    c.x[:before] = 0
    c.x[before + 50:] = 0
    c.check(got)


@pytest.mark.parametrize("lens", [[0, 1, 2, 3, 4, 50], [100]])
def test_conv_in_place(lens):
    c = Conv(lens)
    want, got = c.run(), c.run(in_place=True)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("K", [2, 3, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_conv_gives_the_bits_of_verification(K, dtype):
    n = 40
    c = Conv([n] * 3, K=K, dtype=dtype, D=72)
    y, new, _ = c.run()
    x = c.x.reshape(3, n, 72).contiguous()
    parent = torch.arange(-1, n - 1, dtype=torch.int32, device="cuda").repeat(3, 1)
    o, state = torch.empty_like(x), c.state.clone()
    B.sla_conv_verify(state, x, c.w, parent, o, bias=c.bias)
    B.sla_conv_commit(state, x, parent, parent + 1, torch.full((3,), n, dtype=torch.int32, device="cuda"), kernel_size=K)
    assert torch.equal(o.view(-1, 72), y) and torch.equal(state, new)


@pytest.mark.parametrize("starts", [[0, 10, 5, 20], [-1, 5, 6, 20], [0, 5, 10, 21], [0, 0, 0, (1 << 31) - 1]])
def test_conv_bad_starts(starts):
    c = Conv([5, 5, 10])
    c.start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    y, new, status = c.run()
    torch.cuda.synchronize()
    assert status.tolist() == [B.SLA_ERR_LENGTH] * 3 and y.eq(7).all() and new.eq(7).all()


# --------------------------------------------------------------- the inputs
def rows_case(N, kh, dk, H, dtype, seed=0, fused=True, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: (scale * torch.randn(*s, generator=g)).to(DT[dtype]).cuda()
    if fused:
        q, k, rest, ab = rand(N, 2 * kh * dk + 16 + 2 * H + 8 * (H % 4)).split([kh * dk, kh * dk, 16, 2 * H + 8 * (H % 4)], 1)
        if ab.stride(0) * ab.element_size() % 16:
            q, k = q.contiguous(), k.contiguous()
        a, b = ab[:, :H], ab[:, H:2 * H]
    else:
        q, k, a, b = rand(N, kh * dk), rand(N, kh * dk), rand(N, H), rand(N, H)
    return (q.unflatten(1, (kh, dk)), k.unflatten(1, (kh, dk)), a, b,
            torch.log(1 + 15 * torch.rand(H, generator=g)).cuda(), torch.randn(H, generator=g).cuda())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dk", [64, 128, 256])
@pytest.mark.parametrize("N,kh,H,repeat", [(1, 1, 1, 1), (7, 2, 4, 2), (33, 3, 5, 1), (300, 1, 3, 3), (1024, 8, 16, 2)])
def test_inputs(N, kh, H, repeat, dk, dtype):
    """q, k: a sum of dk squares, a root and a quotient, off by dk / 2 2^-24 + 4 2^-24 at most.  The gates: a rate of
    a few ulp (16 2^-24 of it, exponentials and logarithm included) in the exponent of alpha; beta by 2e-6."""
    q, k, a, b, a_log, dt_bias = rows_case(N, kh, dk, H, dtype, seed=N)
    out = [torch.empty(N, kh * repeat, dk, dtype=DT[dtype], device="cuda") for _ in "qk"]
    gates = [torch.empty(N, H, device="cuda") for _ in "ab"]
    B.sla_recurrent_inputs(q, k, a, b, a_log, dt_bias, *out, *gates)
    want = O.inputs(f64(q), f64(k), f64(a), f64(b), f64(a_log), f64(dt_bias), dk ** -0.5, 1e-6, repeat)
    torch.cuda.synchronize()
    for x, w in zip(out, want):
        rounds_to(x, w, (dk / 2 + 4) * 2.0 ** -24)
    rate = -np.log(np.maximum(want[2], 1e-300))
    assert (abs(f64(gates[0]) - want[2]) <= (16 * rate + 4) * 2.0 ** -24 * want[2] + 1e-37).all()
    rounds_to(gates[1], want[3], 2e-6)


def test_inputs_without_a_gate_and_extremes():
    q, k, a, b, a_log, dt_bias = rows_case(6, 2, 64, 3, "f32")
    q[0], k[1] = 0, 1e18
    a[:, 0], a[:, 1], b[:, 0], b[:, 1] = 100.0, -100.0, 100.0, -80.0
    out = [torch.empty(6, 2, 64, device="cuda") for _ in "qk"]
    alpha, beta = torch.full((6, 3), 7.0, device="cuda"), torch.full((6, 3), 7.0, device="cuda")
    B.sla_recurrent_inputs(q, k, a, None, a_log, None, *out, alpha, None, q_scale=1.0, eps=0.5)
    B.sla_recurrent_inputs(q, k, None, b, None, None, *out, None, beta, q_scale=1.0, eps=0.5)
    want = O.inputs(f64(q), f64(k), f64(a), f64(b), f64(a_log), None, 1.0, 0.5)
    assert out[0][0].eq(0).all() and torch.isfinite(out[1]).all()
    rounds_to(out[0], want[0], 40 * 2.0 ** -24)
    rounds_to(out[1], want[1], 40 * 2.0 ** -24)
    assert (abs(f64(alpha) - want[2]) <= 1e-6).all() and alpha[:, 1].eq(1).all() and (alpha >= 0).all()
    rounds_to(beta, want[3], 1e-5)  # exp2 of an argument of 115, itself rounded: 115 2^-24 = 7e-6


# ----------------------------------------------------------------- the norm
@pytest.mark.parametrize("x32,dtype", [(True, "bf16"), (False, "bf16"), (True, "f32"), (False, "f32")])
@pytest.mark.parametrize("gate", ["none", "silu", "sigmoid"])
@pytest.mark.parametrize("N,H,dv", [(1, 1, 16), (5, 3, 48), (9, 2, 80), (17, 4, 128), (3, 5, 256), (2, 3, 400), (3, 1, 1024),
                                    (2, 2, 640), (700, 16, 32), (65, 16, 64)])
def test_norm(N, H, dv, gate, x32, dtype):
    """A sum of dv squares, a root, a quotient, the gate (2e-6) and four products in fp32."""
    g = torch.Generator().manual_seed(dv)
    x = torch.randn(N, H, dv, generator=g).to(torch.float32 if x32 else DT[dtype]).cuda()
    z = torch.randn(N, H * dv + 16, generator=g).to(DT[dtype]).cuda()[:, :H * dv].unflatten(1, (H, dv))
    w = torch.randn(dv, generator=g).cuda() if dv != 48 else None
    y = torch.empty(N, H, dv, dtype=DT[dtype], device="cuda")
    B.sla_gated_norm(x, None if gate == "none" else z, w, y, gate=gate, eps=1e-5)
    rounds_to(y, O.gated_norm(f64(x), f64(z), f64(w), 1e-5, gate), (dv / 2 + 8) * 2.0 ** -24 + 2e-6)


@pytest.mark.parametrize("over", ["x", "z"])
def test_norm_in_place(over):
    x, z = torch.randn(50, 4, 80, device="cuda"), torch.randn(50, 4, 80, device="cuda")
    w, y = torch.randn(80, device="cuda"), torch.empty(50, 4, 80, device="cuda")
    B.sla_gated_norm(x, z, w, y)
    mine = x if over == "x" else z
    B.sla_gated_norm(x, z, w, mine)
    assert torch.equal(mine, y)


def test_norm_of_zeros_and_large_gates():
    x, z = torch.zeros(2, 1, 16, device="cuda"), torch.zeros(2, 1, 16, device="cuda")
    x[1], z[0], z[1, 0, 0], z[1, 0, 1] = 1.0, 3.0, -200.0, 200.0
    y = torch.empty_like(x)
    B.sla_gated_norm(x, z, None, y, eps=0.0)
    assert torch.isnan(y[0]).all()  # 0 / 0, as the formula has it
    B.sla_gated_norm(x, z, None, y, eps=1e-6)
    assert y[0].eq(0).all() and y[1, 0, 0] == 0 and abs(float(y[1, 0, 1]) - 200) < 1e-3


def test_no_rows():
    e = lambda *s: torch.empty(*s, device="cuda")
    B.sla_gated_norm(e(0, 2, 16), e(0, 2, 16), None, e(0, 2, 16))
    B.sla_recurrent_inputs(e(0, 2, 64), e(0, 2, 64), e(0, 2), e(0, 2), e(2), None, e(0, 2, 64), e(0, 2, 64), e(0, 2), e(0, 2))
    start, state = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.randn(2, 3, 8, device="cuda")
    new = torch.empty_like(state)
    B.sla_conv_prefill(e(0, 8), e(8, 4), start, e(0, 8), new, conv_state=state)
    assert torch.equal(new, state)
    state = torch.randn(2, 4, 64, 32, device="cuda")
    new = torch.empty_like(state)
    q, v = e(0, 2, 64), e(0, 4, 32)
    B.sla_prefill(q, q, v, e(0, 4), e(0, 4), start, e(0, 4, 32), new, state=state, workspace=B.prefill_workspace(q, v, 2))
    assert torch.equal(new, state)


# ------------------------------------------------------- a layer, end to end
class Layer:
    """A recurrent layer between its projections: rows of q | k | v | gate | a | b in, gated rows out."""

    def __init__(self, dtype, H=4, kh=2, dk=64, dv=48, K=4, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dt, self.H, self.kh, self.dk, self.dv, self.K = DT[dtype], H, kh, dk, dv, K
        self.D = 2 * kh * dk + H * dv
        self.taps = (0.5 * torch.randn(self.D, K, generator=g)).cuda()
        self.a_log, self.dt_bias = torch.log(1 + torch.rand(H, generator=g)).cuda(), torch.randn(H, generator=g).cuda()
        self.weight = (1 + 0.1 * torch.randn(dv, generator=g)).cuda()
        self.width = self.D + H * dv + 2 * H

    def split(self, row):
        return row.split([self.D, self.H * self.dv, self.H, self.H], 1)

    def run(self, row, start, conv, state):
        """Gated outputs; conv and state advance in place."""
        x, z, a, b = self.split(row)
        T, H, kh, dk, dv = row.shape[0], self.H, self.kh, self.dk, self.dv
        e = lambda *s, dt=self.dt: torch.empty(*s, dtype=dt, device="cuda")
        u = e(T, self.D)
        B.sla_conv_prefill(x, self.taps, start, u, conv, conv_state=conv)
        q, k, v = u.split([kh * dk, kh * dk, H * dv], 1)
        qn, kn, alpha, beta = e(T, kh, dk), e(T, kh, dk), e(T, H, dt=torch.float32), e(T, H, dt=torch.float32)
        B.sla_recurrent_inputs(q.unflatten(1, (kh, dk)), k.unflatten(1, (kh, dk)), a, b, self.a_log, self.dt_bias, qn, kn,
                               alpha, beta)
        o, v = e(T, H, dv), v.unflatten(1, (H, dv))
        B.sla_prefill(qn, kn, v, alpha, beta, start, o, state, state=state,
                      workspace=B.prefill_workspace(qn, v, len(start) - 1))
        y = e(T, H, dv)
        B.sla_gated_norm(o, z.unflatten(1, (H, dv)), self.weight, y)
        return y

    def exact(self, row, starts, conv, state):
        x, z, a, b = (f64(t) for t in self.split(row))
        T, H, kh, dk, dv = row.shape[0], self.H, self.kh, self.dk, self.dv
        u, conv = O.conv(conv, x, f64(self.taps), None, starts)
        q, k, v = np.split(u, [kh * dk, 2 * kh * dk], 1)
        qn, kn, alpha, beta = O.inputs(q.reshape(T, kh, dk), k.reshape(T, kh, dk), a, b, f64(self.a_log), f64(self.dt_bias),
                                       dk ** -0.5, 1e-6)
        o, state = O.prefill(state, qn, kn, v.reshape(T, H, dv), alpha, beta, starts)
        return O.gated_norm(o, z.reshape(T, H, dv), f64(self.weight), 1e-6, "silu"), conv, state


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_layer_over_prompts_and_then_tokens(dtype):
    """Prompts of four sequences, then three steps of one token each, all steps captured in graphs that share
    their buffers: outputs and states of the whole as the oracle has them.  fp32 to 1e-5 of the largest value at
    four times the sums' length (four operators); bf16 rounds u, q, k, o and y, each by 2^-8 of its size: 2^-8 sqrt(5)
    of the norm of rows of 48 values if independent, bounded by their sum, 5 x 2^-8."""
    L = Layer(dtype)
    lens, steps = [70, 1, 0, 129], 3
    starts = starts_of(lens)
    g = torch.Generator().manual_seed(5)
    rows = [torch.randn(n + steps, L.width, generator=g).to(L.dt) for n in lens]
    conv, state = torch.zeros(4, L.K - 1, L.D, device="cuda"), torch.zeros(4, L.H, L.dk, L.dv, device="cuda")
    ys = [L.run(torch.cat([r[:n] for r, n in zip(rows, lens)]).cuda(), torch.from_numpy(starts).cuda(), conv, state)]
    one = torch.arange(5, dtype=torch.int32, device="cuda")
    row = torch.empty(4, L.width, dtype=L.dt, device="cuda")
    warm = conv.clone(), state.clone()
    row.zero_()
    L.run(row, one, *warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = L.run(row, one, conv, state)
    for t in range(steps):
        row.copy_(torch.stack([r[n + t] for r, n in zip(rows, lens)]))
        graph.replay()
        ys.append(y.clone())
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        whole = rows[b].cuda()
        want, wconv, wstate = L.exact(whole, np.array([0, n + steps], np.int32), None, None)
        got = torch.cat([ys[0][starts[b]:starts[b + 1]]] + [s[b:b + 1] for s in ys[1:]])
        assert np.array_equal(f64(conv[b]), wconv[0])
        tol = 4e-5 if dtype == "f32" else 5 * 2.0 ** -8
        for x, w in ((f64(got), want), (f64(state[b]), wstate[0])):
            assert np.linalg.norm(x - w) <= tol * np.linalg.norm(w), np.linalg.norm(x - w) / np.linalg.norm(w)

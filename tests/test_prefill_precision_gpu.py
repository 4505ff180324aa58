"""What fp32 values keep on their way through sla_prefill's matrix products: calls
arranged so that an output is one value, or one product of two, whose bits are
known."""
import pytest
import torch

from prompt_util import Prompt, f64

pytestmark = pytest.mark.gpu

N = 60  # tokens: one chunk, distinct one-hot keys of 64


def near_ties(shape, seed, lo=120, hi=134):
    """fp32 values a few of their last bits above or below the middle between two bf16."""
    g = torch.Generator().manual_seed(seed)
    r = lambda a, b: torch.randint(a, b, shape, generator=g)
    off = 1 << r(0, 5)
    low = torch.where(r(0, 2) == 1, 0x8000 + off, 0x8000 - off)
    return (r(lo, hi) << 23 | r(0, 128) << 16 | low).int().view(torch.float32).cuda()


def one_chunk(dtype="bf16", heads=2, dv=32, batch=1, **gates):
    """Sequences of N tokens whose keys are e_0, e_1, .. of 64."""
    p = Prompt([N] * batch, heads=heads, dk=64, dv=dv, dtype=dtype, **gates)
    p.k.copy_(torch.eye(64)[:N].repeat(batch, 1)[:, None].expand_as(p.k))
    return p


ONES, ZEROS = (lambda T, H, g: torch.ones(T, H)), (lambda T, H, g: torch.zeros(T, H))


@pytest.mark.parametrize("heads,dv,batch", [(2, 32, 1), (16, 128, 3)])  # 16 and 32 columns to a workgroup
def test_bf16_outputs_are_the_state_rounded_once(heads, dv, batch):
    p = one_chunk(heads=heads, dv=dv, batch=batch, alpha=ONES, beta=ZEROS)
    p.state = near_ties((batch, heads, 64, dv), 1)
    p.q.copy_(p.k)
    out, state, _ = p.run()
    assert torch.equal(state, p.state)
    assert torch.equal(out.view(batch, N, heads, dv).transpose(1, 2), p.state[:, :, :N].bfloat16())


@pytest.mark.parametrize("heads,dv,batch", [(2, 32, 1), (16, 128, 3)])
def test_bf16_outputs_are_the_corrected_values_rounded_once(heads, dv, batch):
    x = near_ties((N * batch, heads), 2)
    p = one_chunk(heads=heads, dv=dv, batch=batch, fresh=True, alpha=ONES, beta=lambda T, H, g: x)
    p.v.fill_(1.0)
    p.q.copy_(p.k)
    out, state, _ = p.run()
    assert torch.equal(out, x.bfloat16()[..., None].expand_as(out))
    assert torch.equal(state[:, :, :N], x.view(batch, N, heads).transpose(1, 2)[..., None].expand(-1, -1, -1, dv))


def test_bf16_outputs_are_the_decays_rounded_once():
    x = near_ties((N, 2), 3, lo=110, hi=127)
    p = one_chunk(fresh=True, alpha=lambda T, H, g: x, beta=ONES)
    p.v.fill_(1.0)
    p.q[1:].copy_(p.k[:-1])  # each looks for the token before it
    p.q[0] = 0
    out, _, _ = p.run()
    assert torch.equal(out[1:], x[1:].bfloat16()[..., None].expand_as(out[1:])) and out[0].eq(0).all()


WORST = [1 + 2.0 ** -7 - 2.0 ** -23, 1 + 2.0 ** -8 - 2.0 ** -23, 1 + 2.0 ** -8 + 2.0 ** -16 + 2.0 ** -23, 2 - 2.0 ** -23, 1.7]


@pytest.mark.parametrize("x", WORST)
@pytest.mark.parametrize("y", WORST)
@pytest.mark.parametrize("sign", [1, -1])
def test_a_product_of_fp32_values_keeps_24_bits(x, y, sign):
    """Left out of a product is 2^-24 of it, and the sum of the six others rounds five times, half of 2^-23 of it
    each: 6 x 2^-24.  (Planes that are cut lose 2^-21 = 8 x 2^-24 of the first value's square by themselves.)"""
    x, y = torch.tensor([sign * x, y]).tolist()
    unit = 2.0 ** -24
    p = one_chunk("f32", alpha=ONES, beta=ZEROS)  # Q H
    p.state.fill_(x)
    p.q.copy_(p.k * y)
    assert abs(f64(p.run()[0]) - x * y).max() <= 6 * unit * abs(x * y)
    p = one_chunk("f32", fresh=True, alpha=ONES, beta=ONES)  # (Q K^T) U, and K^T U with a key of 1
    p.v.fill_(x)
    p.q.copy_(p.k * y)
    out, state, _ = p.run()
    assert abs(f64(out) - x * y).max() <= 6 * unit * abs(x * y) and abs(f64(state[:, :, :N]) - x).max() == 0
    # K H of a single key, then K^T U with it: two products in a row, added to H in eight roundings at most
    p = one_chunk("f32", alpha=ONES, beta=ONES)
    p.state.fill_(x)
    p.k[1:] = 0
    p.k[0, :, 0] = y / 2
    p.v.zero_()
    p.q.zero_()
    state, part = f64(p.run()[1])[:, :, 0], abs(x * y * y / 4)
    assert abs(state - (x - x * y * y / 4)).max() <= unit * (12 * part + 8 * (abs(x) + part))


@pytest.mark.parametrize("value", [3.3895e38, 3.396e38, -3.396e38])
def test_the_largest_values(value):
    """Values that round to the largest bf16 are finite in a chunk as they are token by token."""
    p = one_chunk("f32", fresh=True, alpha=ONES, beta=lambda T, H, g: torch.full((T, H), 0.5))
    p.v.fill_(value)
    p.q.copy_(p.k)
    p.check(p.run())
    assert p.workspace() is not None

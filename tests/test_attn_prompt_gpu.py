"""A prompt as a batch of 64-node chains that share one page-table row, chunk c
behind 64 c committed rows: appended together, then attended together."""
import numpy as np
import pytest
import torch

from attn_util import Case, rounded_bound
from oracle import attention as O
from paper_2607_16673_amd import binding as B
from test_attn_gpu import check_verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,page,hq,hkv,tokens", [(64, 16, 4, 2, 300), (128, 64, 8, 2, 640), (256, 256, 2, 1, 65)])
def test_prompt(dtype, D, page, hq, hkv, tokens):
    chunks = -(-tokens // 64)
    c = Case([chunks * 64 - 64], 64, hq, hkv, D, page, dtype, chain=True, seed=D)
    q, k, v = (c.values((chunks, 64, h, D)) for h in (hq, hkv, hkv))
    c.B, c.lens = chunks, np.arange(chunks, dtype=np.int32) * 64
    c.table = np.tile(c.table, (chunks, 1))
    c.parent = np.tile(np.arange(-1, 63, dtype=np.int32), (chunks, 1))
    rope = c.rng.uniform(-1, 1, (chunks * 64, D // 2)).astype(np.float32)
    w = [(1 + 0.3 * c.rng.standard_normal(D)).astype(np.float32) for _ in "qk"]
    want = O.append(q, k, v, c.parent, c.table, c.lens, c.k, c.v, q_norm=w[0], k_norm=w[1], eps=1e-6, rope=rope)
    dq, dk, dv, kc, vc = map(c.dev, (q, k, v, c.k, c.v))
    par, tab, ln = map(c.dev, (c.parent, c.table, c.lens))
    turned, out, st = torch.empty_like(dq), torch.full_like(dq, float("nan")), torch.full((2, chunks), 7, device="cuda").int()
    f32 = lambda x: torch.from_numpy(x).cuda()
    B.sla_attn_append(dq, dk, dv, par, tab, ln, turned, kc, vc, q_norm=f32(w[0]), k_norm=f32(w[1]), rope=f32(rope),
                      status=st[0], topology="chain")
    longest = int(c.lens.max())
    B.sla_attn_verify(turned, kc, vc, par, tab, ln, out, max_len=longest, status=st[1], topology="chain",
                      workspace=B.attn_workspace(turned, kc, tab, max_len=longest))
    assert not st.any()
    for got, ref in zip((turned, kc), want):
        assert np.all(np.abs(got.float().cpu().numpy() - ref) <= rounded_bound(ref, dtype))
    np.testing.assert_array_equal(vc.float().cpu().numpy(), want[2])
    # attention over what the cache now holds
    c.q, c.k, c.v = (t.float().cpu().numpy() for t in (turned, kc, vc))
    check_verify(c, out.float().cpu().numpy())

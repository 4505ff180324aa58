"""Out-of-range writes of the attention calls: every buffer of append, verify,
commit and page copy between guard bands, at ragged shapes and through both ways
of dividing the keys; inputs that are only read stay as they were."""
import numpy as np
import pytest
import torch

from attn_util import TORCH, Case, path_of
from paper_2607_16673_amd import binding as B
from test_attn_spans_gpu import LONG, wide
from test_canary_gpu import Guarded

pytestmark = pytest.mark.gpu

SHAPES = [  # lengths, n, q heads, kv heads, D, page
    ([0], 1, 1, 1, 64, 16), ([15, 700, 3], 17, 6, 2, 64, 16), ([1, 129, 0, 64], 33, 3, 3, 128, 32),
    ([255, 30], 64, 8, 1, 256, 256), ([400, 31, 90], 5, 10, 2, 256, 64), ([1000] + [5] * 600, 1, 2, 1, 64, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=["%dx%d_h%d_%d_D%d_p%d" % ((len(s[0]),) + s[1:]) for s in SHAPES])
def test_calls_stay_in_bounds(shape, equal, dtype):
    lens, n, hq, hkv, D, page = shape
    c = Case(lens, n, hq, hkv, D, page, dtype, layers=2, seed=n)
    if equal:
        c = wide(c)
    dt, G = TORCH[dtype], Guarded()
    dev = lambda x, ro=True: G.make(x.shape, dt if x.dtype == np.float32 else torch.int32,
                                    torch.from_numpy(np.ascontiguousarray(x)), ro)
    path, acc = path_of(c.rng, c.parent)
    q, k, v = (dev(c.values((c.B, n, h, D))) for h in (hq, hkv, hkv))
    par, tab, ln, path, acc = map(dev, (c.parent, c.table, c.lens, path, acc))
    kc, vc = dev(c.k, False), dev(c.v, False)
    f32 = lambda *s: G.make(s, torch.float32, torch.rand(*s), True)
    wq, wk, rope = f32(D), f32(D), f32(max(lens) + n, D // 2)
    turned, out = (G.make((c.B, n, hq, D), dt) for _ in "qo")
    st, new = [G.make((c.B,), torch.int32) for _ in range(3)], G.make((c.B,), torch.int32)
    max_len = LONG if equal else max(lens)
    B.sla_attn_append(q, k, v, par, tab, ln, turned, kc[1], vc[1], q_norm=wq, k_norm=wk, rope=rope, status=st[0])
    G.check("append")
    ws = B.attn_workspace(turned, kc[1], tab, max_len=max_len)
    if ws is not None:
        ws = G.make(tuple(ws.shape), torch.uint8)
    B.sla_attn_verify(turned, kc[1], vc[1], par, tab, ln, out, max_len=max_len, workspace=ws, status=st[1])
    G.check("verify")
    B.sla_attn_commit(kc, vc, par, path, acc, tab, ln, new_len=new, status=st[2])
    G.check("commit")
    assert not torch.stack(st).any() and new.tolist() == (ln + acc).tolist()
    src = dev(np.array([0, c.pages - 1], np.int32))
    dst, rows = dev(np.array([1, 2], np.int32)), dev(np.array([page, 3], np.int32))
    assert c.pages > 3
    B.sla_page_copy(kc, vc, src, dst, rows=rows, status=G.make((2,), torch.int32))
    G.check("page copy")

"""Statuses of small drafts: fewer query heads times nodes than a wave of the
joining kernel has rows, so that neighbouring sequences share one.  Each
sequence is told of its own error, and of no other's, whichever way the keys
are divided and however many groups of lanes join a row."""
import numpy as np
import pytest
import torch

from attn_util import Case, verify_bound
from oracle import attention as O
from paper_2607_16673_amd import binding as B
from test_attn_gpu import run_verify
from test_attn_spans_gpu import LONG, wide

pytestmark = pytest.mark.gpu


def spoil(c, far):
    """Every other sequence at first, then neighbours, spoiled in turn: (statuses, parent, table, lens)."""
    want = np.zeros(c.B, np.int32)
    parent, table, lens = c.parent.copy(), c.table.copy(), c.lens.copy()
    for b in range(c.B):
        what = (b // 2 if b % 2 else 3) if b < c.B // 2 else b
        if what % 4 == 0:
            parent[b, 0], want[b] = -2, B.SLA_ERR_TOPOLOGY
        elif what % 4 == 1:
            lens[b], want[b] = (-1, far)[what // 4 % 2], B.SLA_ERR_LENGTH
        elif what % 4 == 2:
            table[b, what % (int(lens[b] + c.n - 1) // 16 + 1)], want[b] = c.pages, B.SLA_ERR_PAGE
    return want, parent, table, lens


# batches that one, two, and all groups of lanes join
@pytest.mark.parametrize("count", [3, 20, 100, 300])
@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,hq,hkv", [(1, 1, 1), (1, 2, 2), (1, 3, 1), (3, 1, 1), (2, 1, 1)])
def test_neighbours_keep_their_statuses(n, hq, hkv, D, equal, count):
    lens = [(b * 61 + 17) % 400 for b in range(count)]
    c = Case(lens, n, hq, hkv, D, 16, "bf16", seed=count)
    if equal:
        c = wide(c)
    want, parent, table, lens = spoil(c, LONG + 1)
    st = torch.full((count,), 7, dtype=torch.int32, device="cuda")
    y = run_verify(c, status=st, parent=parent, table=table, lens=lens, max_len=LONG if equal else 0)
    assert st.tolist() == want.tolist()
    ok = want == 0
    o, a = O.verify(c.q[ok], c.k, c.v, c.parent[ok], c.table[ok], c.lens[ok])
    assert np.all(np.abs(y[ok] - o) <= verify_bound(o, a, "bf16"))

"""Attention over batches long enough that a workgroup ends one sequence and
begins the next.  That goes by the promised length, which stays far above the
lengths here: parts that end anywhere in a sequence, on its first tile and on
its last, sequences of one tile among them, for every form of a workgroup."""
import numpy as np
import pytest
import torch

from attn_util import Case, verify_bound
from oracle import attention as O
from paper_2607_16673_amd import binding as B
from test_attn_gpu import check_verify, run_verify

pytestmark = pytest.mark.gpu
LONG = 1 << 19


def wide(c):
    """A page table with room for the promise."""
    c.table = np.concatenate([c.table, np.full((c.B, LONG // c.page + 4 - c.table.shape[1]), 1 << 30, np.int32)], 1)
    return c


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,G", [(1, 1), (1, 8), (7, 4), (16, 3), (8, 8), (23, 3), (64, 2), (64, 4), (64, 5)])
def test_forms(dtype, D, n, G):
    c = wide(Case([300, 0, 1, 700, 40, 0, 127, 128, 129, 63], n, 2 * G, 2, D, 16, dtype, seed=n * G, fill=np.nan))
    st = torch.full((c.B,), 7, dtype=torch.int32, device="cuda")
    check_verify(c, run_verify(c, max_len=LONG, status=st))
    assert not st.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["even", "short", "one long", "rising", "many"])
@pytest.mark.parametrize("hkv", [1, 5, 48])
def test_lengths(dtype, kind, hkv):
    lens = {"even": [515] * 12, "short": [0, 1, 2] * 5, "one long": [9, 6000, 3], "rising": list(range(0, 900, 29)),
            "many": [k * 37 % 400 for k in range(600 if hkv == 1 else 60)]}[kind]
    c = wide(Case(lens, 2, hkv, hkv, 64, 64, dtype, seed=len(lens)))
    check_verify(c, run_verify(c, max_len=LONG))


@pytest.mark.parametrize("count", [3, 70])
def test_errors(count):
    """Sequences with bad data among good ones that share their workgroups."""
    rng = np.random.default_rng(count)
    c = wide(Case(rng.integers(0, 900, count), 5, 4, 2, 64, 16, "f32", seed=count))
    want = np.zeros(count, np.int32)
    parent, table, lens = c.parent.copy(), c.table.copy(), c.lens.copy()
    for b in rng.permutation(count)[:max(count // 3, 2)]:
        what = int(rng.integers(4))
        if what == 0:
            parent[b, 3], want[b] = 4, B.SLA_ERR_TOPOLOGY
        elif what == 1:
            lens[b], want[b] = (-5, LONG + 1)[b % 2], B.SLA_ERR_LENGTH
        else:
            table[b, int(rng.integers((int(lens[b]) + 4) // 16 + 1))] = (-1, c.pages)[b % 2]
            want[b] = B.SLA_ERR_PAGE
    st = torch.full((count,), 7, dtype=torch.int32, device="cuda")
    y = run_verify(c, status=st, parent=parent, table=table, lens=lens, max_len=LONG)
    assert st.tolist() == want.tolist()
    ok = want == 0
    o, a = O.verify(c.q[ok], c.k, c.v, c.parent[ok], c.table[ok], c.lens[ok])
    assert np.all(np.abs(y[ok] - o) <= verify_bound(o, a, "f32"))


@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_one_sequences_infinities_do_not_reach_the_next(value):
    c = wide(Case([200, 90, 310, 5], 6, 4, 2, 128, 16, "bf16", fill=value))
    c.parent[:] = [-1, 0, 0, 1, 2, 3]
    want = run_verify(c, max_len=LONG)
    for b in (0, 2):
        pg, row = O.row_of(c.table[b], int(c.lens[b]) + 2, 16)
        c.v[pg, :, row] = value
    got = run_verify(c, max_len=LONG)
    for b in range(4):
        clean = [0, 1, 3, 5] if b in (0, 2) else range(6)
        np.testing.assert_array_equal(got[b][clean], want[b][clean])
        if b in (0, 2):
            assert not np.isfinite(got[b][[2, 4]]).any()


def test_the_same_from_run_to_run():
    c = wide(Case([1500, 20, 700], 9, 8, 2, 128, 16, "bf16"))
    assert np.array_equal(run_verify(c, max_len=LONG), run_verify(c, max_len=LONG))

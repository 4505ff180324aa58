"""Attention where its work is divided differently: every number of query
tiles a workgroup may take, batches larger than a workgroup and of very uneven
lengths, calls without a workspace, pools whose pages lie 2 to 4 GiB in, and
tensors made on another stream."""
import numpy as np
import pytest
import torch

from attn_util import Case, verify_bound
from oracle import attention as O
from paper_2607_16673_amd import binding as B
from test_attn_gpu import check_verify, run_verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows", [15, 16, 17, 32, 33, 48, 49, 64, 65, 80, 81, 96, 112, 128, 129, 160, 161, 256, 260, 320])
def test_rows_of_a_kv_head(dtype, D, rows):
    """n nodes of G query heads: n G rows, in full and partly filled query tiles."""
    G = next(g for g in (1, 3, 4, 5, 7, 8) if rows % g == 0 and rows // g <= 64)
    c = Case([150, 1], rows // G, G * 2, 2, D, 16, dtype, seed=rows, fill=np.nan)
    check_verify(c, run_verify(c))


def uneven(rng, count, top):
    """Mostly short lengths, a few long ones, zeros and a run of equal ones."""
    lens = rng.integers(0, 40, count)
    lens[rng.integers(0, count, max(count // 50, 1))] = rng.integers(top // 2, top + 1, max(count // 50, 1))
    lens[rng.integers(0, count, max(count // 10, 1))] = 0
    lens[-1] = top
    return lens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count,n", [(1, 1), (2, 1), (63, 2), (64, 1), (65, 1), (255, 1), (256, 1), (257, 3), (513, 1), (700, 1)])
def test_uneven_batches(dtype, count, n):
    """Sequences' shares of the work, over batches of less and more sequences than
    a workgroup has threads."""
    c = Case(uneven(np.random.default_rng(count), count, 2500), n, 2, 1, 64, 32, dtype, seed=count)
    st = torch.full((count,), 7, dtype=torch.int32, device="cuda")
    check_verify(c, run_verify(c, status=st))
    assert not st.any()


@pytest.mark.parametrize("lens,max_len", [([9000] + [1] * 600, 0), ([0] * 400 + [4000] * 3, 0), ([7] * 300, 100000)])
def test_one_long_sequence_among_many(lens, max_len):
    c = Case(lens, 1, 4, 2, 64, 16, "bf16", seed=2)
    check_verify(c, run_verify(c, max_len=max_len))


@pytest.mark.parametrize("count", [3, 300])
def test_errors_in_every_part(count):
    """Bad lengths, pages and drafts scattered over a batch of uneven lengths: each
    is reported, all others are right."""
    rng = np.random.default_rng(count)
    c = Case(uneven(rng, count, 2500), 4, 2, 1, 64, 16, "f32", seed=count)
    want = np.zeros(count, np.int32)
    parent, table, lens = c.parent.copy(), c.table.copy(), c.lens.copy()
    for b in rng.permutation(count)[:max(count // 3, 2)]:
        what = int(rng.integers(4))
        if what == 0:
            parent[b, 2], want[b] = 3, B.SLA_ERR_TOPOLOGY
        elif what == 1:
            lens[b], want[b] = -1 - int(rng.integers(1000)), B.SLA_ERR_LENGTH
        else:
            last = (int(lens[b]) + 3) // 16
            table[b, 0 if what == 2 else int(rng.integers(last + 1))] = (-1, c.pages)[b % 2]
            want[b] = B.SLA_ERR_PAGE
    st = torch.full((count,), 7, dtype=torch.int32, device="cuda")
    y = run_verify(c, status=st, parent=parent, table=table, lens=lens, max_len=2500)
    assert st.tolist() == want.tolist()
    ok = want == 0
    o, a = O.verify(c.q[ok], c.k, c.v, c.parent[ok], c.table[ok], c.lens[ok])
    assert np.all(np.abs(y[ok] - o) <= verify_bound(o, a, "f32"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_workspace_for_one_tile(dtype):
    c = Case([0, 3, 7], 5, 4, 2, 64, 16, dtype, fill=np.nan)
    q, k, tab = c.dev(c.q), c.dev(c.k), c.dev(c.table)
    assert B.attn_workspace(q, k, tab, max_len=11) is None
    st = torch.full((3,), 7, dtype=torch.int32, device="cuda")
    check_verify(c, run_verify(c, max_len=11, status=st))
    assert not st.any()


@pytest.mark.parametrize("D,page", [(128, 64), (256, 256)])
def test_pages_between_2_and_4_gib(D, page):
    """Offsets with the sign bit of 32 set, in the cache's bytes and in its elements."""
    hkv, n = 2, 3
    each = hkv * page * D * 2
    pages = ((9 << 30) >> 1) // each + 3
    small = Case([4 * page - 2, 9], n, 4, hkv, D, page, "bf16", spare=0)
    spots = [(2 << 30) // each + 1, (3 << 30) // each, (4 << 30) // each - 1, (4 << 30) // each, 0, 1, pages - 1]
    assert small.pages <= len(spots)
    big = [torch.zeros(pages, hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    at = torch.tensor(spots[:small.pages], device="cuda")
    big[0][at], big[1][at] = small.dev(small.k), small.dev(small.v)
    table = np.array([[spots[p] if p < small.pages else -1 for p in row] for row in small.table], np.int32)
    q, par, tab, ln = small.dev(small.q), small.dev(small.parent), small.dev(table), small.dev(small.lens)
    out = torch.empty_like(q)
    B.sla_attn_verify(q, *big, par, tab, ln, out, max_len=4 * page,
                      workspace=B.attn_workspace(q, big[0], tab, max_len=4 * page))
    check_verify(small, out.float().cpu().numpy())
    kn, vn = small.values((2, n, hkv, D)), small.values((2, n, hkv, D))
    _, rk, rv = O.append(small.q, kn, vn, small.parent, small.table, small.lens, small.k, small.v)
    B.sla_attn_append(q, small.dev(kn), small.dev(vn), par, tab, ln, out, *big)
    small.parent[:] = [-1, -1, 1]
    path, acc = np.array([[1, 2, -1]] * 2, np.int32), np.array([2, 2], np.int32)
    B.sla_attn_commit(*big, small.dev(small.parent), small.dev(path), small.dev(acc), tab, ln)
    rk, rv = (O.commit(x[None], path, acc, small.table, small.lens)[0] for x in (rk, rv))
    B.sla_page_copy(*big, at[1:2].int(), torch.tensor([spots[2] - 5], dtype=torch.int32, device="cuda"))
    for x, r in zip(big, (rk, rv)):
        np.testing.assert_array_equal(x[at].float().cpu().numpy(), r)
        np.testing.assert_array_equal(x[spots[2] - 5].float().cpu().numpy(), r[1])
        assert not x[2:spots[0]].any()


def test_tensors_of_another_stream():
    """Inputs that a side stream is still making: the call joins that stream's queue."""
    c = Case([700, 30], 4, 4, 2, 128, 16, "bf16")
    side = torch.cuda.Stream()
    q, k, v = c.dev(c.q), c.dev(c.k), c.dev(c.v)
    par, tab, ln, out = c.dev(c.parent), c.dev(c.table), c.dev(c.lens), torch.zeros_like(q)
    ws = B.attn_workspace(q, k, tab, max_len=700)
    big = torch.randn(4096, 4096, device="cuda")
    late = [torch.zeros_like(t) for t in (q, k, v)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = big
        for _ in range(30):
            x = big @ x
        for t, s in zip(late, (q, k, v)):
            t.copy_(s)
        B.sla_attn_verify(*late, par, tab, ln, out, max_len=700, workspace=ws)
    side.synchronize()
    check_verify(c, out.float().cpu().numpy())

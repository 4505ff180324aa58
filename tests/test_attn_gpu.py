"""Attention over a paged cache on the GPU against the fp64 oracle: verify,
append, commit and page copy over types, head layouts, lengths, page sizes and
drafts; rows that take no part filled with NaN and infinities; data errors;
pools past 32-bit offsets; streams and graphs."""
import numpy as np
import pytest
import torch

from attn_util import Case, path_of, rounded_bound, verify_bound
from oracle import attention as O
from paper_2607_16673_amd import binding as B

pytestmark = pytest.mark.gpu


def run_verify(c, *, max_len=None, status=None, scale=None, parent=None, table=None, lens=None, out=None):
    q, k, v = c.dev(c.q), c.dev(c.k), c.dev(c.v)
    out = torch.full_like(q, float("nan")) if out is None else out
    table = c.dev(c.table if table is None else table)
    max_len = int(c.lens.max()) if max_len is None else max_len
    ws = B.attn_workspace(q, k, table, max_len=max_len)
    if ws is not None:
        ws.fill_(0xff)  # NaN patterns: it needs no initialisation
    B.sla_attn_verify(q, k, v, c.dev(c.parent if parent is None else parent), table,
                      c.dev(c.lens if lens is None else lens), out, max_len=max_len, workspace=ws, status=status,
                      scale=scale, topology=c.topology)
    torch.cuda.synchronize()
    return out.float().cpu().numpy()


def check_verify(c, y, scale=None):
    o, a = O.verify(c.q, c.k, c.v, c.parent, c.table, c.lens, scale)
    err = np.abs(y - o)
    bound = verify_bound(o, a, c.dtype)
    assert np.all(err <= bound), (float(np.nanmax(err / bound)), int(np.isnan(y).sum()))


LENGTHS = {"empty": [0], "short": [0, 1, 5, 15, 16, 17, 31, 33], "tile": [63, 64, 65, 127, 128, 129],
           "long": [1000, 0, 2049], "even": [300] * 5}
HEADS = [(1, 1), (16, 2), (6, 2), (7, 1), (8, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lens", list(LENGTHS))
def test_verify_lengths(dtype, D, lens):
    for i, (n, page) in enumerate([(1, 16), (7, 32), (16, 16), (64, 64)]):
        c = Case(LENGTHS[lens], n, 4, 2, D, page, dtype, seed=i, fill=np.nan)
        st = torch.full((c.B,), 7, dtype=torch.int32, device="cuda")
        check_verify(c, run_verify(c, status=st))
        assert st.tolist() == [0] * c.B


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("n", [1, 2, 3, 9, 23, 33, 64])
def test_verify_heads_and_nodes(dtype, hq, hkv, n):
    c = Case([40, 0, 201], n, hq, hkv, 128, 16, dtype, seed=n, fill=np.inf)
    check_verify(c, run_verify(c))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("chain", [False, True])
def test_verify_pages_and_chains(page, chain):
    for dtype, D in (("bf16", 64), ("bf16", 256), ("f32", 128)):
        c = Case([page - 1, page, page + 1, 3 * page - 5], 12, 6, 3, D, page, dtype, chain=chain, fill=np.nan)
        check_verify(c, run_verify(c))


@pytest.mark.parametrize("max_len", [0, 30000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_split_over_long_axis(dtype, max_len):
    """Few rows behind a long cache, and short sequences beside a long one: work
    split over workgroups and joined, with and without a promise on the length."""
    c = Case([5000, 3, 0, 777], 3, 8, 1, 128, 16, dtype, seed=5)
    check_verify(c, run_verify(c, max_len=max_len))


def test_verify_scale():
    c = Case([77], 5, 4, 4, 64, 16, "f32", qstd=1.0)
    for scale in (0.0, 0.01, 0.5, -0.3):
        check_verify(c, run_verify(c, scale=scale), scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf, 3e38])
def test_verify_siblings_are_isolated(dtype, value):
    """A node whose key and value are not finite, or huge, reaches its own
    subtree only: every other node's output is as if it held zeros."""
    n, bad = 9, 3
    parent = np.array([[-1, 0, 0, 0, 1, 3, 4, 5, 2]], np.int32)
    sub = [j for j in range(n) if bad in O.root_path(parent[0], j)]
    clean = [j for j in range(n) if j not in sub]
    for lens in ([0], [50], [64], [2100]):
        c = Case(lens, n, 4, 2, 128, 16, dtype, seed=1, fill=value)
        c.parent = parent
        pg, row = O.row_of(c.table[0], lens[0] + bad, 16)
        c.k[pg, :, row] = 0
        c.v[pg, :, row] = 0
        want = run_verify(c)
        c.k[pg, :, row] = value
        c.v[pg, :, row, ::3] = value
        got = run_verify(c)
        np.testing.assert_array_equal(got[:, clean], want[:, clean])
        if not np.isfinite(value):
            assert not np.isfinite(got[:, sub][..., ::3]).any()


def test_verify_values_beyond_a_masked_infinity():
    """Visible infinities come out as infinities of their sign, not as NaN."""
    c = Case([20], 4, 2, 1, 64, 16, "f32")
    c.parent = np.array([[-1, 0, 0, 1]], np.int32)
    pg, row = O.row_of(c.table[0], 22, 16)
    c.v[pg, 0, row, 5], c.v[pg, 0, row, 6] = np.inf, -np.inf
    y = run_verify(c)
    assert np.all(y[0, 2, :, 5] == np.inf) and np.all(y[0, 2, :, 6] == -np.inf)
    assert np.isfinite(y[0, [0, 1, 3]]).all() and np.isfinite(np.delete(y[0, 2], [5, 6], axis=1)).all()


def test_verify_extreme_scores():
    """Scores of +-2e4: one key takes all the weight; nothing overflows."""
    c = Case([100], 6, 4, 2, 64, 16, "f32", qstd=3000.0)
    y = run_verify(c)
    o, _ = O.verify(c.q, c.k, c.v, c.parent, c.table, c.lens)
    # a score is off by |s| 2^-22, a weight by as much relative to itself
    assert np.abs(y - o).max() <= 2e4 * 2.0 ** -20


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_verify_is_deterministic(dtype):
    c = Case([3000, 10], 16, 8, 2, 128, 16, dtype)
    assert np.array_equal(run_verify(c), run_verify(c))


def test_verify_prompt_as_chunks():
    """A prompt as a batch of 64-node chains that share one page-table row."""
    T, page, D = 300, 32, 64
    c = Case([T], 20, 4, 2, D, page, "f32", chain=True, spare=4)
    chunks = T // 64 + 1
    need = -(-chunks * 64 // page)
    table = np.random.default_rng(0).permutation(c.pages)[:need].astype(np.int32)
    c.B, c.n, c.table = chunks, 64, np.tile(table, (chunks, 1))
    c.lens = np.arange(chunks, dtype=np.int32) * 64
    c.parent = np.tile(np.arange(-1, 63, dtype=np.int32), (chunks, 1))
    c.q = c.values((chunks, 64, 4, D))
    check_verify(c, run_verify(c))


ERRORS = {"cycle": (B.SLA_ERR_TOPOLOGY, dict(parent=(2, 5))), "below": (B.SLA_ERR_TOPOLOGY, dict(parent=(0, -2))),
          "negative": (B.SLA_ERR_LENGTH, dict(len=-1)), "past": (B.SLA_ERR_LENGTH, dict(len=1 << 20)),
          "max": (B.SLA_ERR_LENGTH, dict(len=0x7fffffff)), "page": (B.SLA_ERR_PAGE, dict(page=1 << 20)),
          "minus": (B.SLA_ERR_PAGE, dict(page=-1)), "last": (B.SLA_ERR_PAGE, dict(page=None))}


def broken(c, what):
    code, change = ERRORS[what]
    parent, table, lens = c.parent.copy(), c.table.copy(), c.lens.copy()
    if "parent" in change:
        parent[1, change["parent"][0]] = change["parent"][1]
    if "len" in change:
        lens[1] = change["len"]
    if "page" in change:
        last = (lens[1] + c.n - 1) // c.page
        table[1, last] = c.pages if change["page"] is None else change["page"]
    return code, parent, table, lens


@pytest.mark.parametrize("what", list(ERRORS))
@pytest.mark.parametrize("n", [4, 9])
def test_data_errors(what, n):
    """A sequence with bad data is reported, its cache stays as it was and its
    neighbours' results are not touched."""
    c = Case([70, 90, 20], n, 4, 2, 64, 16, "bf16")
    code, parent, table, lens = broken(c, what)
    st = torch.full((3,), 7, dtype=torch.int32, device="cuda")
    want = run_verify(c)
    got = run_verify(c, status=st, parent=parent, table=table, lens=lens, max_len=128)
    assert st.tolist() == [0, code, 0]
    np.testing.assert_array_equal(got[[0, 2]], want[[0, 2]])
    # append
    k, v, q = c.dev(c.k), c.dev(c.v), c.dev(c.q)
    kn, vn = c.values((3, n, 2, 64)), c.values((3, n, 2, 64))
    _, rk, rv = O.append(c.q, kn, vn, c.parent, c.table, c.lens, c.k, c.v)
    st.fill_(7)
    B.sla_attn_append(q, c.dev(kn), c.dev(vn), c.dev(parent), c.dev(table), c.dev(lens), torch.empty_like(q), k, v,
                      status=st)
    own = [int(p) for p in c.table[1] if p < c.pages]
    rk[own], rv[own] = c.k[own], c.v[own]
    assert st.tolist() == [0, code, 0]
    np.testing.assert_array_equal(k.float().cpu().numpy(), rk)
    np.testing.assert_array_equal(v.float().cpu().numpy(), rv)
    # commit
    if "parent" in ERRORS[what][1]:
        return
    path, acc = np.full((3, n), -1, np.int32), np.array([0, 2, 1], np.int32)
    c.parent[1] = [-1] + [0] * (n - 1)
    path[1, :2] = 0, n - 1
    path[2, 0] = 0
    k, v, st = c.dev(c.k), c.dev(c.v), torch.full((3,), 7, dtype=torch.int32, device="cuda")
    new = torch.empty(3, dtype=torch.int32, device="cuda")
    B.sla_attn_commit(k, v, c.dev(c.parent), c.dev(path), c.dev(acc), c.dev(table), c.dev(lens), new_len=new, status=st)
    assert st.tolist() == [0, code, 0] and new.tolist() == [70, int(lens[1]), 21]
    np.testing.assert_array_equal(k.float().cpu().numpy(), c.k)


def test_topology_hint_is_checked():
    c = Case([5, 6], 4, 2, 1, 64, 16, "f32", chain=True)
    c.parent[1, 3] = 0
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    run_verify(c, status=st)
    assert st.tolist() == [0, B.SLA_ERR_TOPOLOGY]


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_append(dtype, D, layout):
    for i, (n, hq, hkv, rot, norm, fused) in enumerate([
            (1, 16, 2, D, True, True), (5, 6, 3, D // 2, True, True), (64, 4, 4, D // 4, False, False),
            (9, 3, 1, 0, True, True), (16, 8, 2, 16, True, False), (7, 5, 5, D - 16, True, True)]):
        c = Case([0, 1, 15, 16, 100], n, hq, hkv, D, 16, dtype, seed=i, chain=i == 4)
        x = c.values((c.B, n, (hq + 2 * hkv) * D))
        parts = [x[..., :hq * D], x[..., hq * D:(hq + hkv) * D], x[..., (hq + hkv) * D:]]
        q, k, v = [p.reshape(c.B, n, -1, D) for p in parts]
        rope = c.rng.uniform(-1, 1, (200, rot)).astype(np.float32) if rot else None
        wq, wk = [(1 + 0.3 * c.rng.standard_normal(D)).astype(np.float32) if norm else None for _ in range(2)]
        eps = 1e-6
        want = O.append(q, k, v, c.parent, c.table, c.lens, c.k, c.v, q_norm=wq, k_norm=wk, eps=eps, rope=rope,
                        layout=layout)
        if fused:
            dq, dk, dv = [t.unflatten(2, (-1, D)) for t in c.dev(x).split([hq * D, hkv * D, hkv * D], 2)]
        else:
            dq, dk, dv = c.dev(q), c.dev(k), c.dev(v)
        out, kc, vc = torch.empty(c.B, n, hq, D, dtype=dq.dtype, device="cuda"), c.dev(c.k), c.dev(c.v)
        f32 = lambda t: None if t is None else torch.from_numpy(t).cuda()
        st = torch.full((c.B,), 7, dtype=torch.int32, device="cuda")
        B.sla_attn_append(dq, dk, dv, c.dev(c.parent), c.dev(c.table), c.dev(c.lens), out, kc, vc, q_norm=f32(wq),
                          k_norm=f32(wk), eps=eps, rope=f32(rope), layout=layout, status=st, topology=c.topology)
        assert st.tolist() == [0] * c.B
        for got, ref in zip((out, kc), want):
            err = np.abs(got.float().cpu().numpy() - ref)
            assert np.all(err <= rounded_bound(ref, dtype)), (i, float(err.max()))
        np.testing.assert_array_equal(vc.float().cpu().numpy(), want[2])


def test_append_positions_past_the_table():
    c = Case([3, 10], 4, 2, 1, 64, 16, "f32", chain=True)
    q, k = c.dev(c.q), c.dev(c.values((2, 4, 1, 64)))
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    for length, want in ((14, [0, 0]), (13, [0, B.SLA_ERR_LENGTH]), (6, [B.SLA_ERR_LENGTH] * 2)):
        B.sla_attn_append(q, k, k, c.dev(c.parent), c.dev(c.table), c.dev(c.lens), torch.empty_like(q), c.dev(c.k),
                          c.dev(c.v), rope=torch.zeros(length, 32, device="cuda"), status=st)
        assert st.tolist() == want


def test_append_zero_and_huge_rows():
    """A zero head stays zero for eps > 0; values near the type's limits do not
    turn into NaN through the norm's mean square more than fp32 makes them."""
    c = Case([0], 2, 2, 1, 64, 16, "f32")
    q = c.dev(c.q) * 0
    k = torch.full((1, 2, 1, 64), 1e18, device="cuda")
    out, kc = torch.empty_like(q), c.dev(c.k)
    w = torch.ones(64, device="cuda")
    B.sla_attn_append(q, k, k, c.dev(c.parent), c.dev(c.table), c.dev(c.lens), out, kc, c.dev(c.v), q_norm=w, k_norm=w)
    pg, _ = O.row_of(c.table[0], 0, 16)
    assert out.abs().max().item() == 0
    np.testing.assert_allclose(kc[pg, 0, :2].cpu().numpy(), 1.0, rtol=2.0 ** -21)


# ------------------------------------------------------- commit, page copy
def bits(t):
    return t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_commit(dtype, D):
    for i, (n, hkv, page, layers, chain) in enumerate([(1, 1, 16, 1, False), (16, 2, 16, 3, False), (64, 3, 32, 2, False),
                                                       (33, 5, 64, 1, True), (64, 1, 128, 1, False)]):
        c = Case([0, 1, 14, 16, 63, 100], n, hkv, hkv, D, page, dtype, seed=i, layers=layers, chain=chain, fill=np.nan)
        path, acc = path_of(c.rng, c.parent)
        if i == 4:  # a path whose rows move onto one another's places
            c.parent[:] = np.arange(-1, n - 1)
            c.parent[:, 1] = -1
            path[:], acc[:] = -1, n - 1
            path[:, :n - 1] = np.arange(1, n)
        k, v = c.dev(c.k), c.dev(c.v)
        bk, bv = bits(k), bits(v)
        new = torch.empty(c.B, dtype=torch.int32, device="cuda")
        st = torch.full((c.B,), 7, dtype=torch.int32, device="cuda")
        B.sla_attn_commit(k, v, c.dev(c.parent), c.dev(path), c.dev(acc), c.dev(c.table), c.dev(c.lens), new_len=new,
                          status=st)
        assert st.tolist() == [0] * c.B and new.tolist() == (c.lens + acc).tolist()
        np.testing.assert_array_equal(bits(k), O.commit(bk, path, acc, c.table, c.lens))
        np.testing.assert_array_equal(bits(v), O.commit(bv, path, acc, c.table, c.lens))


def test_commit_bad_paths():
    c = Case([8] * 6, 6, 1, 1, 64, 16, "f32")
    c.parent[:] = [-1, 0, 0, 1, 2, 3]
    c.parent[5] = [-1, 3, 0, -1, 2, 3]  # out of topological order
    path = np.full((6, 6), -1, np.int32)
    rows = [[0, 1, 3], [1, 3], [0, 2, 3], [0, 7], [0, 2], [3, 1]]
    for b, r in enumerate(rows):
        path[b, :len(r)] = r
    acc = np.array([3, 2, 3, 2, 9, 2], np.int32)
    k, v = c.dev(c.k), c.dev(c.v)
    st = torch.zeros(6, dtype=torch.int32, device="cuda")
    new = torch.zeros(6, dtype=torch.int32, device="cuda")
    B.sla_attn_commit(k, v, c.dev(c.parent), c.dev(path), c.dev(acc), c.dev(c.table), c.dev(c.lens), new_len=new,
                      status=st)
    assert st.tolist() == [0] + [B.SLA_ERR_PATH] * 5 and new.tolist() == [11] + [8] * 5
    good = O.commit(c.k[None], path[:1], acc[:1], c.table[:1], c.lens[:1])[0]
    np.testing.assert_array_equal(k.cpu().numpy(), good)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_copy(dtype):
    for i, (D, hkv, page, layers, m) in enumerate([(64, 1, 16, 1, 1), (128, 2, 16, 3, 7), (256, 3, 256, 1, 2),
                                                   (128, 5, 64, 2, 40)]):
        c = Case([0], 1, hkv, hkv, D, page, dtype, layers=layers, spare=2 * m + 3, seed=i)
        ids = c.rng.permutation(c.pages).astype(np.int32)
        src, dst = ids[:m].copy(), ids[m:2 * m].copy()
        rows = c.rng.integers(0, page + 1, m).astype(np.int32)
        rows[0] = page - 1
        for r in (None, rows):
            k, v = c.dev(c.k), c.dev(c.v)
            bk, bv = bits(k), bits(v)
            st = torch.full((m,), 7, dtype=torch.int32, device="cuda")
            B.sla_page_copy(k, v, c.dev(src), c.dev(dst), rows=None if r is None else c.dev(r), status=st)
            assert st.tolist() == [0] * m
            np.testing.assert_array_equal(bits(k), O.page_copy(bk, src, dst, r))
            np.testing.assert_array_equal(bits(v), O.page_copy(bv, src, dst, r))


def test_page_copy_errors():
    c = Case([0], 1, 2, 2, 64, 16, "f32", spare=9)
    src = np.array([0, c.pages, -1, 2, 3, 4, 5], np.int32)
    dst = np.array([1, 6, 6, c.pages, 7, 8, 5], np.int32)
    rows = np.array([3, 1, 1, 1, 17, -1, 16], np.int32)
    k, v = c.dev(c.k), c.dev(c.v)
    st = torch.zeros(7, dtype=torch.int32, device="cuda")
    B.sla_page_copy(k, v, c.dev(src), c.dev(dst), rows=c.dev(rows), status=st)
    P, L = B.SLA_ERR_PAGE, B.SLA_ERR_LENGTH
    assert st.tolist() == [0, P, P, P, L, L, 0]
    np.testing.assert_array_equal(k.cpu().numpy(), O.page_copy(c.k[None], src[:1], dst[:1], rows[:1])[0])


# --------------------------------------------------------- the pool's reach
def test_pool_past_32_bit_offsets():
    """Pages beyond 2^32 bytes and 2^31 elements into the pool."""
    hkv, page, D, n = 2, 64, 128, 6
    pages = (1 << 32) // (hkv * page * D * 2) + 1000
    small = Case([100, 70], n, 4, hkv, D, page, "bf16", spare=0)
    big_k = torch.zeros(pages, hkv, page, D, dtype=torch.bfloat16, device="cuda")
    big_v = torch.zeros_like(big_k)
    at = torch.tensor([pages - 1 - 7 * i for i in range(small.pages)], device="cuda")
    big_k[at], big_v[at] = small.dev(small.k), small.dev(small.v)
    table = np.where(small.table < small.pages, pages - 1 - 7 * np.minimum(small.table, small.pages), 1 << 30).astype(np.int32)
    q = small.dev(small.q)
    out = torch.empty_like(q)
    par, tab, ln = small.dev(small.parent), small.dev(table), small.dev(small.lens)
    ws = B.attn_workspace(q, big_k, tab, max_len=100)
    B.sla_attn_verify(q, big_k, big_v, par, tab, ln, out, max_len=100, workspace=ws)
    check_verify(small, out.float().cpu().numpy())
    # append, commit and copy out there
    kn, vn = small.values((2, n, hkv, D)), small.values((2, n, hkv, D))
    _, rk, rv = O.append(small.q, kn, vn, small.parent, small.table, small.lens, small.k, small.v)
    B.sla_attn_append(q, small.dev(kn), small.dev(vn), par, tab, ln, out, big_k, big_v)
    np.testing.assert_array_equal(big_k[at].float().cpu().numpy(), rk)
    path, acc = path_of(small.rng, small.parent)
    B.sla_attn_commit(big_k, big_v, par, small.dev(path), small.dev(acc), tab, ln)
    rk = O.commit(rk[None], path, acc, small.table, small.lens)[0]
    np.testing.assert_array_equal(big_k[at].float().cpu().numpy(), rk)
    ids = at.int()
    B.sla_page_copy(big_k, big_v, ids[:1].clone(), ids[1:2] - 1)
    np.testing.assert_array_equal(big_k[int(at[1]) - 1].float().cpu().numpy(), rk[0])
    assert not big_k[:1000].any()


# --------------------------------------------------------- streams, graphs
def test_calls_run_on_the_current_stream_and_in_a_graph():
    """append, verify and commit of a round from a graph on a stream of its
    own: every replay equals the eager result."""
    c = Case([500, 33, 0], 8, 8, 2, 128, 16, "bf16")
    kn, vn = c.dev(c.values((3, 8, 2, 128))), c.dev(c.values((3, 8, 2, 128)))
    path, acc = path_of(c.rng, c.parent)
    q, par, tab, ln = c.dev(c.q), c.dev(c.parent), c.dev(c.table), c.dev(c.lens)
    path, acc = c.dev(path), c.dev(acc)
    k0, v0 = c.dev(c.k), c.dev(c.v)
    k, v = k0.clone(), v0.clone()
    q2, out, new = torch.empty_like(q), torch.empty_like(q), torch.empty_like(acc)
    ws = B.attn_workspace(q, k, tab, max_len=500)
    w = torch.ones(128, device="cuda")

    def round_():
        B.sla_attn_append(q, kn, vn, par, tab, ln, q2, k, v, q_norm=w, k_norm=w)
        B.sla_attn_verify(q2, k, v, par, tab, ln, out, max_len=500, workspace=ws)
        B.sla_attn_commit(k, v, par, path, acc, tab, ln, new_len=new)

    round_()
    torch.cuda.synchronize()
    want = [x.clone() for x in (out, k, v, new)]
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        k.copy_(k0), v.copy_(v0)
        round_()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        round_()
    for _ in range(3):
        k.copy_(k0), v.copy_(v0), out.fill_(float("nan")), new.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, k, v, new), want):
            assert torch.equal(x, y)

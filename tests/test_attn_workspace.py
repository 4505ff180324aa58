"""The workspace of attention calls: room for what workgroups leave unfinished,
which the chip bounds, and not for every sequence of a large batch; and nothing
written outside it."""
import ctypes

import numpy as np
import pytest
import torch

from attn_util import Case
from paper_2607_16673_amd import binding as B
from test_attn_gpu import check_verify
from test_attn_spans_gpu import LONG, wide

WORKGROUPS = 2 * 256  # that run at once, of up to 256 rows each


def need(**o):
    f = dict(batch=1, q_heads=64, kv_heads=8, head_dim=128, n_nodes=64, qkv_dtype=B.SLA_DTYPE_BF16, topology=0,
             page_size=64, n_pages=1 << 20, max_pages=2048, max_len=0)
    s = B.SlaAttnShape(**{**f, **o})
    return B.lib().sla_attn_workspace_bytes(ctypes.byref(s))


@pytest.mark.parametrize("dtype", [B.SLA_DTYPE_BF16, B.SLA_DTYPE_F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (16, 2), (64, 8), (64, 64), (128, 1), (96, 3)])
def test_workspace_goes_by_the_chip(q_heads, kv_heads, D, dtype):
    """At most two unfinished sequences a workgroup, or those of one sequence's rows."""
    for n in (1, 7, 64):
        for max_len in (1, 100, 1000, 10000, 131072):
            # a workgroup may have fewer rows than it could: never less than half of a block of them
            rows = 2 * max(2 * WORKGROUPS * 256, n * q_heads)
            for batch in (1, 2, 63, 256, 300, 513, 2048, 16384, 65535):
                got = need(batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=D, n_nodes=n, max_len=max_len,
                           qkv_dtype=dtype)
                assert got <= rows * (D + 2) * 4 + 8 * batch + 4 * 2 * WORKGROUPS, (n, max_len, batch, got)


def test_a_long_prompt():
    """131072 tokens as 2048 chunks of 64: 16 workers a kv head and block of queries,
    two unfinished sequences each."""
    assert need(batch=2048, max_len=131072) <= 8 * 32 * 512 * 130 * 4 + 2048 * 8 + 32 * 4


GUARD = 1 << 16


def guarded(c, max_len):
    """The call with a workspace of just the size asked for, between guard bands."""
    q, k, v, tab = c.dev(c.q), c.dev(c.k), c.dev(c.v), c.dev(c.table)
    ws = B.attn_workspace(q, k, tab, max_len=max_len)
    size = 0 if ws is None else ws.numel()
    raw = torch.full((size + 2 * GUARD,), 0xa5, dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, float("nan"))
    st = torch.full((c.B,), 7, dtype=torch.int32, device="cuda")
    B.sla_attn_verify(q, k, v, c.dev(c.parent), tab, c.dev(c.lens), out, max_len=max_len,
                      workspace=raw[GUARD:GUARD + size] if size else None, status=st, topology=c.topology)
    torch.cuda.synchronize()
    assert not st.any()
    assert (raw[:GUARD] == 0xa5).all() and (raw[GUARD + size:] == 0xa5).all()
    return out.float().cpu().numpy()


LENS = {"ranges": lambda r: r.integers(0, 900, 40), "more ranges": lambda r: r.integers(0, 900, 300),
        # more sequences than that: a few, and many, that are divided
        "few long": lambda r: np.where(np.arange(700) % 90 == 7, 2000, r.integers(0, 120, 700)),
        "many long": lambda r: np.where(np.arange(700) % 9 == 7, 1800, r.integers(0, 60, 700)),
        "none long": lambda r: np.full(700, 500)}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", list(LENS))
@pytest.mark.parametrize("n,hq,hkv", [(1, 2, 1), (3, 4, 2), (9, 8, 1)])
def test_ranges_stay_inside(kind, n, hq, hkv, dtype):
    lens = LENS[kind](np.random.default_rng(n))
    if n == 9:
        lens = lens[:len(lens) * 3 // 4]
    c = Case(lens, n, hq, hkv, 64, 16, dtype, seed=n)
    check_verify(c, guarded(c, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(2, 1), (48, 48), (128, 32)])
@pytest.mark.parametrize("count", [2, 9, 17, 130])
def test_equal_parts_stay_inside(count, hq, hkv, dtype):
    """Fewer sequences than workers, and more."""
    rng = np.random.default_rng(count)
    c = wide(Case(rng.integers(0, 300 if count > 20 else 1500, count), 2, hq, hkv, 64, 64, dtype, seed=count))
    check_verify(c, guarded(c, LONG))


@pytest.mark.gpu
@pytest.mark.parametrize("spoilt", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,count,every", [(8, 140, 10), (8, 200, 29), (16, 100, 20), (16, 65, 64), (32, 40, 7)])
def test_only_long_sequences_are_divided(hkv, count, every, dtype, spoilt):
    """More sequences than twice the workgroups of a kv head: a few are far longer
    than a workgroup's even share.  With errors among the divided ones and the whole."""
    keys, want = (128 if dtype == "bf16" else 64), WORKGROUPS // hkv
    top = min(40 * want // count - 1, 20) * keys - 3  # shorter than the work that goes in equal parts
    lens = [top - b % 50 if b % every == every - 1 else b % 30 for b in range(count)]
    c = Case(lens, 1, hkv, hkv, 64, 16, dtype, seed=count)
    tiles = [-(-(l + 1) // keys) for l in lens]
    assert max(tiles) > -(-sum(tiles) // (want // 2)) and count > 2 * want
    q, k, v, tab = c.dev(c.q), c.dev(c.k), c.dev(c.v), c.dev(c.table)
    assert B.attn_workspace(q, k, tab, max_len=top).numel() == 4 * want * (66 * hkv + 1) + 8 * count
    if not spoilt:
        check_verify(c, guarded(c, top))
        return
    status = np.zeros(count, np.int32)
    parent, table, lens = c.parent.copy(), c.table.copy(), c.lens.copy()
    for b in list(range(1, count, 5)) + list(range(every - 1, count, 2 * every)):
        if b % 3 == 0:
            parent[b, 0], status[b] = 0, B.SLA_ERR_TOPOLOGY
        elif b % 3 == 1:
            table[b, int(lens[b]) // 16 // 2], status[b] = -1, B.SLA_ERR_PAGE
        else:
            lens[b], status[b] = top + 1, B.SLA_ERR_LENGTH
    st, out = torch.full((count,), 7, dtype=torch.int32, device="cuda"), torch.full_like(q, float("nan"))
    B.sla_attn_verify(q, k, v, c.dev(parent), c.dev(table), c.dev(lens), out, max_len=top, status=st,
                      workspace=B.attn_workspace(q, k, tab, max_len=top))
    assert st.tolist() == status.tolist()
    ok = status == 0
    c.q, c.parent, c.table, c.lens = c.q[ok], c.parent[ok], c.table[ok], c.lens[ok]
    check_verify(c, out.float().cpu().numpy()[ok])

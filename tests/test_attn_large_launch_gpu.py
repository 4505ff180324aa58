"""Launches of more workgroups than fit one dimension's 2^32 work-items: many
copies of many pieces, many sequences of many heads, many rows to join."""
import ctypes

import pytest
import torch

from paper_2607_16673_amd import binding as B

pytestmark = pytest.mark.gpu


def int32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def test_many_copies():
    """70000 pages: more than a launch is high."""
    m = 70000
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randperm(2 * m + 1, generator=g, device="cuda").int()
    src, dst = ids[:m].clone(), ids[m:2 * m].clone()
    rows = torch.randint(0, 17, (m,), generator=g, device="cuda", dtype=torch.int32)
    k = torch.randn(1, 2 * m + 1, 1, 16, 64, generator=g, device="cuda").bfloat16()
    v = k.flip(1)
    want = [x.clone() for x in (k, v)]
    keep = (torch.arange(16, device="cuda") < rows[:, None])[:, None, :, None]
    for x in want:
        x[0, dst.long()] = torch.where(keep, x[0, src.long()], x[0, dst.long()])
    st = torch.full((m,), 7, dtype=torch.int32, device="cuda")
    B.sla_page_copy(k, v, src, dst, rows=rows, status=st)
    assert not st.any() and torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_many_copies_of_many_pieces():
    """2^24 workgroups and more, nearly all of which have nothing to move."""
    m, layers, heads = (1 << 17) + 5, 16, 4
    k = torch.randn(layers, 3, heads, 16, 64, device="cuda").bfloat16()
    v = torch.randn(layers, 3, heads, 16, 64, device="cuda").bfloat16()
    src, dst = int32([0] * m), int32([0] * m)
    dst[-1], src[7] = 1, 99
    st = torch.full((m,), 7, dtype=torch.int32, device="cuda")
    want = [x.clone() for x in (k, v)]
    for x in want:
        x[:, 1] = x[:, 0]
    B.sla_page_copy(k, v, src, dst, status=st)
    assert int(st[7]) == B.SLA_ERR_PAGE and int(st.abs().sum()) == -B.SLA_ERR_PAGE
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def reference(q, k, v, rows):
    """q [B][1][heads][D] over rows [0, rows] of k, v [kv heads][rows][D] in 32 bits."""
    b, _, hq, d = q.shape
    hkv = k.shape[0]
    x = q.float().reshape(b, hkv, hq // hkv, d).permute(1, 0, 2, 3).reshape(hkv, -1, d)
    s = torch.bmm(x, k.float().transpose(1, 2).contiguous()) * d ** -0.5
    hide = torch.arange(k.shape[1], device="cuda") > rows.repeat_interleave(hq // hkv)[:, None]
    p = torch.softmax(s.masked_fill(hide, -torch.inf), -1)
    return torch.bmm(p, v.float()).reshape(hkv, b, hq // hkv, d).permute(1, 0, 2, 3).reshape(b, 1, hq, d)


def shared_pages(batch, hq, hkv, D, lens, pages, room=None):
    """One-token sequences that all read the same pages.  Two chosen blocks of
    sequences against the reference: bf16 weights and outputs are each off by up to
    2^-8 of values of up to max |v|."""
    k, v = (torch.randn(pages, hkv, 16, D, device="cuda").bfloat16() for _ in "kv")
    q = torch.empty(batch, 1, hq, D, dtype=torch.bfloat16, device="cuda").normal_()
    lens = int32(lens)
    table = torch.arange(room or pages, device="cuda", dtype=torch.int32).clamp(max=pages - 1).repeat(batch, 1)
    out, st = torch.full_like(q, float("nan")), torch.full((batch,), 7, dtype=torch.int32, device="cuda")
    parent = int32([-1]).repeat(batch, 1)
    B.sla_attn_verify(q, k, v, parent, table, lens, out, max_len=int(lens.max()),
                      workspace=B.attn_workspace(q, k, table, max_len=int(lens.max())), status=st)
    assert not st.any() and not out.isnan().any()
    flat = [x.transpose(0, 1).reshape(hkv, -1, D) for x in (k, v)]
    bound = float(v.abs().max()) * 2.0 ** -7
    for part in (slice(0, 64), slice(batch // 2, batch // 2 + 64), slice(batch - 64, batch)):
        err = (out[part].float() - reference(q[part], *flat, lens[part])).abs().max()
        assert float(err) <= bound


def test_many_sequences_of_many_heads():
    """65535 sequences of 257 kv heads: 1.7e7 workgroups of 256 threads."""
    shared_pages(65535, 257, 257, 64, [b % 16 for b in range(65535)], 1)


def test_many_rows_to_join():
    """1.7e7 rows, four to a workgroup of the join: the last sequence is long, and
    divided."""
    lens = [b % 60 for b in range(65535)]
    lens[-1] = lens[32768] = 3000
    shared_pages(65535, 260, 20, 256, lens, 188)


def test_rows_past_32_bits_are_refused():
    s = B.SlaAttnShape(batch=65535, q_heads=1 << 16, kv_heads=1, head_dim=64, n_nodes=1, qkv_dtype=0, topology=0,
                       page_size=16, n_pages=4, max_pages=4, max_len=0)
    assert B.lib().sla_attn_workspace_bytes(ctypes.byref(s)) == 0

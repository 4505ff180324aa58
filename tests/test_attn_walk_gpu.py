"""Attention where every workgroup walks many tiles: batches that fill the chip
several times over, with scores that rise along the keys, come in waves or stay
level, for every form of a workgroup and both ways of dividing the keys."""
import numpy as np
import pytest
import torch

from attn_util import TORCH, draft, verify_bound
from oracle import attention as O
from paper_2607_16673_amd import binding as B
from test_attn_spans_gpu import LONG

pytestmark = pytest.mark.gpu
TILE, AT_ONCE = 16384, 512  # bytes of a tile's keys; workgroups that run at once, or fewer


def offsets(kind, i, length):
    """What a row's score is raised by, from its number: up to 40 over the whole
    length, or up to 12 and down again every 400 rows."""
    return {"rising": 40.0 * i / length, "waves": 12.0 * (i % 400) / 400, "level": 0.0 * i}[kind]


class Batch:
    """A batch on the GPU over shuffled pages; rows of no sequence are NaN."""

    def __init__(self, kind, dtype, D, n, G, hkv, count, page=64, seed=0):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = TORCH[dtype]
        keys = TILE // (D * (2 if dtype == "bf16" else 4))
        blocks = -(-n * G // 256)
        each = 6 * AT_ONCE // (hkv * blocks * count) + 3
        self.lens = (each * keys + np.arange(count) * 37 % (2 * keys)).astype(np.int32)
        assert int(sum(-(-(l + n) // keys) for l in self.lens)) * hkv * blocks >= 5 * AT_ONCE
        counts = -(-(self.lens + n) // page)
        ids = rng.permutation(int(counts.sum()) + 2).astype(np.int32)
        self.table = np.full((count, counts.max()), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = ids[at:at + c]
            at += c
        self.parent = draft(rng, count, n)
        shape = (len(ids), hkv, page, D)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=dt, device="cuda") for _ in "kv")
        self.q = torch.randn(count, n, hkv * G, D, generator=g, device="cuda")
        self.q[..., 0] = 4.0
        self.q = self.q.to(dt)
        self.rows = []
        for b in range(count):
            total = int(self.lens[b]) + n
            k, v = (torch.randn(hkv, total, D, generator=g, device="cuda") for _ in "kv")
            i = torch.arange(total, device="cuda", dtype=torch.float64)
            k[..., 0] = (offsets(kind, i, total) * D ** 0.5 / 4).float()
            k, v = k.to(dt), v.to(dt)
            self.rows.append((k, v))
            pg = torch.from_numpy(self.table[b, :counts[b]]).long().cuda()
            for pool, x in ((self.k, k), (self.v, v)):
                pad = torch.full((hkv, len(pg) * page - total, D), float("nan"), dtype=dt, device="cuda")
                pool[pg] = torch.cat([x, pad], 1).view(hkv, len(pg), page, D).transpose(0, 1)

    def run(self, max_len):
        table = self.table
        if max_len == LONG:  # room for the promise
            table = np.concatenate([table, np.full((len(table), LONG // 64 + 2 - table.shape[1]), -1, np.int32)], 1)
        par, tab, ln = (torch.from_numpy(x).cuda() for x in (self.parent, np.ascontiguousarray(table), self.lens))
        ws = B.attn_workspace(self.q, self.k, tab, max_len=max_len)
        ws.fill_(0xff)
        out, st = torch.full_like(self.q, float("nan")), torch.full((len(ln),), 7, dtype=torch.int32, device="cuda")
        B.sla_attn_verify(self.q, self.k, self.v, par, tab, ln, out, max_len=max_len, workspace=ws, status=st)
        assert not st.any()
        return out

    def check(self, out, dtype):
        n, G = self.q.shape[1], self.q.shape[2] // self.k.shape[1]
        for b, (k, v) in enumerate(self.rows):
            hide = torch.zeros(n, k.shape[1], dtype=torch.bool)
            hide[:, -n:] = True
            for j in range(n):
                hide[j, [k.shape[1] - n + a for a in O.root_path(self.parent[b], j)]] = False
            hide = hide.cuda().repeat_interleave(G, 0)
            o, a, size = [], [], 0.0
            for h in range(k.shape[0]):
                q = self.q[b, :, h * G:(h + 1) * G].reshape(n * G, -1).double()
                p = torch.softmax((q @ k[h].double().t() * q.shape[1] ** -0.5).masked_fill(hide, -torch.inf), 1)
                size = max(size, float((q.abs() @ k[h].double().abs().t()).max()) * q.shape[1] ** -0.5)
                o.append((p @ v[h].double()).view(n, G, -1))
                a.append((p @ v[h].double().abs()).view(n, G, -1))
            o, a = torch.cat(o, 1).cpu().numpy(), torch.cat(a, 1).cpu().numpy()
            err, bound = np.abs(out[b].double().cpu().numpy() - o), verify_bound(o, a, dtype)
            if dtype == "f32":
                # A score whose first product is large is rounded D times at that size:
                # fp32 sums of D products are off by up to D 2^-24 sum |q k|, and weights
                # off by that much of themselves turn the output by twice as much.
                bound = bound + 2 * q.shape[1] * 2.0 ** -24 * size * a
            assert np.all(err <= bound), (b, float(np.nanmax(err / bound)), int(np.isnan(err).sum()))


FORMS = [("bf16", D, n, G) for D in (64, 128, 256) for n, G in ((1, 1), (1, 8), (7, 7), (16, 8), (50, 2), (64, 4), (40, 8))]
FORMS += [("f32", 64, n, G) for n, G in ((1, 1), (16, 1), (8, 4), (23, 2), (21, 3), (23, 3), (64, 3))]
FORMS += [("f32", D, n, G) for D in (128, 256) for n, G in ((1, 1), (8, 4), (16, 4), (23, 6))]


@pytest.mark.parametrize("kind", ["rising", "waves", "level"])
@pytest.mark.parametrize("dtype,D,n,G", FORMS)
def test_walks(dtype, D, n, G, kind):
    b = Batch(kind, dtype, D, n, G, hkv=4, count=9, seed=n * G)
    for max_len in (int(b.lens.max()), LONG):
        b.check(b.run(max_len), dtype)


@pytest.mark.parametrize("kind", ["rising", "waves"])
@pytest.mark.parametrize("dtype,D,n,G", [("bf16", 128, 1, 1), ("bf16", 256, 1, 8), ("f32", 64, 3, 2)])
def test_walks_of_more_sequences_than_workgroups(dtype, D, n, G, kind):
    """Whole sequences, one to a workgroup, for the most part."""
    b = Batch(kind, dtype, D, n, G, hkv=64, count=40, seed=5)
    for max_len in (int(b.lens.max()), LONG):
        b.check(b.run(max_len), dtype)

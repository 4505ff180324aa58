"""Performance cases of the attention layer of a hybrid target: drafted tokens
over a paged key/value cache.

A hybrid target interleaves its recurrent layers with attention layers.  In
one speculative round such a layer normalises and rotates the draft's queries
and keys and writes the draft's rows into the cache behind the committed
tokens (``append``), attends every node of the draft tree to the cache and to
its own root path (``attend``), and, once a path is accepted, moves the rows of
its nodes together behind the committed tokens (``commit``).  A sequence that
splits in two shares its full pages and copies its last one (``copy``).

A case is a dict of plain values: ``listed`` gives the fixed ones, ``draw`` one
more of the same ranges, ``prepare`` the device tensors of a case, ``run`` one
pass, ``work`` the bytes and operations a pass cannot do without, and ``exact``
the same outputs in 64 bits.

Layout.  A cache is [layers][pages][kv heads][page size][head size] for keys
and the same for values; ``page_table`` [B][pages of a sequence] names a
sequence's pages in order, ``cache_len`` [B] its committed tokens.  Node j of a
draft has the cache row cache_len + j and the position cache_len + depth(j) - 1
(a root has depth 1).  Query head h reads kv head h // (q_heads / kv_heads).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------- cases
def _attend(name, batch, n, lo, hi, *, q_heads=16, kv_heads=2, head=128, page=16, dtype="bf16", depth=5, chain=False):
    case = dict(op="attend", batch=batch, n=n, lo=lo, hi=hi, q_heads=q_heads, kv_heads=kv_heads, head=head, page=page,
                dtype=dtype, depth=depth, chain=chain, layers=1)
    return dict(name=name, **case) if name else case


def _append(name, batch, n, lo, hi, *, q_heads=16, kv_heads=2, head=128, page=16, dtype="bf16", depth=5, chain=False,
            rope=64, layout="half", norm=True, fused=True):
    case = dict(op="append", batch=batch, n=n, lo=lo, hi=hi, q_heads=q_heads, kv_heads=kv_heads, head=head, page=page,
                dtype=dtype, depth=depth, chain=chain, layers=1, rope=rope, layout=layout, norm=norm, fused=fused)
    return dict(name=name, **case) if name else case


def _commit(name, batch, n, lo, hi, *, layers=24, kv_heads=2, head=128, page=16, dtype="bf16", depth=5):
    case = dict(op="commit", batch=batch, n=n, lo=lo, hi=hi, q_heads=kv_heads, kv_heads=kv_heads, head=head, page=page,
                dtype=dtype, depth=depth, chain=False, layers=layers)
    return dict(name=name, **case) if name else case


def _copy(name, copies, *, layers=24, kv_heads=2, head=128, page=16, dtype="bf16", partial=True):
    case = dict(op="copy", copies=copies, layers=layers, kv_heads=kv_heads, head=head, page=page, dtype=dtype,
                partial=partial)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # one interactive sequence decoding one token behind a short cache: the
        # smallest call, latency only
        _attend("attend_token", 1, 1, 1000, 1000, depth=1, chain=True),
        # one interactive sequence, a 32-node tree behind a very long cache:
        # all of the work lies along one axis
        _attend("attend_long", 1, 32, 131072, 131072, page=64, depth=6),
        # plain decoding of a large batch with lengths from short to long
        _attend("attend_decode", 256, 1, 17, 16384, depth=1, chain=True),
        # batched serving: 64 sequences, 16-node trees; the ordinary load
        _attend("attend_serving", 64, 16, 512, 4096),
        # fp32 activations and sizes that fit no tile: 23-node trees, three
        # query heads a kv head, some sequences nearly empty
        _attend("attend_ragged_f32", 40, 23, 0, 3001, q_heads=12, kv_heads=4, head=64, page=32, dtype="f32", depth=6),
        # throughput serving with the largest drafts at head size 256
        _attend("attend_tree64", 64, 64, 2048, 8192, head=256, page=64, depth=8),
        # the draft of a serving round behind one fused projection: norms, a
        # rotation of half of the head, and the cache's rows
        _append("append_serving", 64, 16, 512, 4096),
        # the largest drafts with fp32 activations, pairs side by side, the
        # whole head rotated, projections of their own
        _append("append_large_f32", 256, 64, 0, 1500, head=256, page=64, dtype="f32", depth=8, rope=256,
                layout="interleaved", fused=False),
        # accepted paths of a serving round, every attention layer of a model
        # in one call
        _commit("commit_serving", 64, 16, 100, 600),
        # accepted paths of the largest drafts, many layers
        _commit("commit_large", 256, 64, 10, 150, layers=6, kv_heads=4, head=256, page=64, depth=8),
        # one sequence splits off another: the last, partly filled page of
        # every layer
        _copy("copy_fork", 1),
        # moving whole pages: sequences resumed elsewhere in the pool
        _copy("copy_pages", 512, page=64, partial=False),
    ]


MAX_FLOPS = 1.2e12
MAX_BYTES = 2.2e9


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _pool_bytes(case):
    w = 2 if case["dtype"] == "bf16" else 4
    row = 2 * case["layers"] * case["kv_heads"] * case["head"] * w
    if case["op"] == "copy":
        return row * case["page"] * (2 * case["copies"] + 3)
    return row * case["page"] * (sum(_pages(case)) + 5)


def draw(rng):
    op = rng.choices(["attend", "append", "commit", "copy"], [7, 2, 2, 1])[0]
    while True:
        dtype = rng.choices(["bf16", "f32"], [3, 1])[0]
        head = rng.choice([64, 128, 128, 256])
        page = rng.choice([16, 32, 64, 128])
        kv_heads = rng.choice([1, 2, 2, 3, 4, 8])
        if op == "copy":
            case = _copy(None, _log_int(rng, 1, 512), layers=_log_int(rng, 1, 24), kv_heads=kv_heads, head=head,
                         page=page, dtype=dtype, partial=rng.random() < 0.5)
        else:
            batch = _log_int(rng, 1, 256)
            n = 1 if rng.random() < 0.2 else _log_int(rng, 2, 64)
            hi = _log_int(rng, 16, 131072 if op == "attend" else 3000)
            lo = hi if batch == 1 or rng.random() < 0.2 else rng.randint(0, hi)
            chain = n == 1 or rng.random() < 0.25
            kw = dict(kv_heads=kv_heads, head=head, page=page, dtype=dtype, depth=n if chain else rng.randint(3, 12))
            if op == "attend":
                case = _attend(None, batch, n, lo, hi, q_heads=kv_heads * rng.choice([1, 2, 3, 4, 7, 8]), chain=chain,
                               **kw)
            elif op == "append":
                case = _append(None, batch, n, lo, hi, q_heads=kv_heads * rng.choice([1, 2, 3, 4, 7, 8]), chain=chain,
                               rope=rng.choice([0, head // 4, head // 2, head]),
                               layout=rng.choice(["half", "interleaved"]), norm=rng.random() < 0.75,
                               fused=rng.random() < 0.5, **kw)
            else:
                kw["depth"] = max(3, min(kw["depth"], 12))
                case = _commit(None, batch, max(n, 2), lo, hi, layers=_log_int(rng, 1, 24), **kw)
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and _pool_bytes(case) <= 5e9 and _plain_bytes(case) <= 1e10:
            return case


def _plain_bytes(case):
    """Scores of the plain form."""
    if case["op"] != "attend":
        return 0
    return 4 * case["batch"] * case["q_heads"] * case["n"] * (max(_lens(case)) + case["n"])


# ------------------------------------------------------------------ shapes
def _lens(case):
    """Committed tokens of each sequence: spread evenly over [lo, hi]."""
    lo, hi = case["lo"], case["hi"]
    return [lo + int((hi - lo + 1) * (((b + 1) * 0.6180339887498949) % 1.0)) for b in range(case["batch"])]


def _pages(case):
    return [-(-(l + case["n"]) // case["page"]) for l in _lens(case)]


def _paths(case):
    """Mean accepted path of a commit: between a root and the deepest node."""
    return min(case["depth"], case["n"]) / 2


def work(case):
    w = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "copy":
        rows = case["copies"] * (case["page"] if not case["partial"] else case["page"] / 2)
        return dict(bytes=int(4 * case["layers"] * case["kv_heads"] * rows * case["head"] * w), flops=0)
    B, n, D = case["batch"], case["n"], case["head"]
    qh, kh = case["q_heads"], case["kv_heads"]
    if case["op"] == "commit":
        return dict(bytes=int(4 * case["layers"] * B * _paths(case) * kh * D * w + 4 * B * n), flops=0)
    if case["op"] == "append":
        rows = B * n * (qh + 2 * kh) * D
        table = 4 * B * min(n, case["depth"]) * case["rope"]
        return dict(bytes=2 * rows * w + table + 4 * B * n, flops=6 * B * n * (qh + kh) * D)
    tokens = sum(_lens(case)) + B * n
    # a node's scores: the committed rows and, at most, the draft's
    return dict(bytes=2 * tokens * kh * D * w + 2 * B * n * qh * D * w + 4 * sum(_pages(case)) + 4 * B * n,
                flops=4 * n * qh * D * tokens)


# ------------------------------------------------------------------ inputs
def _gen(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(shape, dtype, g, std=1.0):
    """N(0, std^2) values, the outermost index in pieces: a large pool needs no fp32 copy of itself."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 26
    for i in range(0, flat.numel(), step):
        part = flat[i:i + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * std)
    return out


def _trees(case, rs):
    """Parent arrays [B][n] in topological order within the depth limit."""
    B, n = case["batch"], case["n"]
    parent = np.full((B, n), -1, np.int32)
    depth = np.ones((B, n), np.int32)
    rows = np.arange(B)
    for j in range(1, n):
        if case["chain"]:
            p = np.full(B, j - 1)
        else:
            p = rs.randint(0, j, size=B)
            deep = depth[rows, p] >= case["depth"]
            p = np.where(deep, parent[rows, p], p)  # one level up where the limit is reached
        parent[:, j] = p
        depth[:, j] = np.where(p >= 0, depth[rows, np.maximum(p, 0)], 0) + 1
    return parent


def _accepted(parent, rs):
    """Root paths of drawn nodes.  A path whose rows move onto one another's
    places is passed over, so that a pass can be repeated on its own result."""
    B, n = parent.shape
    path = np.full((B, n), -1, np.int32)
    length = np.zeros(B, np.int32)
    for b in range(B):
        for j in rs.permutation(n):
            nodes = []
            a = int(j)
            while a >= 0:
                nodes.append(a)
                a = int(parent[b, a])
            nodes.reverse()
            moved = [a for t, a in enumerate(nodes) if a != t]
            if all(a >= len(nodes) for a in moved):
                path[b, :len(nodes)] = nodes
                length[b] = len(nodes)
                break
    return path, length


def rope_table(length, dim, base=1e6):
    """cos and sin of position * base^(-2 i / dim), taken in 64 bits: [length][dim], cosines first."""
    inv = base ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    angle = torch.arange(length, dtype=torch.float64, device="cuda")[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    g = _gen(seed, "cuda")
    rs = np.random.RandomState(seed % (1 << 32))
    dt = _dtype(case)
    kh, ps, D, L = case["kv_heads"], case["page"], case["head"], case["layers"]
    st = dict(case=case)
    if case["op"] == "copy":
        m = case["copies"]
        ids = rs.permutation(2 * m + 3).astype(np.int32)
        rows = rs.randint(1, ps + 1, size=m).astype(np.int32) if case["partial"] else None
        if rows is not None and m == 1:
            rows[0] = ps // 2
        st.update(src=torch.from_numpy(ids[:m].copy()).cuda(), dst=torch.from_numpy(ids[m:2 * m].copy()).cuda(),
                  rows=None if rows is None else torch.from_numpy(rows).cuda())
        pages = 2 * m + 3
    else:
        B, n = case["batch"], case["n"]
        counts = _pages(case)
        pages = sum(counts) + 5
        ids = rs.permutation(pages).astype(np.int32)
        table = np.zeros((B, max(counts)), np.int32)
        at = 0
        for b, c in enumerate(counts):
            table[b, :c] = ids[at:at + c]
            at += c
        parent = _trees(case, rs)
        lens = _lens(case)
        st.update(parent=torch.from_numpy(parent).cuda(), page_table=torch.from_numpy(table).cuda(),
                  cache_len=torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len=max(lens),
                  status=torch.zeros(B, dtype=torch.int32, device="cuda"))
    shape = (L, pages, kh, ps, D)
    st["k_cache"], st["v_cache"] = _normal(shape, dt, g), _normal(shape, dt, g)
    if case["op"] == "attend":
        # scores of a standard deviation of 2
        st["q"] = _normal((B, n, case["q_heads"], D), dt, g, 2.0)
        st["out"] = torch.empty_like(st["q"])
        st["k_cache"], st["v_cache"] = st["k_cache"][0], st["v_cache"][0]
        if own:
            from paper_2607_16673_amd import binding
            st["workspace"] = binding.attn_workspace(st["q"], st["k_cache"], st["page_table"], max_len=st["max_len"])
    elif case["op"] == "append":
        qh = case["q_heads"]
        if case["fused"]:
            x = _normal((B, n, (qh + 2 * kh) * D), dt, g)
            parts = x.split([qh * D, kh * D, kh * D], dim=2)
        else:
            parts = [_normal((B, n, h * D), dt, g) for h in (qh, kh, kh)]
        st["q"], st["k"], st["v"] = [p.unflatten(2, (-1, D)) for p in parts]
        st["q_out"] = torch.empty(B, n, qh, D, dtype=dt, device="cuda")
        st["k_cache"], st["v_cache"] = st["k_cache"][0], st["v_cache"][0]
        st["rope"] = rope_table(max(lens) + n, case["rope"]) if case["rope"] else None
        st["q_norm"] = 1 + 0.1 * torch.randn(D, generator=g, device="cuda") if case["norm"] else None
        st["k_norm"] = 1 + 0.1 * torch.randn(D, generator=g, device="cuda") if case["norm"] else None
    elif case["op"] == "commit":
        path, length = _accepted(parent, rs)
        st.update(path=torch.from_numpy(path).cuda(), length=torch.from_numpy(length).cuda(),
                  new_len=torch.empty(B, dtype=torch.int32, device="cuda"))
    return st


# -------------------------------------------------------------- plain forms
def _ancestors(parent, depth):
    """[B][n][n]: whether node i is on the root path of node j."""
    B, n = parent.shape
    nodes = torch.arange(n, device=parent.device)
    at = nodes.expand(B, n)
    seen = at[:, :, None] == nodes
    for _ in range(min(depth, n) - 1):
        at = torch.where(at >= 0, parent.gather(1, at.clamp(min=0)).long(), at)
        seen = seen | (at[:, :, None] == nodes)
    return seen


def _plain_attend(st):
    case = st["case"]
    B, n, qh, D = st["q"].shape
    kh = case["kv_heads"]
    total = st["max_len"] + n
    cols = -(-total // case["page"])
    table = st["page_table"][:, :cols].long()

    def gather(cache):  # [B][kv heads][total][D]
        return cache[table].float().permute(0, 2, 1, 3, 4).reshape(B, kh, -1, D)[:, :, :total]

    q = st["q"].float().reshape(B, n, kh, qh // kh, D).transpose(1, 2).reshape(B, kh, -1, D)
    s = q @ gather(st["k_cache"]).transpose(2, 3).contiguous() * (1.0 / math.sqrt(D))
    node = torch.arange(total, device=q.device) - st["cache_len"][:, None]  # [B][total]
    seen = _ancestors(st["parent"], case["depth"])
    draft = seen.gather(2, node.clamp(0, n - 1)[:, None, :].expand(B, n, total))
    see = (node < 0)[:, None, :] | (draft & ((node >= 0) & (node < n))[:, None, :])
    s = s.view(B, kh, n, qh // kh, total).masked_fill_(~see[:, None, :, None, :], -math.inf).view(B, kh, -1, total)
    s = torch.exp(s - s.amax(3, keepdim=True))
    # rows no query reads hold whatever the pool held
    v = gather(st["v_cache"]) * (node < n)[:, None, :, None]
    o = (s @ v) / s.sum(3, keepdim=True)
    return o.view(B, kh, n, qh // kh, D).transpose(1, 2).reshape(B, n, qh, D).to(st["q"].dtype)


def _rotate(x, cos, sin, layout):
    """x [B][n][heads][D] in 32 bits; cos, sin [B][n][1][rope / 2]."""
    half = cos.shape[-1]
    rot, rest = x[..., :2 * half], x[..., 2 * half:]
    if layout == "half":
        a, b = rot[..., :half], rot[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = rot[..., 0::2], rot[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _rows(page_table, cache_len, nodes, page):
    """Pages and rows in them of each sequence's cache rows cache_len + nodes."""
    at = cache_len.long()[:, None] + nodes
    return page_table.gather(1, at // page).long(), at % page


def _plain_append(st):
    case = st["case"]
    B, n = st["parent"].shape
    depth = _ancestors(st["parent"], case["depth"]).sum(2)
    pos = st["cache_len"][:, None] + depth - 1
    out = []
    for x, w in ((st["q"], st["q_norm"]), (st["k"], st["k_norm"])):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w
        if st["rope"] is not None:
            cos, sin = st["rope"][pos.long()][:, :, None, :].chunk(2, -1)
            y = _rotate(y, cos, sin, case["layout"])
        out.append(y.to(x.dtype))
    st["q_out"].copy_(out[0])
    page, row = _rows(st["page_table"], st["cache_len"], torch.arange(n, device="cuda"), case["page"])
    st["k_cache"][page, :, row] = out[1]
    st["v_cache"][page, :, row] = st["v"]
    return st["q_out"], st["k_cache"], st["v_cache"]


def _plain_commit(st):
    case = st["case"]
    n = st["path"].shape[1]
    steps = torch.arange(n, device="cuda")
    live = steps < st["length"][:, None]
    nodes = torch.where(live, st["path"].long(), steps)  # rows past the path stay
    sp, sr = _rows(st["page_table"], st["cache_len"], nodes, case["page"])
    dp, dr = _rows(st["page_table"], st["cache_len"], steps.expand_as(nodes), case["page"])
    for c in (st["k_cache"], st["v_cache"]):
        c[:, dp, :, dr] = c[:, sp, :, sr]
    torch.add(st["cache_len"], st["length"], out=st["new_len"])
    return st["k_cache"], st["v_cache"], st["new_len"]


def _plain_copy(st):
    ps = st["case"]["page"]
    src, dst = st["src"].long(), st["dst"].long()
    for c in (st["k_cache"], st["v_cache"]):
        if st["rows"] is None:
            c[:, dst] = c[:, src]
        else:
            keep = torch.arange(ps, device="cuda") < st["rows"][:, None]
            c[:, dst] = torch.where(keep[:, None, :, None], c[:, src], c[:, dst])
    return st["k_cache"], st["v_cache"]


# --------------------------------------------------------------------- run
def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return dict(attend=_plain_attend, append=_plain_append, commit=_plain_commit, copy=_plain_copy)[op](st)
    from paper_2607_16673_amd import binding as B
    if op == "copy":
        B.sla_page_copy(st["k_cache"], st["v_cache"], st["src"], st["dst"], rows=st["rows"])
        return st["k_cache"], st["v_cache"]
    topology = "chain" if case["chain"] else "tree"
    if op == "attend":
        B.sla_attn_verify(st["q"], st["k_cache"], st["v_cache"], st["parent"], st["page_table"], st["cache_len"],
                          st["out"], max_len=st["max_len"], workspace=st["workspace"], status=st["status"],
                          topology=topology)
        return st["out"]
    if op == "append":
        B.sla_attn_append(st["q"], st["k"], st["v"], st["parent"], st["page_table"], st["cache_len"], st["q_out"],
                          st["k_cache"], st["v_cache"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS,
                          rope=st["rope"], layout=case["layout"], status=st["status"], topology=topology)
        return st["q_out"], st["k_cache"], st["v_cache"]
    B.sla_attn_commit(st["k_cache"], st["v_cache"], st["parent"], st["path"], st["length"], st["page_table"],
                      st["cache_len"], new_len=st["new_len"], status=st["status"])
    return st["k_cache"], st["v_cache"], st["new_len"]


# ------------------------------------------------------------------- exact
def _root_path(parent, j):
    out = []
    while j >= 0:
        out.append(j)
        j = int(parent[j])
    return out[::-1]


def _exact_attend(st, case):
    """One sequence at a time: its rows in order, each node's own list of them."""
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    qh, kh, D, n = case["q_heads"], case["kv_heads"], case["head"], case["n"]
    parent = st["parent"].cpu().numpy()
    for b, length in enumerate(_lens(case)):
        pages = st["page_table"][b, :-(-(length + n) // case["page"])].long()
        keys = torch.cat(list(st["k_cache"][pages].double()), 1)[:, :length + n]  # [kv heads][rows][D]
        vals = torch.cat(list(st["v_cache"][pages].double()), 1)[:, :length + n]
        hide = torch.zeros(n, length + n, dtype=torch.bool)
        hide[:, length:] = True
        for j in range(n):
            for a in _root_path(parent[b], j):
                hide[j, length + a] = False
        hide = hide.cuda()
        for h in range(kh):
            heads = slice(h * (qh // kh), (h + 1) * (qh // kh))
            q = st["q"][b, :, heads].double()  # [n][group][D]
            s = torch.matmul(q, keys[h].t()) / math.sqrt(D)
            s[hide[:, None, :].expand_as(s)] = -math.inf
            out[b, :, heads] = torch.matmul(torch.softmax(s, -1), vals[h])
    return out


def _exact_append(st, case):
    n, D, rope = case["n"], case["head"], case["rope"]
    parent = st["parent"].cpu().numpy()
    lens = _lens(case)
    depth = np.array([[len(_root_path(p, j)) for j in range(n)] for p in parent])
    pos = torch.from_numpy(depth + np.array(lens)[:, None] - 1).cuda()
    res = []
    for name, weight in (("q", "q_norm"), ("k", "k_norm")):
        x = st[name].double()
        if st[weight] is not None:
            x = st[weight].double() * x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS)
        if rope:
            turn = torch.complex(*[t.contiguous() for t in st["rope"][pos].double().unsqueeze(2).chunk(2, -1)])
            rot = x[..., :rope]
            pairs = rot.unflatten(-1, (2, -1)).transpose(-1, -2) if case["layout"] == "half" else \
                rot.unflatten(-1, (-1, 2))
            pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            rot = pairs.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else pairs.flatten(-2)
            x = torch.cat([rot, x[..., rope:]], -1)
        res.append(x)
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    table = st["page_table"].cpu().numpy()
    for b, length in enumerate(lens):
        for j in range(n):
            page, row = divmod(length + j, case["page"])
            page = int(table[b, page])
            kc[page, :, row] = res[1][b, j]
            vc[page, :, row] = st["v"][b, j].double()
    return res[0], kc, vc


def _exact_commit(st, case):
    lens = _lens(case)
    path, length, table = (st[x].cpu().numpy() for x in ("path", "length", "page_table"))
    ps = case["page"]
    src, dst = [], []
    for b in range(case["batch"]):
        for t in range(length[b]):
            a, c = lens[b] + int(path[b, t]), lens[b] + t
            src.append(int(table[b, a // ps]) * ps + a % ps)
            dst.append(int(table[b, c // ps]) * ps + c % ps)
    src, dst = torch.tensor(src, device="cuda"), torch.tensor(dst, device="cuda")
    out = []
    for name in ("k_cache", "v_cache"):
        c = st[name].double()
        rows = c.transpose(2, 3).flatten(1, 2)  # [layers][pages x rows][kv heads][D]
        moved = rows[:, src]
        rows = rows.clone()
        rows[:, dst] = moved
        out.append(rows.unflatten(1, (-1, ps)).transpose(2, 3).contiguous())
    return out[0], out[1], torch.tensor([a + int(x) for a, x in zip(lens, length)], device="cuda").int()


def _exact_copy(st, case):
    out = []
    rows = [case["page"]] * case["copies"] if st["rows"] is None else st["rows"].tolist()
    for name in ("k_cache", "v_cache"):
        c = st[name].double()
        for s, d, r in zip(st["src"].tolist(), st["dst"].tolist(), rows):
            c[:, d, :, :r] = st[name][:, s, :, :r].double()
        out.append(c)
    return tuple(out)


def exact(case, seed):
    st = prepare(case, seed)
    return dict(attend=_exact_attend, append=_exact_append, commit=_exact_commit, copy=_exact_copy)[case["op"]](st, case)

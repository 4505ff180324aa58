"""Speculative decoding of a small hybrid target: recurrent layers (gated delta
rule behind a short convolution) alternating with attention layers over a paged
cache, random weights, greedy sampling.

    python examples/hybrid_round.py [--tokens 64] [--branches 4] [--plain]

A prompt is run once, in chunks of 64 nodes; its sequence forks into branches
that go on from the prompt's likeliest next tokens and share its pages.  In a
round every branch drafts a tree, looked up in its own text, all layers verify
the trees in one pass, and the accepted paths are committed: the recurrent and
convolution states of every layer, and the cache rows of all attention layers in
one call.  --plain decodes one token a round instead; the tokens are the same.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_16673_amd import binding as sla  # noqa: E402
from paper_2607_16673_amd.cache import PagePool, rope_table  # noqa: E402

VOCAB, WIDTH, BLOCKS = 211, 256, 2   # a block: one recurrent layer, one attention layer
HEADS, KV_HEADS, HEAD, KERNEL = 8, 2, 64, 4
R_HEADS, R_HEAD = 4, 64
CHUNK = 64


def unit_rms(x):
    return x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-6)


class Target:
    """The weights, in fp32 or bf16; the stream between layers is fp32."""

    def __init__(self, seed=0, dtype=torch.float32, max_tokens=4096):
        g = torch.Generator().manual_seed(seed)
        mat = lambda *s: (torch.randn(*s, generator=g) * s[-2] ** -0.5).to(dtype).cuda()
        self.dtype = dtype
        self.embed = torch.randn(VOCAB, WIDTH, generator=g).cuda()
        self.head = mat(WIDTH, VOCAB)
        self.rope = rope_table(max_tokens, HEAD // 2, 1e4)
        self.layers = []
        for _ in range(BLOCKS):
            ones = lambda: (1 + 0.1 * torch.randn(HEAD, generator=g)).cuda()
            self.layers.append(dict(
                qkv=mat(WIDTH, 3 * R_HEADS * R_HEAD), gates=mat(WIDTH, 2 * R_HEADS),
                taps=(torch.randn(3 * R_HEADS * R_HEAD, KERNEL, generator=g) * 0.5).cuda(),
                out=mat(R_HEADS * R_HEAD, WIDTH), attn_qkv=mat(WIDTH, (HEADS + 2 * KV_HEADS) * HEAD),
                q_norm=ones(), k_norm=ones(), attn_out=mat(HEADS * HEAD, WIDTH)))


class Session:
    """A batch of sequences: recurrent and convolution states per layer, pages of one cache for all."""

    def __init__(self, target: Target, batch=1, pool=None, cache=None, pages=512, page_size=16):
        z = lambda *s: torch.zeros(*s, device="cuda")
        self.t, self.B = target, batch
        self.pool = pool or PagePool(pages, page_size)
        self.cache = cache or tuple(torch.zeros(BLOCKS, pages, KV_HEADS, page_size, HEAD, dtype=target.dtype,
                                                device="cuda") for _ in "kv")
        self.seqs = [self.pool.new() for _ in range(batch)]
        self.state = [z(batch, R_HEADS, R_HEAD, R_HEAD) for _ in range(BLOCKS)]
        self.conv = [z(batch, KERNEL - 1, 3 * R_HEADS * R_HEAD) for _ in range(BLOCKS)]

    def fork(self, batch):
        """`batch` continuations of this session's one sequence."""
        s = Session(self.t, 0, self.pool, self.cache)
        s.B, s.seqs = batch, [self.pool.fork(self.seqs[0]) for _ in range(batch)]
        s.state = [x.repeat(batch, 1, 1, 1) for x in self.state]
        s.conv = [x.repeat(batch, 1, 1) for x in self.conv]
        return s

    def verify(self, tokens, parent):
        """Logits [B][n][VOCAB] of every draft node; nothing is committed yet."""
        t, B, n = self.t, self.B, tokens.shape[1]
        copies = self.pool.reserve_all(self.seqs, n)
        if copies:  # pages that a fork shared until now
            src, dst, rows = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in zip(*copies))
            sla.sla_page_copy(*self.cache, src, dst, rows=rows)
        self.parent = torch.from_numpy(parent).cuda()
        self.table = torch.from_numpy(self.pool.table(self.seqs)).cuda()
        self.len = torch.tensor([s.length for s in self.seqs], dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1 + 3 * BLOCKS, B, dtype=torch.int32, device="cuda")
        longest = max(s.length for s in self.seqs)
        self.kept = []
        x = t.embed[torch.from_numpy(tokens).long().cuda()]
        for i, w in enumerate(t.layers):
            # recurrent: projections, convolution, gated delta rule
            h = unit_rms(x).to(t.dtype)
            u, gates = h @ w["qkv"], (h @ w["gates"]).float().sigmoid()
            y = torch.empty_like(u)
            sla.sla_conv_verify(self.conv[i], u, w["taps"], self.parent, y, status=self.status[3 * i])
            q, k, v = (p.unflatten(2, (R_HEADS, R_HEAD)) for p in y.split(R_HEADS * R_HEAD, 2))
            q, k = (torch.nn.functional.normalize(p.float(), dim=-1).to(t.dtype) for p in (q, k))
            alpha, beta = (p.contiguous() for p in (0.9 + 0.1 * gates[..., :R_HEADS], gates[..., R_HEADS:]))
            o = torch.empty(B, n, R_HEADS, R_HEAD, device="cuda")
            factors = sla.Factors.empty(B, n, R_HEADS, R_HEAD, R_HEAD, t.dtype)
            sla.sla_verify(self.state[i], q, k, v.contiguous(), alpha, beta, self.parent, o, factors,
                           status=self.status[3 * i + 1])
            self.kept.append((u, factors))
            x = x + (unit_rms(o).flatten(2).to(t.dtype) @ w["out"]).float()
            # attention: one fused projection, norms and rotation on the way into the cache
            qkv = (unit_rms(x).to(t.dtype) @ w["attn_qkv"]).unflatten(2, (-1, HEAD))
            q, k, v = qkv.split([HEADS, KV_HEADS, KV_HEADS], 2)
            k_cache, v_cache = (c[i] for c in self.cache)
            turned = torch.empty(B, n, HEADS, HEAD, dtype=t.dtype, device="cuda")
            sla.sla_attn_append(q, k, v, self.parent, self.table, self.len, turned, k_cache, v_cache,
                                q_norm=w["q_norm"], k_norm=w["k_norm"], rope=t.rope, status=self.status[3 * i + 2])
            o = torch.empty_like(turned)
            sla.sla_attn_verify(turned, k_cache, v_cache, self.parent, self.table, self.len, o, max_len=longest,
                                workspace=sla.attn_workspace(turned, k_cache, self.table, max_len=longest))
            x = x + (o.flatten(2) @ w["attn_out"]).float()
        return (unit_rms(x).to(t.dtype) @ t.head).float()

    def commit(self, path, length):
        """Advance every layer along the accepted paths."""
        p, m = torch.from_numpy(path).cuda(), torch.from_numpy(length).cuda()
        for i, (u, factors) in enumerate(self.kept):
            sla.sla_conv_commit(self.conv[i], u, self.parent, p, m, kernel_size=KERNEL)
            sla.sla_commit(self.state[i], factors, p, m)
        sla.sla_attn_commit(*self.cache, self.parent, p, m, self.table, self.len, status=self.status[-1])
        if self.status.any():
            raise RuntimeError("a sequence's data are bad: %s" % self.status.tolist())
        for s, k in zip(self.seqs, length):
            s.length += int(k)

    def prompt(self, tokens):
        """Run a prompt (the same in every sequence); returns the last token's logits."""
        for i in range(0, len(tokens), CHUNK):
            part = np.tile(np.asarray(tokens[i:i + CHUNK], np.int32), (self.B, 1))
            chain = np.tile(np.arange(-1, part.shape[1] - 1, dtype=np.int32), (self.B, 1))
            logits = self.verify(part, chain)
            self.commit(chain + 1, np.full(self.B, part.shape[1], np.int32))
        return logits[:, -1]

    def close(self):
        for s in self.seqs:
            self.pool.free(s)


def draft(text, nodes, depth):
    """A tree over the last token: what followed its latest earlier places in the
    text, chains that share their common starts.  Padded with leaves that repeat
    the root's first guess."""
    tokens, parent = [text[-1]], [-1]
    places = [i for i in range(len(text) - 2, -1, -1) if text[i] == text[-1]]
    for place in places:
        at = 0
        for tok in text[place + 1:place + 1 + depth]:
            kids = [j for j in range(len(tokens)) if parent[j] == at and tokens[j] == tok]
            if not kids:
                if len(tokens) == nodes:
                    break
                kids = [len(tokens)]
                tokens.append(tok)
                parent.append(at)
            at = kids[0]
    while len(tokens) < nodes:
        tokens.append(tokens[min(1, len(tokens) - 1)])
        parent.append(0)
    return tokens, parent


def accept(tokens, parent, best):
    """The root path along which every next token is the target's choice, and the choice behind it."""
    path = [0]
    while True:
        nxt = [j for j in range(len(tokens)) if parent[j] == path[-1] and tokens[j] == best[path[-1]]]
        if not nxt:
            return path, int(best[path[-1]])
        path.append(nxt[0])


def generate(target, prompt, tokens, branches, nodes=16, depth=6):
    """(texts, rounds): `branches` continuations of the prompt by `tokens` tokens each."""
    base = Session(target)
    first = base.prompt(prompt)[0].topk(branches).indices.tolist()
    s = base.fork(branches)
    base.close()
    texts, rounds = [list(prompt) + [f] for f in first], 0
    while min(len(t) for t in texts) < len(prompt) + tokens:
        drafts = [draft(t, nodes, depth) for t in texts]
        best = s.verify(np.array([d[0] for d in drafts], np.int32), np.array([d[1] for d in drafts], np.int32))
        best = best.argmax(-1).cpu().numpy()
        path, length = np.full((branches, nodes), -1, np.int32), np.zeros(branches, np.int32)
        for b, (tok, par) in enumerate(drafts):
            nodes_in, nxt = accept(tok, par, best[b])
            path[b, :len(nodes_in)], length[b] = nodes_in, len(nodes_in)
            texts[b] += [tok[j] for j in nodes_in[1:]] + [nxt]
        s.commit(path, length)
        rounds += 1
    s.close()
    return [t[len(prompt):len(prompt) + tokens] for t in texts], rounds


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--branches", type=int, default=4)
    ap.add_argument("--plain", action="store_true", help="one token a round")
    args = ap.parse_args()
    prompt = np.random.default_rng(0).integers(0, VOCAB, 150).tolist()
    target = Target()
    generate(target, prompt, 2, args.branches)  # the first calls load the kernels
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    texts, rounds = generate(target, prompt, args.tokens, args.branches, nodes=1 if args.plain else 16)
    took = time.perf_counter() - t0
    for t in texts:
        print(" ".join(map(str, t)))
    print("%d branches of %d tokens in %d rounds, %.1f ms" % (args.branches, args.tokens, rounds, took * 1e3))


if __name__ == "__main__":
    main()

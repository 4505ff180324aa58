"""Helpers of the attention tests: caches with sequences laid out over
shuffled pages, drafts, and the error bounds of the kernels' roundings."""
from __future__ import annotations

import numpy as np
import torch

from oracle import attention as O
from paper_2607_16673_amd import inputs

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def draft(rng, B, n, chain=False):
    """Parent arrays [B][n]: chains, or trees and forests of random depth."""
    if chain:
        return np.tile(inputs.chain(n), (B, 1))
    return np.stack([np.array([rng.integers(-1 if rng.random() < 0.1 else min(0, j - 1), j) if j else -1
                               for j in range(n)], np.int32) for _ in range(B)])


def path_of(rng, parent):
    """A drawn node's root path per sequence (or none): path [B][n], len [B]."""
    B, n = parent.shape
    path, length = np.full((B, n), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        nodes = O.root_path(parent[b], int(rng.integers(-1, n)))
        path[b, :len(nodes)] = nodes
        length[b] = len(nodes)
    return path, length


class Case:
    """A batch's draft behind committed rows, on the host in the activation type's values."""

    def __init__(self, lens, n, hq, hkv, D, page, dtype, *, seed=0, chain=False, layers=None, spare=3, qstd=2.0,
                 fill=None):
        rng = self.rng = np.random.default_rng(seed)
        self.B, self.n, self.hq, self.hkv, self.D, self.page, self.dtype = len(lens), n, hq, hkv, D, page, dtype
        self.lens = np.array(lens, np.int32)
        counts = [-(-(l + n) // page) for l in lens]
        self.pages = sum(counts) + spare
        ids = rng.permutation(self.pages).astype(np.int32)
        # entries past a sequence's last page are no page numbers
        self.table = np.full((self.B, max(counts) + 1), 1 << 30, np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = ids[at:at + c]
            at += c
        self.parent = draft(rng, self.B, n, chain)
        self.chain = chain
        shape = (self.pages, hkv, page, D)
        self.k, self.v = (self.values((layers,) + shape if layers else shape) for _ in range(2))
        self.q = self.values((self.B, n, hq, D), qstd)
        if fill is not None:  # every row that belongs to no sequence
            used = np.zeros((self.pages, page), bool)
            for b in range(self.B):
                for r in range(int(self.lens[b]) + n):
                    used[O.row_of(self.table[b], r, page)] = True
            for c in (self.k, self.v):
                c.swapaxes(-3, -2)[..., ~used, :, :] = fill

    def values(self, shape, std=1.0):
        x = (self.rng.standard_normal(shape) * std).astype(np.float32)
        return inputs.bf16_to_f32(inputs.bf16_bits(x)) if self.dtype == "bf16" else x

    def dev(self, x):
        t = torch.from_numpy(np.ascontiguousarray(x))
        return (t.to(TORCH[self.dtype]) if t.dtype == torch.float32 else t).cuda()

    @property
    def topology(self):
        return "chain" if self.chain else "tree"


def verify_bound(o, a, dtype):
    """What |y - o| may reach.  bf16: every weight is rounded to 8 significant bits (2^-8
    relative, against sum p |v|) and the output once more (2^-8 |o|).  Both
    types: scores and sums in fp32; a score is D products of size ~|q||k| / D^0.5
    and stays below 2^6, so it is off by 2^6 2^-24 and a few more roundings,
    which 2^-17 of sum p |v| covers; 2^-17 = 7.6e-6 is inside the library's fp32
    bar of 1e-5."""
    fp32 = 2.0 ** -17 * (a + a.max() * 2.0 ** -4)
    return fp32 if dtype == "f32" else fp32 + 2.0 ** -8 * (a + np.abs(o)) * (1 + 2.0 ** -6)


def rounded_bound(r, dtype):
    """One value computed in fp32 (a mean square, a root, a few products: some
    16 roundings of values up to max |r|), then rounded to the activation type."""
    fp32 = 2.0 ** -20 * max(float(np.abs(r).max()), 1e-30)
    return fp32 if dtype == "f32" else fp32 + 2.0 ** -8 * np.abs(r) * (1 + 2.0 ** -6)

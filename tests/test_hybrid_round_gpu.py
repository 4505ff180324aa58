"""The hybrid target of the example on the GPU: branches decoded by drafted
trees give the tokens of decoding one at a time, and of a plain 64-bit model of
the whole text; forked branches share the prompt's pages and give all back."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_round.py")
    spec = importlib.util.spec_from_file_location("hybrid_round", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(E, target, tokens):
    """The model over a whole text, token by token, in 64 bits on the CPU."""
    f = lambda t: t.double().cpu().numpy()
    rms = lambda x: x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)
    sig = lambda x: 1 / (1 + np.exp(-x))
    T, H, D = len(tokens), E.R_HEADS, E.R_HEAD
    x = f(target.embed)[tokens]
    rope = f(target.rope)
    for w in target.layers:
        h = rms(x)
        u, gates, taps = h @ f(w["qkv"]), sig(h @ f(w["gates"])), f(w["taps"])
        pad = np.concatenate([np.zeros((E.KERNEL - 1, u.shape[1])), u])
        y = sum(pad[i:i + T] * taps[:, i] for i in range(E.KERNEL))
        y = y * sig(y)
        q, k, v = [p.reshape(T, H, D) for p in np.split(y, 3, 1)]
        q, k = [p / np.linalg.norm(p, axis=-1, keepdims=True) for p in (q, k)]
        alpha, beta = 0.9 + 0.1 * gates[:, :H], gates[:, H:]
        o, S = np.zeros((T, H, D)), np.zeros((H, D, D))
        for t in range(T):
            S = S * alpha[t, :, None, None]
            S = S + beta[t, :, None, None] * k[t, :, :, None] * (v[t] - np.einsum("hk,hkv->hv", k[t], S))[:, None, :]
            o[t] = np.einsum("hk,hkv->hv", q[t], S)
        x = x + rms(o).reshape(T, -1) @ f(w["out"])
        qkv = (rms(x) @ f(w["attn_qkv"])).reshape(T, -1, E.HEAD)
        q, k, v = np.split(qkv, [E.HEADS, E.HEADS + E.KV_HEADS], 1)
        q, k = rms(q) * f(w["q_norm"]), rms(k) * f(w["k_norm"])
        r = rope.shape[1] // 2
        c, s = rope[:T, None, :r], rope[:T, None, r:]
        for p in (q, k):
            a, b = p[..., :r].copy(), p[..., r:2 * r].copy()
            p[..., :r], p[..., r:2 * r] = a * c - b * s, b * c + a * s
        o, G = np.zeros((T, E.HEADS, E.HEAD)), E.HEADS // E.KV_HEADS
        for h in range(E.HEADS):
            sc = q[:, h] @ k[:, h // G].T * E.HEAD ** -0.5
            sc[np.triu_indices(T, 1)] = -np.inf
            p = np.exp(sc - sc.max(1, keepdims=True))
            o[:, h] = p / p.sum(1, keepdims=True) @ v[:, h // G]
        x = x + o.reshape(T, -1) @ f(w["attn_out"])
    return rms(x) @ f(target.head)


def test_trees_give_the_tokens_of_plain_decoding(E):
    target = E.Target()
    prompt = np.random.default_rng(0).integers(0, E.VOCAB, 150).tolist()
    want, steps = E.generate(target, prompt, 40, 3, nodes=1)
    got, rounds = E.generate(target, prompt, 40, 3, nodes=16)
    assert got == want and steps == 39 and rounds < steps
    for branch in want:  # each token is the plain model's choice, or ties with it in fp32
        logits = plain_logits(E, target, prompt + branch)[len(prompt):-1]
        for row, token in zip(logits, branch[1:]):
            assert row.max() - row[token] < 1e-3


def test_prompt_logits(E):
    target = E.Target(seed=1)
    tokens = np.random.default_rng(1).integers(0, E.VOCAB, 130).tolist()
    got = E.Session(target).prompt(tokens)[0].double().cpu().numpy()
    want = plain_logits(E, target, tokens)[-1]
    # logits of size ~3 through four layers and 130 steps of fp32 sums of up to
    # 768 products: some 2^-24 2^6 a layer, left 2^3 of room
    assert np.abs(got - want).max() < np.abs(want).max() * 2.0 ** -13


def test_branches_share_and_return_pages(E):
    s = E.Session(E.Target(), pages=40)
    tokens = np.random.default_rng(2).integers(0, E.VOCAB, 72).tolist()
    s.prompt(tokens)
    used = 40 - s.pool.free_pages
    b = s.fork(3)
    assert 40 - s.pool.free_pages == used == 5
    s.close()
    one = np.zeros((3, 1), np.int32)
    b.verify(one, one - 1)
    assert len({q.pages[4] for q in b.seqs}) == 3 and len({tuple(q.pages[:4]) for q in b.seqs}) == 1
    for layer in range(E.BLOCKS):  # the shared half page went along
        k = b.cache[0][layer]
        first, rest = [k[q.pages[4], :, :9] for q in b.seqs[:1]], [k[q.pages[4], :, :9] for q in b.seqs[1:]]
        assert all(torch.equal(first[0], x) for x in rest) and first[0].abs().min() > 0
    b.commit(one, np.ones(3, np.int32))
    b.close()
    assert s.pool.free_pages == 40

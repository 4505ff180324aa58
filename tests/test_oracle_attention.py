"""Pins of the attention oracle: against worked numbers, closed forms and a
second formulation with whole masks."""
import numpy as np

from attn_util import Case, path_of
from oracle import attention as O


def rows(cache, table, count, page):
    return np.stack([cache[table[r // page], :, r % page] for r in range(count)])  # [rows][heads][D]


def test_verify_against_whole_masks():
    for seed, (n, hq, hkv, page) in enumerate([(1, 4, 2, 16), (9, 6, 2, 16), (20, 3, 3, 32), (64, 4, 1, 64)]):
        c = Case([0, 5, 70], n, hq, hkv, 64, page, "f32", seed=seed)
        o, a = O.verify(c.q, c.k, c.v, c.parent, c.table, c.lens, 0.3)
        for b in range(c.B):
            T = int(c.lens[b]) + n
            k, v = (rows(x.astype(np.float64), c.table[b], T, page) for x in (c.k, c.v))
            see = np.zeros((n, T), bool)
            see[:, :T - n] = True
            for j in range(n):
                see[j, T - n + j] = True
                if c.parent[b, j] >= 0:
                    see[j, T - n:] |= see[c.parent[b, j], T - n:]
            for h in range(hq):
                s = np.where(see, 0.3 * c.q[b, :, h].astype(np.float64) @ k[:, h // (hq // hkv)].T, -np.inf)
                p = np.exp(s) / np.exp(s).sum(1, keepdims=True)
                np.testing.assert_allclose(o[b, :, h], p @ v[:, h // (hq // hkv)], rtol=0, atol=1e-12)
                np.testing.assert_allclose(a[b, :, h], p @ np.abs(v[:, h // (hq // hkv)]), rtol=0, atol=1e-12)


def test_verify_closed_forms():
    c = Case([6], 3, 2, 1, 64, 16, "f32")
    c.parent = np.array([[-1, 0, 0]], np.int32)
    o, _ = O.verify(c.q, c.k, c.v, c.parent, c.table, c.lens, 0.0)  # equal weights
    v = rows(c.v.astype(np.float64), c.table[0], 9, 16)[:, 0]
    np.testing.assert_allclose(o[0, 2, 1], np.concatenate([v[:7], v[8:9]]).mean(0), atol=1e-14)
    c = Case([0], 1, 1, 1, 64, 16, "f32")  # one key
    np.testing.assert_allclose(O.verify(c.q, c.k, c.v, c.parent, c.table, c.lens)[0][0, 0, 0],
                               c.v[c.table[0, 0], 0, 0], rtol=1e-15)


def test_transform():
    x = np.arange(1.0, 17.0)
    y = O.transform(x, 0, np.full(16, 2.0), 0.0, None, "half")
    np.testing.assert_allclose(np.sqrt(np.mean(y * y)), 2.0)
    rope = np.zeros((4, 8))
    rope[2] = [np.cos(0.3), 0, 1, 1, np.sin(0.3), 1, 0, 0]
    for layout, pairs in (("half", [(0, 4), (1, 5), (2, 6), (3, 7)]), ("interleaved", [(0, 1), (2, 3), (4, 5), (6, 7)])):
        y = O.transform(x, 2, None, 0.0, rope, layout)
        z = [complex(x[a], x[b]) for a, b in pairs]
        want = [z[0] * np.exp(0.3j), z[1] * 1j, z[2], z[3]]
        np.testing.assert_allclose([complex(y[a], y[b]) for a, b in pairs], want, atol=1e-14)
        np.testing.assert_array_equal(y[8:], x[8:])


def test_append_places_rows_by_depth_and_number():
    c = Case([15, 3], 4, 1, 1, 64, 16, "f32")
    c.parent = np.array([[-1, 0, 0, 2], [-1, 0, 1, 2]], np.int32)
    rope = np.zeros((40, 16))
    rope[:, :8] = np.arange(40)[:, None]  # multiplies the pairs by the position
    one = np.ones((2, 4, 1, 64))
    q, k, v = O.append(one, one, 2 * one, c.parent, c.table, c.lens, c.k, c.v, rope=rope)
    assert q[0, :, 0, 0].tolist() == [15, 16, 16, 17] and q[1, :, 0, 0].tolist() == [3, 4, 5, 6]
    assert (q[..., 16:] == 1).all()
    np.testing.assert_array_equal(rows(k, c.table[0], 19, 16)[15:, 0, 0], [15, 16, 16, 17])
    np.testing.assert_array_equal(rows(v, c.table[1], 7, 16)[3:], 2)
    np.testing.assert_array_equal(rows(v, c.table[1], 3, 16), rows(c.v, c.table[1], 3, 16))


def test_a_committed_round_is_the_tokens_one_by_one():
    """Appending a tree and committing a path leaves the cache that appending the
    path's tokens as a chain would."""
    for seed in range(4):
        c = Case([0, 14, 33], 9, 2, 2, 64, 16, "f32", seed=seed)
        rope = c.rng.uniform(-1, 1, (60, 32))
        q, k, v = (c.values((3, 9, 2, 64)) for _ in range(3))
        path, acc = path_of(c.rng, c.parent)
        _, kt, vt = O.append(q, k, v, c.parent, c.table, c.lens, c.k, c.v, rope=rope)
        kt, vt = (O.commit(x[None], path, acc, c.table, c.lens)[0] for x in (kt, vt))
        for b in range(3):
            m = int(acc[b])
            if m == 0:
                continue
            pick = lambda x: x[b:b + 1, path[b, :m]]
            chain = np.arange(-1, m - 1, dtype=np.int32)[None]
            _, kc, vc = O.append(pick(q), pick(k), pick(v), chain, c.table[b:b + 1], c.lens[b:b + 1], c.k, c.v, rope=rope)
            T = int(c.lens[b]) + m
            np.testing.assert_array_equal(rows(kt, c.table[b], T, 16), rows(kc, c.table[b], T, 16))
            np.testing.assert_array_equal(rows(vt, c.table[b], T, 16), rows(vc, c.table[b], T, 16))


def test_page_copy():
    x = np.arange(2 * 3 * 1 * 4 * 2).reshape(2, 3, 1, 4, 2)
    y = O.page_copy(x, [0], [2], [3])
    np.testing.assert_array_equal(y[:, 2, :, :3], x[:, 0, :, :3])
    np.testing.assert_array_equal(y[:, 2, :, 3], x[:, 2, :, 3])
    np.testing.assert_array_equal(y[:, :2], x[:, :2])

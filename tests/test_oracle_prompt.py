"""Pins of the prompt-pass oracle: against the draft oracle, a chunked form with
whole matrices, and worked numbers."""
import numpy as np
import pytest

import oracle
from oracle import prompt as O


def draw(T, Hk, H, dk, dv, seed):
    r = np.random.default_rng(seed)
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)
    f = lambda x: x.astype(np.float32)
    return (f(unit(r.normal(size=(T, Hk, dk)))), f(unit(r.normal(size=(T, Hk, dk)))), f(r.normal(size=(T, H, dv))),
            f(r.uniform(0.5, 1, (T, H))), f(r.uniform(0, 1, (T, H))))


def test_a_chain_of_the_draft_oracle():
    q, k, v, a, b = draw(12, 2, 2, 64, 16, 0)
    S = np.random.default_rng(1).normal(size=(1, 2, 64, 16)).astype(np.float32)
    out, new = O.prefill(S, q, k, v, a, b, [0, 12])
    parent = np.arange(-1, 11, dtype=np.int32)[None]
    one = lambda x: np.ascontiguousarray(x[None])
    want, st = oracle.verify(S, one(q), one(k), one(v), one(a), one(b), parent)
    assert st[0] == 0
    np.testing.assert_allclose(out, want[0], rtol=0, atol=1e-12)
    state, st = oracle.commit(S, one(k), one(v), one(a), one(b), parent, parent + 1, np.array([12], np.int32))
    np.testing.assert_allclose(new, state, rtol=0, atol=1e-12)


@pytest.mark.parametrize("family", ["gdn", "deltanet", "decay"])
def test_against_whole_matrices(family):
    """All tokens as one triangular system."""
    n, H = 20, 4
    q, k, v, a, b = (x.astype(np.float64) for x in draw(n, 2, H, 64, 16, 2))
    S0 = np.random.default_rng(3).normal(size=(1, H, 64, 16))
    out, new = O.prefill(S0, q, k, v, a, b, [0, n], family)
    for h in range(H):
        K, Q, V, S = k[:, h // 2], q[:, h // 2], v[:, h], S0[0, h]
        al = np.ones(n) if family == "deltanet" else a[:, h]
        G = np.cumprod(al)
        D = np.tril(G[:, None] / G[None, :])
        U = V
        if family != "decay":
            X = np.linalg.inv(np.eye(n) + np.tril(b[:, h, None] * D * (K @ K.T), -1))
            U = X @ (b[:, h, None] * (V - G[:, None] * (K @ S)))
        np.testing.assert_allclose(out[:, h], G[:, None] * (Q @ S) + (D * (Q @ K.T)) @ U, rtol=0, atol=1e-11)
        np.testing.assert_allclose(new[0, h], G[-1] * S + (K * D[-1][:, None]).T @ U, rtol=0, atol=1e-11)


def test_packed_sequences():
    q, k, v, a, b = draw(30, 1, 1, 64, 16, 4)
    out, new = O.prefill(None, q, k, v, a, b, [3, 10, 10, 27])
    assert np.isnan(out[:3]).all() and np.isnan(out[27:]).all() and not new[1].any()
    for i, (s, e) in enumerate([(3, 10), (10, 10), (10, 27)]):
        o, n = O.prefill(None, q[s:e], k[s:e], v[s:e], a[s:e], b[s:e], [0, e - s])
        np.testing.assert_array_equal(out[s:e], o)
        np.testing.assert_array_equal(new[i], n[0])


def test_conv():
    x = np.arange(1.0, 6.0)[:, None]
    w = np.array([[100.0, 10.0, 1.0]])
    y, new = O.conv(np.array([[[8.0], [9.0]], [[3.0], [4.0]]]), x, w, None, [0, 1, 5], silu=False)
    np.testing.assert_array_equal(y[:, 0], [891.0, 342.0, 423.0, 234.0, 345.0])
    np.testing.assert_array_equal(new[:, :, 0], [[9.0, 1.0], [4.0, 5.0]])
    y, _ = O.conv(None, x[:1], w, np.array([-1.0]), [0, 1])
    assert y[0, 0] == 0.0
    y, _ = O.conv(None, x[:1], w, np.array([1.0]), [0, 1])
    np.testing.assert_allclose(y[0, 0], 2 / (1 + np.exp(-2.0)))


def test_inputs_and_norm():
    q, k, a, b = O.inputs(np.array([[[3.0, 4.0]]]), np.array([[[0.0, 2.0]]]), np.array([[1.0]]), np.array([[0.0]]),
                          np.array([np.log(2.0)]), np.array([-1.0]), 0.5, 0.0, 2)
    np.testing.assert_allclose(q, [[[0.3, 0.4]] * 2])
    np.testing.assert_allclose(k, [[[0.0, 1.0]] * 2])
    np.testing.assert_allclose([a[0, 0], b[0, 0]], [0.25, 0.5])  # exp(-2 log 2)
    x, z, w = np.array([[[1.0, -1.0]]]), np.array([[[0.0, np.log(3.0)]]]), np.array([2.0, 4.0])
    np.testing.assert_allclose(O.gated_norm(x, z, w, 3.0, "sigmoid"), [[[0.5, -1.5]]])
    np.testing.assert_allclose(O.gated_norm(x, z, w, 3.0, "silu"), [[[0.0, -1.5 * np.log(3.0)]]])
    np.testing.assert_allclose(O.gated_norm(x, None, None, 0.0, "none"), x)

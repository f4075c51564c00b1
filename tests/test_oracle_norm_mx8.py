"""Pins of the norm's, the 8-bit blocks' and the kept-activation experts' oracles: worked numbers, search over every code,
central differences of the forward, the plain layer's oracle."""

import numpy as np
import pytest

from oracle import ffn
from oracle import mx8 as M
from oracle import norm as N


def test_a_worked_block():
    v = np.zeros((1, 64))
    v[0, :6] = [3.0, -1.5, 0.0234375, 0.015625, 0.046875, 3.99]   # exponent 1: steps of 1/32
    c, e = M.quantize(v)
    assert e.tolist() == [[1, -127]] and c[0, :6].tolist() == [96, -48, 1, 0, 2, 127] and not c[0, 6:].any()
    assert M.values(c, e)[0, :6].tolist() == [3.0, -1.5, 0.03125, 0.0, 0.0625, 3.96875]


def test_nearest_code_by_search():
    g = np.random.default_rng(0)
    v = g.standard_normal((200, 32)) * 10.0 ** g.integers(-30, 30, (200, 1))
    c, e = M.quantize(v)
    every = np.arange(-127, 128) * np.exp2(e - 6.0)[..., None]      # [200, 1, 255]
    best = np.abs(v[..., None] - every).min(-1)
    assert np.array_equal(np.abs(M.values(c, e) - v), best)
    assert (np.abs(v).max(-1) >= np.exp2(e[:, 0])).all() and (np.abs(v).max(-1) < np.exp2(e[:, 0] + 1)).all()


def test_blocks_at_the_ends_of_the_range():
    v = np.zeros((4, 32))
    v[0, 0], v[1, 0], v[2, 0], v[3, 0] = 2.0 ** -149, 2.0 ** -127, 1.5 * 2.0 ** 127, np.inf
    c, e = M.quantize(v)
    assert e[:, 0].tolist() == [-127, -127, 127, 128] and c[:, 0].tolist() == [0, 64, 96, 0]
    assert np.isnan(M.values(c, e)[3]).all() and M.values(c, e)[2, 0] == v[2, 0]


@pytest.mark.parametrize("residual", [False, True])
def test_norm_gradient_by_differences(residual):
    g = np.random.default_rng(1)
    T, d, eps = 3, 7, 1e-3
    x, r, w, dy, dh = (g.standard_normal(s) for s in ((T, d), (T, d), (d,), (T, d), (T, d)))
    r = r if residual else None

    def loss(x, w):
        s, _, y, _, _ = N.forward(x, r, w, eps, 0.0)
        return (dy * y).sum() + (dh * s).sum()
    h = x if r is None else x + r
    dx, _, dw, _ = N.backward(h, w, dy, dh, eps, 0.0)
    for a, grad in ((x, dx), (w, dw)):
        num = np.zeros_like(a)
        for i in np.ndindex(a.shape):
            for s in (1, -1):
                b = a.copy()
                b[i] += s * 1e-5
                num[i] += s * (loss(b, w) if a is x else loss(x, b)) / 2e-5
        assert np.abs(num - grad).max() <= 1e-8 * max(1, np.abs(grad).max())


def make(T=5, d=6, F=32, E=4, K=2, ns=1, seed=2):
    g = np.random.default_rng(seed)
    x, dy = g.standard_normal((2, T, d))
    idx = np.stack([g.permutation(E)[:K] for _ in range(T)])
    idx[1, 0] = -1
    idx[2] = idx[2, 0]
    return x, idx, g.random((T, K)), g.standard_normal((E + ns, 2 * F, d)), g.standard_normal((E + ns, d, F)), ns, dy


def test_forward_is_the_plain_layer():
    x, idx, gate, wg, wd, ns, _ = make()
    y, _, ab, _ = M.forward(x, idx, gate, wg, wd, ns)
    for t in range(len(x)):
        want = sum(gate[t, k] * ffn.expert_ffn(x[t:t + 1], wg[e], wd[e])[0] for k, e in enumerate(idx[t]) if e >= 0)
        want = want + sum(ffn.expert_ffn(x[t:t + 1], wg[-1 - s], wd[-1 - s])[0] for s in range(ns))
        assert np.allclose(y[t], want, rtol=1e-12, atol=1e-12)
    assert len(ab) == (idx >= 0).sum() + ns * len(x)
    r = M.rows(idx, len(wg) - ns, ns)
    assert r == sorted(r, key=lambda v: (v[2], v[0], v[1])) and len(set(r)) == len(r)
    t, _, e = r[3]
    assert np.allclose(ab[3], wg[e] @ x[t])


def test_gradients_by_differences():
    x, idx, gate, wg, wd, ns, dy = make()
    ab = M.forward(x, idx, gate, wg, wd, ns)[2]
    grads = M.backward(x, idx, gate, wg, wd, ns, ab, dy)
    args = dict(d_x=x, d_gate=gate, d_w_gate_up=wg, d_w_down=wd)
    g = np.random.default_rng(3)
    for name, a in args.items():
        grad = grads[name][0]
        at = list(np.ndindex(a.shape))
        for i in [at[j] for j in g.permutation(len(at))[:40]]:
            keep, num = a[i], 0.0
            for s in (1, -1):
                a[i] = keep + s * 1e-6
                num += s * (dy * M.forward(x, idx, gate, wg, wd, ns)[0]).sum() / 2e-6
            a[i] = keep
            assert abs(num - grad[i]) <= 1e-6 * max(1.0, np.abs(grad).max()), (name, i)
    assert grads["d_gate"][0][1, 0] == 0

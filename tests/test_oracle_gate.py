"""Pins of the gate and MX4 oracles that do not rest on their own formulas."""

import numpy as np
import pytest
import torch

from oracle import gate as G
from oracle import mx4 as M
from oracle import routing as R


def _z(T, E, seed=0, std=1.3):
    return std * np.random.default_rng(seed).standard_normal((T, E))


@pytest.mark.parametrize("renorm", [False, True])
def test_softmax_without_bias_is_the_plain_routing_rule(renorm):
    z = _z(50, 64)
    idx, gate, load = G.forward(z, 6, G.SOFTMAX, renorm=renorm)
    io, go, _ = R.route_logits(z, 6, R.PLAIN, R.GATE_RENORM if renorm else R.GATE_P)
    assert np.array_equal(idx, io) and np.abs(gate - go).max() < 1e-12
    assert load.sum() == 300 and load[idx[0, 0]] >= 1


def test_hard_mask_and_prior_are_the_routing_rules_sets():
    z = _z(40, 16, 1)
    mask = np.zeros(16, np.uint8)
    mask[[1, 2, 5, 9, 12]] = 1
    assert np.array_equal(G.forward(z, 3, G.SOFTMAX, mask=mask)[0], R.route_logits(z, 3, R.HARD_MASK, R.GATE_P, mask=mask)[0])
    prior = np.exp(np.random.default_rng(2).standard_normal(16))
    prior /= prior.sum()
    assert np.array_equal(G.forward(z, 3, G.SOFTMAX, prior=prior)[0],
                          R.route_logits(z, 3, R.SOFT_PRIOR, R.GATE_P, prior=prior)[0])


def test_hand_worked_groups():
    """Six experts in three groups of two, scores by hand: sums of two prefer group 1, maxima group 0 and 2."""
    s = np.array([[0.9, 0.1, 0.6, 0.55, 0.8, 0.2]])
    z = np.log(s / (1 - s))
    kw = dict(n_group=3, topk_group=1, renorm=False)
    assert G.forward(z, 2, G.SIGMOID, group_rule=G.GROUP_SUM2, **kw)[0].tolist() == [[2, 3]]
    assert G.forward(z, 2, G.SIGMOID, group_rule=G.GROUP_MAX, **kw)[0].tolist() == [[0, 1]]
    bias = np.array([0, 0, 0, 0, 0.05, 0.15])
    idx, gate, _ = G.forward(z, 2, G.SIGMOID, group_rule=G.GROUP_SUM2, bias=bias, **kw)
    assert idx.tolist() == [[4, 5]] and np.allclose(gate, [[0.8, 0.2]])
    mask = np.array([1, 1, 0, 1, 0, 0])   # one expert left in group 1, none in group 2
    assert G.forward(z, 2, G.SIGMOID, mask=mask, n_group=3, topk_group=2)[0].tolist() == [[0, 3]]
    assert G.forward(z, 2, G.SIGMOID, mask=np.zeros(6))[0].tolist() == [[-1, -1]]


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences_and_autograd(score, renorm):
    z = _z(5, 12, 3)
    idx, gate, _ = G.forward(z, 4, score, renorm=renorm, scale=2.5)
    dg = np.random.default_rng(4).standard_normal(gate.shape)
    got = G.backward(z, idx, dg, score, renorm, 2.5)
    zt = torch.tensor(z, requires_grad=True)
    p = torch.softmax(zt, -1) if score == G.SOFTMAX else torch.sigmoid(zt)
    s = p.gather(1, torch.tensor(idx))
    g = s / s.sum(-1, keepdim=True) if renorm else s
    (2.5 * g * torch.tensor(dg)).sum().backward()
    assert np.abs(got - zt.grad.numpy()).max() < 1e-12
    h = 1e-6
    for e in (0, int(idx[2, 1]), 11):
        up, dn = z.copy(), z.copy()
        up[2, e] += h
        dn[2, e] -= h

        def loss(v):
            sc = np.array([G.scores(r, score)[0] for r in v])[np.arange(5)[:, None], idx]
            return (2.5 * (sc / sc.sum(-1, keepdims=True) if renorm else sc) * dg).sum()
        assert abs((loss(up) - loss(dn)) / (2 * h) - got[2, e]) < 1e-7


def test_mx4_hand_worked_block():
    v = np.zeros(32)
    v[:10] = [7.9, -6, 5, 3.5, 2.5, 1.25, 0.75, 0.25, -0.26, 0.2]   # largest in [4, 8): scale 1
    codes, e = M.quantize(v)
    assert e.tolist() == [0]
    assert M.values(codes, e)[:10].tolist() == [6, -6, 4, 4, 2, 1, 1, 0, -0.5, 0]
    assert M.quantize(np.zeros(32))[1].tolist() == [-127]
    codes, e = M.quantize(8 * np.ones(32))
    assert e.tolist() == [1] and (M.values(codes, e) == 8).all()
    v[3] = np.inf
    codes, e = M.quantize(v)
    assert e.tolist() == [128] and np.isnan(M.values(codes, e)).all()


def test_mx4_is_the_nearest_element():
    v = np.random.default_rng(5).standard_normal((20, 64)) * 10.0 ** np.random.default_rng(6).integers(-20, 20, (20, 1))
    codes, e = M.quantize(v)
    q = M.values(codes, e)
    s = np.exp2(e.astype(float)).repeat(32, -1)
    grid = np.concatenate((-M.GRID, M.GRID))
    best = np.abs(v[..., None] - s[..., None] * grid).min(-1)
    assert np.allclose(np.abs(q - v), best, rtol=1e-12, atol=0)
    amax = np.abs(v.reshape(20, 2, 32)).max(-1) / np.exp2(e.astype(float))
    assert ((amax >= 4) & (amax < 8)).all()


def test_mx4_experts_with_exact_weights_is_the_dense_layer():
    g = np.random.default_rng(7)
    x, wgu, wdn = g.standard_normal((6, 64)), g.standard_normal((3, 128, 64)), g.standard_normal((3, 64, 64))
    idx = np.array([[0, 1], [1, 0], [-1, 0], [1, 1], [-1, -1], [5, 0]])
    gate = g.random((6, 2))
    y, bound = M.experts(x, idx, gate, wgu, wdn, 1, False)
    want = np.zeros((6, 64))
    f = lambda e, v: wdn[e] @ (M.silu(wgu[e, :64] @ v) * (wgu[e, 64:] @ v))
    for t in range(6):
        want[t] = f(2, x[t])
        for k in range(2):
            if 0 <= idx[t, k] < 2:
                want[t] += gate[t, k] * f(idx[t, k], x[t])
    assert np.abs(y - want).max() < 1e-10 and (bound > 0).all()

"""maskmoe_gate_forward and maskmoe_gate_backward against the fp64 oracle: indices and loads equal, gates and
gradients within a bound derived from fp32 rounding (half a step is U = 2^-24).

Gates: a softmax score is an expf of a difference that is off by U |z - max| and U of its own, over a sum
of up to 256 such terms (8 levels) and a division: (range + 16) U relative; renormalised gates and sigmoids
stay within the same. Gradients: products of up to three such factors and K = 16 terms, relative to
scale * sum |d_gate|, since every weight is at most 1: (3 (range + 16) + 16) U.
"""

import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import gate as G
from paper_2609_34077_amd import _lib as L

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# E, K, n_group, topk_group
SHAPES = [(1, 1, 1, 1), (5, 5, 1, 1), (8, 2, 1, 1), (8, 2, 4, 2), (16, 3, 8, 4), (17, 2, 1, 1), (24, 4, 3, 2), (60, 6, 4, 2),
          (64, 6, 1, 1), (64, 16, 32, 16), (64, 8, 8, 4), (65, 3, 5, 2), (100, 8, 10, 3), (128, 6, 2, 1), (160, 6, 8, 3),
          (255, 16, 51, 8), (256, 8, 8, 4), (256, 16, 128, 8), (256, 1, 256, 1), (256, 8, 1, 1)]
RULES = [dict(), dict(bias=True), dict(prior=True), dict(bias=True, mask=True, group_rule=G.GROUP_SUM2),
         dict(mask=True, group_rule=G.GROUP_SUM2, renorm=False), dict(bias=True, prior=True, renorm=False, scale=2.5)]


def make(T, E, seed, rule, score):
    g = np.random.default_rng(seed)
    z = (1.3 * g.standard_normal((T, E))).astype(np.float32)
    kw = {k: v for k, v in rule.items() if k not in ("bias", "mask", "prior")}
    if rule.get("bias"):
        kw["bias"] = (0.05 if score == G.SIGMOID else 0.3 / E) * g.standard_normal(E).astype(np.float32)
    if rule.get("prior"):
        kw["prior"] = np.exp(g.standard_normal(E)).astype(np.float32)
    if rule.get("mask"):
        kw["mask"] = (g.random(E) < 0.6).astype(np.uint8)
    return z, kw


def run(z, K, score, **kw):
    b = kw.pop("bias", None)
    out = L.maskmoe_gate_forward(torch.from_numpy(z).cuda(), K, score, with_load=True,
                                 bias=None if b is None else torch.from_numpy(np.asarray(b, np.float32)).cuda(), **kw)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in out]


def check(z, K, score, **kw):
    idx, gate, load = run(z, K, score, **kw)
    io, go, lo = G.forward(z, K, score, **kw)
    assert np.array_equal(idx, io), (np.flatnonzero((idx != io).any(1))[:5], idx[(idx != io).any(1)][:2], io[(idx != io).any(1)][:2])
    assert np.array_equal(load, lo)
    fin = np.where(np.isfinite(z), z, 0)
    rel = (fin.max() - fin.min() + 16) * U
    assert (np.abs(gate - go) <= rel * np.abs(go) + 1e-37).all(), np.abs(gate - go).max()
    return idx, gate


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("E,K,ng,tg", SHAPES)
def test_forward(E, K, ng, tg, score):
    for i, rule in enumerate(RULES):
        T = (1, 37, 200)[i % 3]
        say(f"gate E={E} K={K} groups {ng}/{tg} score {score} rule {i} T={T}")
        z, kw = make(T, E, 100 * E + i, rule, score)
        check(z, K, score, n_group=ng, topk_group=tg, **kw)


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
def test_equal_and_nearly_equal_keys(score):
    """Ties go to the lower expert and group; differences below fp32's resolution of a key still count."""
    g = np.random.default_rng(3)
    z = np.round(g.standard_normal((64, 256)) * 2) / 2    # many equal logits
    z = z.astype(np.float32)
    kw = dict(n_group=8, topk_group=4, group_rule=G.GROUP_SUM2)
    for bias in (np.zeros(256, np.float32), np.full(256, 0.125, np.float32)):
        check(z, 8, score, bias=bias, **kw)
    check(np.zeros((3, 256), np.float32), 8, score, bias=np.zeros(256, np.float32), **kw)
    check(np.zeros((3, 64), np.float32), 6, score)
    near = (0.5 + 1e-7 * g.integers(-4, 5, (64, 256))).astype(np.float32)   # steps of 6e-8
    check(near, 8, score, bias=np.full(256, 0.7, np.float32), **kw)
    check(near, 8, score, prior=np.full(256, 0.3, np.float32))
    # a bias that cancels the difference of two scores but for the bits that fp32 keys lose
    z = np.array([[0.3, -0.4] + [-9.0] * 6] * 4, np.float32)
    z[:, 1] = np.nextafter(z[:, 1], [np.float32(9), np.float32(-9), np.float32(-0.4), np.float32(9)])
    s = G.scores(z[2], score)[0]
    bias = np.zeros(8, np.float32)
    bias[1] = s[0] - s[1]
    check(z, 2, score, bias=bias)


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("E", [8, 64, 256])
def test_infinities_nan_and_rows_without_experts(E, score):
    g = np.random.default_rng(E)
    z = (1.3 * g.standard_normal((40, E))).astype(np.float32)
    z[0] = -np.inf
    z[1] = np.nan
    z[2, :] = np.finfo(np.float32).min
    z[3, 1:] = -np.inf
    z[4, : E // 2] = np.nan
    z[5, 3] = np.inf
    z[6, [2, 5]] = np.inf
    z[7] = -200.0 - np.arange(E) / 64       # every sigmoid underflows
    z[8] = 200.0 + np.arange(E) / 64
    z[9, 0] = np.finfo(np.float32).max
    mask = np.ones(E, np.uint8)
    mask[1::3] = 0
    z[10:20, 1] = np.inf                       # masked places
    z[20:30, 4] = np.nan
    for kw in (dict(), dict(mask=mask), dict(mask=np.zeros(E, np.uint8)), dict(n_group=4, topk_group=2, mask=mask)):
        idx, gate = check_special(z, 4, score, **kw)
        if kw.get("mask") is not None and not kw["mask"].any():
            assert (idx == -1).all() and (gate == 0).all()


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("E", [32, 256])
def test_largest_and_smallest_priors_and_biases(E, score):
    g = np.random.default_rng(E)
    z, _ = make(60, E, E, {}, score)
    low = (2.0 ** -100 * g.uniform(1, 2, E)).astype(np.float32)
    high = (2.0 ** 100 * g.uniform(0.5, 1, E)).astype(np.float32)
    for prior in (low, high, np.where(g.random(E) < 0.5, low, high)):
        check(z, 6, score, prior=prior)
        check(z, 6, score, prior=prior, bias=np.where(g.random(E) < 0.1, 2.0 ** 100, -1.0).astype(np.float32), n_group=8,
              topk_group=4, group_rule=G.GROUP_SUM2)


def check_special(z, K, score, **kw):
    """As check, with the gates' bound by the row's own finite range."""
    idx, gate, load = run(z, K, score, **kw)
    with np.errstate(over="ignore", invalid="ignore"):
        io, go, lo = G.forward(z, K, score, **kw)
    assert np.array_equal(idx, io) and np.array_equal(load, lo)
    assert np.isfinite(gate).all()
    # a sigmoid of a large negative logit is subnormal in fp32; softmax terms too
    assert (np.abs(gate - go) <= (24 + 220) * U * np.abs(go) + 1e-37).all()
    return idx, gate


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("E,K,T", [(1, 1, 3), (8, 2, 1), (16, 16, 33), (60, 6, 50), (64, 6, 129), (128, 8, 40), (256, 8, 200),
                                   (255, 16, 31)])
def test_backward(E, K, T, renorm, score):
    say(f"gate backward E={E} K={K} T={T} renorm={renorm} score={score}")
    g = np.random.default_rng(E + T)
    z = (1.3 * g.standard_normal((T, E))).astype(np.float32)
    idx = G.forward(z, K, score)[0]
    idx[0, 0] = -1
    idx[T // 2, K - 1] = E + 5
    if K > 1:
        idx[T - 1, 1] = idx[T - 1, 0]            # the same expert twice
    if T > 4:
        z[3, idx[3, 0]] = -np.inf                # an entry without a logit
        z[4, (idx[4, 0] + 1) % E] = np.nan
    dg = g.standard_normal((T, K)).astype(np.float32)
    dz = L.maskmoe_gate_backward(torch.from_numpy(z).cuda(), torch.from_numpy(idx.astype(np.int32)).cuda(),
                                 torch.from_numpy(dg).cuda(), score, renorm=renorm, scale=2.5)
    torch.cuda.synchronize()
    want = G.backward(z, idx, dg, score, renorm, 2.5)
    fin = np.where(np.isfinite(z), z, 0)
    tol = (3 * (fin.max() - fin.min() + 16) + 16) * U * 2.5 * np.abs(dg).sum(1, keepdims=True)
    assert (np.abs(dz.cpu().numpy() - want) <= tol + 1e-37).all()


def test_empty_batch():
    z = torch.empty((0, 64), device="cuda")
    idx, gate, load = L.maskmoe_gate_forward(z, 6, L.SCORE_SIGMOID, with_load=True)
    assert idx.shape == (0, 6) and (load == 0).all()
    assert L.maskmoe_gate_backward(z, idx, gate, L.SCORE_SIGMOID).shape == (0, 64)


def test_many_tokens_and_unaligned_rows():
    """More tokens than one round of workgroups; logits that start off a 16-byte border."""
    say("gate 20011 tokens")
    z, kw = make(20011, 64, 5, dict(bias=True), G.SIGMOID)
    flat = torch.empty(z.size + 1, device="cuda")
    odd = flat[1:].view(z.shape)
    odd.copy_(torch.from_numpy(z))
    bias = torch.from_numpy(kw["bias"]).cuda()
    a = L.maskmoe_gate_forward(odd, 6, L.SCORE_SIGMOID, bias=bias, with_load=True)
    b = L.maskmoe_gate_forward(odd.clone(), 6, L.SCORE_SIGMOID, bias=bias, with_load=True)
    assert all(torch.equal(u, v) for u, v in zip(a, b))
    io, _, lo = G.forward(z[::97], 6, G.SIGMOID, bias=kw["bias"])
    assert np.array_equal(a[0][::97].cpu().numpy(), io)
    assert int(a[2].sum()) == 20011 * 6
    assert torch.equal(a[2], torch.bincount(a[0].reshape(-1).long(), minlength=64).int())


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("E,K,ng,tg", [(65, 12, 5, 3), (100, 10, 10, 5), (160, 6, 8, 3), (256, 8, 8, 4), (256, 16, 1, 1),
                                       (256, 11, 1, 1), (255, 16, 51, 40), (256, 16, 128, 12)])
def test_many_tokens_above_64_experts(E, K, ng, tg, score):
    """Several tokens of a wavefront ranked at once, the last ones fewer: as in batches too small for that, and as
    the oracle for a sample and the last rows. Rows without a finite logit, and rows of equal ones, among them."""
    T = 9001
    for i, rule in enumerate((RULES[0], RULES[3], RULES[5])):
        say(f"gate T={T} E={E} K={K} groups {ng}/{tg} score {score} rule {i}")
        z, kw = make(T, E, E + K + i, rule, score)
        z[5::1000] = -np.inf
        z[6::1000, E // 4:] = np.nan
        z[7::1000] = 0.25
        kw.update(n_group=ng, topk_group=tg)
        idx, gate, load = run(z, K, score, **kw)
        parts = [run(z[at:at + 4000], K, score, **kw) for at in (0, 4000, 8000)]
        assert np.array_equal(idx, np.concatenate([p[0] for p in parts]))
        assert np.array_equal(gate, np.concatenate([p[1] for p in parts]))
        assert np.array_equal(load, sum(p[2] for p in parts))
        pick = np.unique(np.r_[np.arange(0, T, 211), 1005:1008, T - 5:T])
        io, go, _ = G.forward(z[pick], K, score, **kw)
        assert np.array_equal(idx[pick], io)
        fin = np.where(np.isfinite(z), z, 0)
        assert (np.abs(gate[pick] - go) <= (fin.max() - fin.min() + 16) * U * np.abs(go) + 1e-37).all()


def test_logits_past_32_bit_offsets():
    """More than 2^32 bytes of logits, forward and both gradients: the last rows as they are alone."""
    T, E, K, last = (1 << 24) + 77, 72, 6, 300
    say(f"gate T={T} E={E}")
    z = torch.randn((1 << 16, E), device="cuda").repeat(257, 1)[:T].contiguous()
    z[-last:] = torch.randn((last, E), device="cuda")
    idx, gate, load = L.maskmoe_gate_forward(z, K, L.SCORE_SIGMOID, with_load=True)
    tail = z[-last:].contiguous()
    i, g, _ = L.maskmoe_gate_forward(tail, K, L.SCORE_SIGMOID)
    assert torch.equal(idx[-last:], i) and torch.equal(gate[-last:], g)
    assert int(load.sum()) == T * K and torch.equal(idx[: 1 << 16], idx[1 << 23:(1 << 23) + (1 << 16)])
    for score, renorm in ((L.SCORE_SIGMOID, True), (L.SCORE_SOFTMAX, False)):
        dz = L.maskmoe_gate_backward(z, idx, gate, score, renorm=renorm)
        assert torch.equal(dz[-last:], L.maskmoe_gate_backward(tail, i, g, score, renorm=renorm))
        assert torch.equal(dz[: 1 << 16], dz[1 << 23:(1 << 23) + (1 << 16)])
        del dz


def test_captured_and_replayed_with_other_work():
    say("gate graph")
    z, kw = make(3000, 256, 9, dict(bias=True), G.SIGMOID)
    zt, bias = torch.from_numpy(z).cuda(), torch.from_numpy(kw["bias"]).cuda()
    args = dict(bias=bias, n_group=8, topk_group=4, group_rule=L.GROUP_SUM2, with_load=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        L.maskmoe_gate_forward(zt, 8, L.SCORE_SIGMOID, **args)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = L.maskmoe_gate_forward(zt, 8, L.SCORE_SIGMOID, **args)
        dz = L.maskmoe_gate_backward(zt, out[0], out[1], L.SCORE_SIGMOID)
    for i in range(4):
        zt.copy_(torch.from_numpy(np.roll(z, i + 1, 0)))
        graph.replay()
        torch.cuda.synchronize()
        want = L.maskmoe_gate_forward(zt, 8, L.SCORE_SIGMOID, **args)
        assert all(torch.equal(u, v) for u, v in zip(out, want))
        assert torch.equal(dz, L.maskmoe_gate_backward(zt, want[0], want[1], L.SCORE_SIGMOID))


def test_python_refusals():
    z = torch.zeros((4, 64), device="cuda")
    for bad in (z.double(), z.t(), z.cpu(), z[0]):
        with pytest.raises(ValueError):
            L.maskmoe_gate_forward(bad, 2, L.SCORE_SOFTMAX)
    with pytest.raises(ValueError):
        L.maskmoe_gate_forward(z, 2, L.SCORE_SOFTMAX, bias=torch.zeros(63, device="cuda"))
    with pytest.raises(L.MaskMoEError):
        L.maskmoe_gate_forward(z, 17, L.SCORE_SOFTMAX)
    with pytest.raises(ValueError):
        L.maskmoe_gate_backward(z, torch.zeros((4, 2), dtype=torch.int64, device="cuda"), z[:, :2].contiguous(), 0)


def fastest(calls, reps=9, n=20):
    """Shortest mean time (us) of n calls of each, the calls timed in turn."""
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    best = [float("inf")] * len(calls)
    for f in calls:
        f()
    for _ in range(reps):
        for i, f in enumerate(calls):
            torch.cuda.synchronize()
            start.record()
            for _ in range(n):
                f()
            end.record()
            end.synchronize()
            best[i] = min(best[i], start.elapsed_time(end) / n * 1e3)
    return best


# groups of 3, 5, 6 or 7 lanes (V experts each: 1 up to 16 experts, 4 up to 64), with lanes past the last expert
ODD_GROUPS = [(6, 2, 2, 1), (9, 3, 3, 2), (12, 2, 4, 1), (12, 4, 4, 2), (14, 3, 2, 1), (15, 4, 3, 2), (24, 4, 2, 1), (36, 6, 3, 2),
              (40, 8, 2, 1), (48, 4, 4, 2), (56, 4, 2, 1), (60, 6, 5, 2), (60, 16, 5, 4)]


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("E,K,ng,tg", ODD_GROUPS)
def test_groups_of_odd_numbers_of_lanes(E, K, ng, tg, score):
    for i, rule in enumerate(RULES):
        say(f"gate odd groups E={E} K={K} groups {ng}/{tg} score {score} rule {i}")
        z, kw = make((37, 200)[i % 2], E, 10 * E + i, rule, score)
        check(z, K, score, n_group=ng, topk_group=tg, **kw)


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("E,K,ng", [(24, 2, 2), (48, 4, 4), (60, 4, 5)])
def test_keeping_the_last_group_costs_no_more_than_the_first(E, K, ng, score):
    """The row's own work is the same whichever group leads; selecting every row again in fp64 takes 1.5 to 2.1
    times as long."""
    say(f"gate time of the last group E={E} groups {ng} score {score}")
    z = torch.from_numpy(make(65536, E, E, {}, score)[0]).cuda()
    bias = torch.zeros((2, E), device="cuda")
    bias[0, : E // ng] = bias[1, E - E // ng:] = 1.0
    calls = [lambda b=b: L.maskmoe_gate_forward(z, K, score, n_group=ng, topk_group=1, group_rule=L.GROUP_SUM2, bias=b)
             for b in bias]
    first, last = fastest(calls)
    assert last <= 1.25 * first, (first, last)


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("E,K,ng,tg", [(8, 2, 1, 1), (60, 4, 1, 1), (60, 6, 5, 2), (160, 6, 1, 1), (160, 6, 8, 3)])
def test_priors_and_biases_of_masked_experts(E, K, ng, tg, score):
    """Small priors, and masked experts with priors and biases at the ends of their ranges: they have no key."""
    say(f"gate masked priors and biases E={E} groups {ng}/{tg} score {score}")
    z, _ = make(150, E, E + ng, {}, score)
    g = np.random.default_rng(E)
    mask = np.ones(E, np.uint8)
    mask[::2] = 0
    out = mask == 0
    kw = dict(n_group=ng, topk_group=tg, group_rule=G.GROUP_SUM2)
    for unit in (2.0 ** -100, 2.0 ** -20, 1.0 / E):
        prior = (unit * g.uniform(0.5, 1, E)).clip(2.0 ** -100).astype(np.float32)
        check(z, K, score, prior=prior, **kw)
        check(z, K, score, prior=np.where(out, np.float32(2.0 ** 100), prior), mask=mask, **kw)
        check(z, K, score, prior=prior, mask=mask, bias=np.where(out, -(2.0 ** 100), unit * g.standard_normal(E)).astype(np.float32), **kw)


@pytest.mark.parametrize("E", [60, 160])
def test_what_has_no_key_costs_no_second_selection(E):
    """A factor of every prior, and the prior and bias of masked experts, leave the selection as it is; so the time too.
    Selecting every row again in fp64 takes 1.9 to 2.9 times as long."""
    say(f"gate time of priors E={E}")
    z, kw = make(65536, E, E, dict(bias=True), G.SIGMOID)
    z, mask = torch.from_numpy(z).cuda(), np.ones(E, np.uint8)
    mask[::2] = 0
    far = np.where(mask, kw["bias"], -1e30).astype(np.float32)
    bias = [torch.from_numpy(b).cuda() for b in (kw["bias"], far)]
    one, few = np.ones(E, np.float32), np.full(E, 2.0 ** -20, np.float32)
    calls = [lambda k=k: L.maskmoe_gate_forward(z, 4, L.SCORE_SIGMOID, **k) for k in (
        dict(prior=one), dict(prior=few), dict(mask=mask, bias=bias[0]), dict(mask=mask, bias=bias[1]),
        dict(mask=mask, prior=one), dict(mask=mask, prior=np.where(mask, one, np.float32(2.0 ** 100))))]
    for f in (0, 2, 4):
        assert all(torch.equal(u, v) for u, v in zip(calls[f]()[:1], calls[f + 1]()[:1]))
    us = fastest(calls)
    for f in (0, 2, 4):
        assert us[f + 1] <= 1.25 * us[f], us


@pytest.mark.parametrize("score", [G.SOFTMAX, G.SIGMOID])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("E", [8, 64, 100, 256])
def test_backward_of_infinities_nan_and_saturated_scores(E, renorm, score):
    """The forward's special rows. An unnormalised weight e^-v is off by (v + 2) 2^-23 relative, so by at most 4 U of the
    largest weight whatever v; its sum (256 terms, 8 levels), the division and the sums over K = 4 entries stay within
    16 U more, for each of three factors: (3 * 16 + 16) U of scale * sum |d_gate|, as test_backward's for a range of 0.
    Renormalised sigmoids are not relative to the largest one above -30, where e^-z is off by (30 + 2) 2^-23 = 64 U: 80."""
    say(f"gate backward special rows E={E} renorm={renorm} score={score}")
    K, scale = 4, 2.5
    g = np.random.default_rng(E)
    z = (1.3 * g.standard_normal((40, E))).astype(np.float32)
    z[0] = -np.inf
    z[1] = np.nan
    z[2] = np.finfo(np.float32).min
    z[3, 1:] = -np.inf
    z[4, : E // 2] = np.nan
    z[5, 3] = np.inf
    z[6, [2, 5]] = np.inf
    z[7] = -200.0 - np.arange(E) / 64       # every sigmoid underflows
    z[8] = 200.0 + np.arange(E) / 64
    z[9, 0] = np.finfo(np.float32).max
    z[10:20, 1] = np.inf
    z[20:30, 4] = np.nan
    z[30:34] *= 30
    z[34] = -29.9 - np.arange(E) / 16       # across the border below which sigmoids are taken as e^z
    chosen = G.forward(z, K, score)[0]
    any4 = np.argsort(g.random((40, E)), 1)[:, :K]             # entries without a logit among them
    dg = g.standard_normal((40, K)).astype(np.float32)
    for idx in (chosen, any4, np.repeat(any4[:, :1], K, 1)):
        dz = L.maskmoe_gate_backward(torch.from_numpy(z).cuda(), torch.from_numpy(idx.astype(np.int32)).cuda(),
                                     torch.from_numpy(dg).cuda(), score, renorm=renorm, scale=scale).cpu().numpy()
        with np.errstate(over="ignore", invalid="ignore"):
            want = G.backward(z, idx, dg, score, renorm, scale)
        assert np.isfinite(want).all() and np.isfinite(dz).all()
        factor = 80 if renorm and score == G.SIGMOID else 16
        tol = (3 * factor + 16) * U * scale * np.abs(dg).sum(1, keepdims=True)
        assert (np.abs(dz - want) <= tol + 1e-37).all(), np.abs(dz - want).max()
        assert (dz[:2] == 0).all()


@pytest.mark.parametrize("E", [8, 256])
def test_renormalised_sigmoids_far_below_the_largest(E):
    """Gates are ratios of scores, e^-60 as well as 1/2, where a score by itself is 0 in fp32. Relative bounds: a weight is
    off by (range + 16) U as in the forward's tests; a gradient w (dg - mean) (1 - s) by three such factors."""
    say(f"gate ratios of sigmoids E={E}")
    K, scale = 4, 2.5
    T = 64
    z = np.full((T, E), -np.inf, np.float32)
    z[:, :4] = np.array([0.0, -1.0, -70.0, -86.0]) + np.linspace(-31, 1, T)[:, None]
    z[::2, 2] = -89.0
    z[:, 3] = np.minimum(z[:, 3], -90.0)
    idx, gate, _ = run(z, K, G.SIGMOID, scale=scale)
    io, go, _ = G.forward(z, K, G.SIGMOID, scale=scale)
    fin = z[:, :4].astype(np.float64)
    rel = (fin.max(1, keepdims=True) - fin.min(1, keepdims=True) + 16) * U
    assert np.array_equal(idx, io)
    assert (np.abs(gate - go) <= rel * np.abs(go) + 1e-37).all()
    dg = np.random.default_rng(E).standard_normal((T, K)).astype(np.float32)
    dz = L.maskmoe_gate_backward(torch.from_numpy(z).cuda(), torch.from_numpy(io.astype(np.int32)).cuda(),
                                 torch.from_numpy(dg).cuda(), G.SIGMOID, scale=scale).cpu().numpy()
    want = G.backward(z, io, dg, G.SIGMOID, True, scale)
    t = np.arange(T)[:, None]
    part = np.abs(go) * (np.abs(dg) + (np.abs(go) / scale * np.abs(dg)).sum(1, keepdims=True))
    assert (np.abs(dz - want)[t, io] <= (3 * rel + 16 * U) * part + 1e-37).all()

"""MX4 conversion bit for bit, and the experts on MX4 weights within the bound that the oracle derives from
every rounding on the way (oracle/mx4.py)."""

import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import mx4 as M
from paper_2609_34077_amd import _lib as L

pytestmark = pytest.mark.gpu


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float32)).bfloat16()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (7, 96), (33, 416), (130, 2048), (1, 4096)])
def test_quantize_and_back(rows, cols, dtype):
    say(f"mx4 {rows} x {cols} {dtype}")
    g = np.random.default_rng(rows * cols)
    v = g.standard_normal((rows, cols)) * 10.0 ** g.integers(-44, 38, (rows, cols // 32)).repeat(32, 1)
    v[0, :32] = 0
    v[-1, -32:] = g.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 6.0, 7.99], 32)   # rounding borders
    v[-1, -1] = 7
    x = torch.from_numpy(np.clip(v, -3e38, 3e38).astype(np.float32)).to(dtype)
    codes, scales = L.maskmoe_mx4_quantize(x.cuda())
    co, eo = M.quantize(x.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), eo + 127)
    assert np.array_equal(codes.cpu().numpy(), M.pack_codes(co))
    want = torch.from_numpy(M.values(co, eo))
    for dt in (torch.float32, torch.bfloat16):
        back = L.maskmoe_mx4_dequantize(codes, scales, dt).cpu()
        assert torch.equal(back, want.to(dt))


def test_every_bf16_value():
    """Each finite bf16 number as the largest of a block, beside one, three quarters and a half of it."""
    bits = torch.arange(0, 0x7F80, dtype=torch.int32).to(torch.int16)
    top = bits.view(torch.bfloat16).float()
    x = (top[:, None] * torch.linspace(-1, 1, 32)).bfloat16()
    x[:, 31] = top.bfloat16()
    codes, scales = L.maskmoe_mx4_quantize(x.cuda())
    co, eo = M.quantize(x.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), eo + 127) and np.array_equal(codes.cpu().numpy(), M.pack_codes(co))


def test_infinities_and_nan_stay_in_their_block():
    x = torch.ones((4, 96))
    x[0, 5], x[1, 40], x[2, 95] = float("inf"), float("nan"), float("-inf")
    codes, scales = L.maskmoe_mx4_quantize(x.cuda())
    back = L.maskmoe_mx4_dequantize(codes, scales, torch.float32).cpu()
    bad = torch.zeros((4, 3), dtype=torch.bool)
    bad[0, 0] = bad[1, 1] = bad[2, 2] = True
    assert torch.equal(back.isnan().view(4, 3, 32).all(-1), bad) and torch.equal(back.isnan().view(4, 3, 32).any(-1), bad)
    assert torch.equal(scales.cpu() == 255, bad) and (codes.cpu().view(4, 3, 16)[bad] == 0).all()


def make(T, d, F, E, K, ns, seed, pad=0):
    g = np.random.default_rng(seed)
    n = E + ns
    x = bf16(g.standard_normal((T, d)) * np.where(g.random(d) < 0.05, 6, 1))
    wq, dev = [], []
    for shape in ((n, 2 * F, d), (n, d, F)):
        c, e = M.quantize(g.standard_normal(shape) * shape[-1] ** -0.5 * 2.0 ** g.integers(-1, 2, shape[:2] + (1,)))
        wq.append(M.values(c, e))
        dev += [torch.from_numpy(M.pack_codes(c)).cuda(), torch.from_numpy((e + 127).astype(np.uint8)).cuda()]
    idx = np.argsort(-(g.standard_normal((T, E)) + np.linspace(0, 2, E)), 1)[:, :K].astype(np.int32)
    gate = g.random((T, K)).astype(np.float32)
    if pad:
        idx[T - pad:] = -1
    return x, wq, dev, idx, gate


def call(x, dev, idx, gate, ns, act, **kw):
    packed = L.maskmoe_mx4_pack_experts(*dev)
    return L.maskmoe_experts_forward_mx4(x.cuda(), torch.from_numpy(idx).cuda(), torch.from_numpy(gate).cuda(), packed,
                                         n_shared=ns, act=act, **kw)


def check(x, wq, dev, idx, gate, ns, act):
    y = call(x, dev, idx, gate, ns, act).double().cpu().numpy()
    want, bound = M.experts(x.double().numpy(), idx, gate, *wq, ns, act == L.ACT_MX4)
    worst = (np.abs(y - want) / (bound + 1e-300)).max()
    assert worst <= 1, worst
    return y


# T, d, F, E, K, shared, empty slots at the end
LAYERS = [(1, 64, 64, 1, 1, 0, 0), (1, 128, 192, 8, 2, 0, 0), (2, 192, 64, 4, 2, 1, 1), (5, 256, 320, 64, 6, 2, 0),
          (16, 320, 128, 8, 2, 0, 3), (17, 64, 576, 3, 3, 0, 0), (33, 512, 256, 5, 2, 0, 2), (64, 128, 128, 2, 1, 1, 0),
          (65, 192, 64, 2, 2, 0, 0), (100, 256, 512, 8, 2, 0, 7), (130, 64, 64, 256, 16, 0, 0), (200, 384, 448, 4, 2, 2, 0),
          (300, 128, 1408, 16, 4, 1, 11), (700, 640, 192, 3, 2, 0, 0), (1100, 192, 256, 8, 2, 1, 50)]


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T,d,F,E,K,ns,pad", LAYERS)
def test_experts(T, d, F, E, K, ns, pad, act):
    say(f"mx4 experts T={T} d={d} F={F} E={E} K={K} shared={ns} pad={pad} act={act}")
    x, wq, dev, idx, gate = make(T, d, F, E, K, ns, T + d + F, pad)
    y = check(x, wq, dev, idx, gate, ns, act)
    if pad and not ns:
        assert (y[T - pad:] == 0).all()


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T", [1, 16, 17, 40])
def test_most_experts_entries_and_shared_experts(T, act):
    """E = 256, K = 16 and 8 shared experts; then no token with an expert, with and without shared ones."""
    say(f"mx4 limits T={T} act={act}")
    x, wq, dev, idx, gate = make(T, 64, 64, 256, 16, 8, T)
    idx = np.random.default_rng(T).permuted(np.tile(np.arange(256, dtype=np.int32), (T, 1)), axis=1)[:, :16].copy()
    check(x, wq, dev, idx, gate, 8, act)
    idx[:] = -1
    check(x, wq, dev, idx, gate, 8, act)
    routed = [t[:256].contiguous() for t in dev]
    assert (call(x, routed, idx, gate, 0, act) == 0).all()


# the same with enough rows and columns that 256 x 256 tiles cover the chip (the last: with MX4 activations alone)
WIDE = [(2100, 64, 4096, 1, 1, 0, 0), (900, 192, 4160, 2, 2, 1, 37), (700, 320, 4160, 3, 2, 1, 0), (1500, 448, 4160, 2, 1, 0, 1),
        (210, 128, 4160, 16, 2, 0, 5)]


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T,d,F,E,K,ns,pad", WIDE)
def test_experts_on_wide_tiles(T, d, F, E, K, ns, pad, act):
    say(f"mx4 wide T={T} d={d} F={F} E={E} K={K} shared={ns} pad={pad} act={act}")
    x, wq, dev, idx, gate = make(T, d, F, E, K, ns, T + d + F, pad)
    bad = (T // 3, T - pad - 1)
    y = check(x, wq, dev, idx, gate, ns, act)
    if pad and not ns:
        assert (y[T - pad:] == 0).all()
    clean = torch.from_numpy(y)
    x[bad[0], 7], x[bad[1], d - 1] = float("nan"), float("inf")     # they stay in their tokens
    y2 = call(x, dev, idx, gate, ns, act).cpu().double()
    rows = torch.ones(T, dtype=torch.bool)
    rows[list(bad)] = False
    assert torch.equal(y2[rows], clean[rows]) and not y2[~rows].isfinite().any()


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T", [1, 7, 40, 300])
def test_uneven_and_odd_routing(T, act):
    """All tokens to one expert; experts named twice; indices outside the experts; no expert at all."""
    say(f"mx4 experts routing T={T} act={act}")
    x, wq, dev, idx, gate = make(T, 128, 192, 6, 2, 0, T)
    idx[:] = [4, 4]
    check(x, wq, dev, idx, gate, 0, act)
    idx[:, 0], idx[:, 1] = np.arange(T) % 9 - 2, 2 ** 31 - 1 - np.arange(T) % 3
    check(x, wq, dev, idx, gate, 0, act)
    idx[:] = np.iinfo(np.int32).min
    assert (check(x, wq, dev, idx, gate, 0, act) == 0).all()
    x2, wq2, dev2, idx2, gate2 = make(T, 128, 192, 4, 2, 2, T)
    idx2[:] = -1
    check(x2, wq2, dev2, idx2, gate2, 2, act)


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T", [3, 16, 90, 600])
def test_nan_and_infinity_stay_in_their_token(T, act):
    x, wq, dev, idx, gate = make(T, 192, 128, 4, 2, 0, T + 1)
    clean = call(x, dev, idx, gate, 0, act).cpu()
    x[1, 7], x[T - 1, 100] = float("nan"), float("inf")
    y = call(x, dev, idx, gate, 0, act).cpu()
    rows = torch.ones(T, dtype=torch.bool)
    rows[1] = rows[T - 1] = False
    assert torch.equal(y[rows], clean[rows]) and y[1].isnan().all() and not y[T - 1].isfinite().any()


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T", [2, 5, 16, 17, 130])
@pytest.mark.parametrize("at", [0, -1])
def test_a_token_of_nan_beside_rows_of_odd_length(T, at, act):
    """Rows that end inside a 128-column step: nothing of the first or last token's is read in place of their rest."""
    x, wq, dev, idx, gate = make(T, 192, 192, 3, 2, 1, T + 5)
    clean = call(x, dev, idx, gate, 1, act).cpu()
    x[at] = float("nan")
    y = call(x, dev, idx, gate, 1, act).cpu()
    rows = torch.ones(T, dtype=torch.bool)
    rows[at] = False
    assert torch.equal(y[rows], clean[rows]) and y[at].isnan().all()


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T", [2, 40, 520])
def test_scales_at_their_ends(T, act):
    """Weight blocks with the smallest scales (bytes 0 and 1), a large one, and NaN scales of one expert."""
    x, wq, dev, idx, gate = make(T, 128, 64, 4, 1, 0, T + 2)
    idx[:, 0] = np.arange(T) % 4
    gu, sc = dev[0].cpu().numpy(), dev[1].cpu().numpy()
    sc[0, :, 0], sc[0, :, 1], sc[1, :, 2] = 0, 1, 150
    sc[3, 0, 0] = 255
    dev[1] = torch.from_numpy(sc).cuda()
    codes = np.empty((4, 128, 128), np.int64)
    codes[..., 0::2], codes[..., 1::2] = gu & 15, gu >> 4
    wq[0] = M.values(codes, sc.astype(np.int64) - 127)
    y = call(x, dev, idx, gate, 0, act).double().cpu().numpy()
    want, bound = M.experts(x.double().numpy()[idx[:, 0] < 3], idx[idx[:, 0] < 3], gate[idx[:, 0] < 3], *wq, 0, act == L.ACT_MX4)
    assert (np.abs(y[idx[:, 0] < 3] - want) <= bound + 1e-37).all()
    assert np.isnan(y[idx[:, 0] == 3]).all()


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T,F", [(4, 320), (100, 320), (900, 320), (1400, 4160)])
def test_dirty_workspace_streams_and_graphs(T, F, act):
    """The workspace's contents do not matter; calls on two streams with a workspace each; captured and replayed
    with other work between; the same bits every time."""
    say(f"mx4 experts graph T={T} act={act}")
    E, K, ns, d = 8, 2, 1, 256
    x, wq, dev, idx, gate = make(T, d, F, E, K, ns, T + 3)
    packed = L.maskmoe_mx4_pack_experts(*dev)
    xs, it, gt = x.cuda(), torch.from_numpy(idx).cuda(), torch.from_numpy(gate).cuda()
    n = L.maskmoe_experts_mx4_workspace_bytes(T, d, E, K, F, ns)
    ws = [torch.full((n,), fill, dtype=torch.uint8, device="cuda") for fill in (0xFF, 0x7F)]
    f = lambda w, v=xs: L.maskmoe_experts_forward_mx4(v, it, gt, packed, n_shared=ns, act=act, workspace=w)
    ref = f(None)
    assert torch.equal(f(ws[0]), ref) and torch.equal(f(ws[1]), ref)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    torch.cuda.synchronize()
    for s, w in zip(streams, ws):
        with torch.cuda.stream(s):
            outs.append([f(w) for _ in range(5)])
    torch.cuda.synchronize()
    assert all(torch.equal(y, ref) for o in outs for y in o)
    buf = xs.clone()
    y = torch.empty_like(buf)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.maskmoe_experts_forward_mx4(buf, it, gt, packed, n_shared=ns, act=act, workspace=ws[0], y=y)
    for i in range(4):
        buf.copy_(xs.roll(i, 0))
        want = f(None, buf)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_gate_to_experts():
    """As a serving step runs them: logits, gates, the experts on quantised weights, an empty slot in the batch; the
    bf16 layer on the values of the same weights agrees within the bf16 layer's bound."""
    say("mx4 gate -> experts")
    T, d, F, E, K = 50, 256, 192, 64, 6
    g = torch.Generator(device="cuda").manual_seed(1)
    w_gu = torch.randn((E, 2 * F, d), generator=g, device="cuda").mul_(d ** -0.5).bfloat16()
    w_dn = torch.randn((E, d, F), generator=g, device="cuda").mul_(F ** -0.5).bfloat16()
    x = torch.randn((T, d), generator=g, device="cuda").bfloat16()
    wr = torch.randn((E, d), generator=g, device="cuda").mul_(0.1).bfloat16()
    q = L.maskmoe_mx4_quantize(w_gu) + L.maskmoe_mx4_quantize(w_dn)
    packed = L.maskmoe_mx4_pack_experts(*q)
    z = x.float() @ wr.float().t()
    z[T - 1] = float("nan")
    idx, gate, load = L.maskmoe_gate_forward(z, K, L.SCORE_SIGMOID, n_group=8, topk_group=3, group_rule=L.GROUP_SUM2,
                                             bias=0.02 * torch.randn(E, generator=g, device="cuda"), scale=2.5, with_load=True)
    assert int(load.sum()) == (T - 1) * K and (idx[T - 1] == -1).all()
    y = L.maskmoe_experts_forward_mx4(x, idx, gate, packed)
    vals = [L.maskmoe_mx4_dequantize(*q[i:i + 2], torch.float32).double().cpu().numpy() for i in (0, 2)]
    want, bound = M.experts(x.double().cpu().numpy(), idx.cpu().numpy(), gate.cpu().numpy(), *vals, 0, False)
    assert (np.abs(y.double().cpu().numpy() - want) <= bound).all() and (y[T - 1] == 0).all()
    # maskmoe_route's routing drives the same experts; the bf16 layer runs on the values of the blocks
    ri, rg, _ = L.maskmoe_route(x, wr, 2, L.ROUTE_PLAIN, L.GATE_RENORM)
    dense = [L.maskmoe_mx4_dequantize(*q[i:i + 2], torch.bfloat16) for i in (0, 2)]
    yd = L.maskmoe_layer_forward(x, wr, *dense, 2, L.ROUTE_PLAIN, L.GATE_RENORM).float()
    ym = L.maskmoe_experts_forward_mx4(x, ri, rg, packed).float()
    assert (yd - ym).abs().max() <= 2e-2 * yd.abs().max()


def test_blocks_past_32_bit_offsets():
    """More than 2^32 elements: the rows at the end are converted as they are alone."""
    rows, cols = (1 << 17) + 3, 1 << 15
    say(f"mx4 quantize {rows} x {cols}")
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[:] = torch.randn(cols, device="cuda").bfloat16()
    x[-3:] = torch.randn((3, cols), device="cuda").bfloat16()
    codes, scales = L.maskmoe_mx4_quantize(x)
    c, e = L.maskmoe_mx4_quantize(x[-3:].contiguous())
    assert torch.equal(codes[-3:], c) and torch.equal(scales[-3:], e)
    assert torch.equal(codes[: rows - 3], codes[:1].expand(rows - 3, -1))
    back = L.maskmoe_mx4_dequantize(codes, scales, torch.bfloat16)
    assert torch.equal(back[-3:], L.maskmoe_mx4_dequantize(c, e, torch.bfloat16))
    assert torch.equal(back[: rows - 3], back[:1].expand(rows - 3, -1))


def test_experts_past_32_bit_offsets():
    """Weights of more than 2^32 bytes: the last of 256 experts give the bits that the first ones give, which are
    copies of them (with fewer experts in all, a reduction may be split into other parts)."""
    E, d, F, at = 256, 4096, 4096, 250
    say("mx4 experts past 4 GiB")
    g = torch.Generator(device="cuda").manual_seed(4)
    dev = []
    for shape in ((E, 2 * F, d), (E, d, F)):
        dev += [torch.randint(0, 256, shape[:2] + (shape[2] // 2,), dtype=torch.uint8, generator=g, device="cuda"),
                torch.randint(118, 121, shape[:2] + (shape[2] // 32,), dtype=torch.uint8, generator=g, device="cuda")]
    for t in dev:
        t[:E - at] = t[at:]
    packed = L.maskmoe_mx4_pack_experts(*dev)
    del dev
    # few tokens; a batch; wide tiles (rows per expert of all: 6000 / 256 = 23.4)
    for T, act in ((1, L.ACT_BF16), (5, L.ACT_MX4), (40, L.ACT_BF16), (40, L.ACT_MX4), (6000, L.ACT_MX4)):
        say(f"  T={T} act={act}")
        x = torch.randn((T, d), generator=g, device="cuda").bfloat16()
        idx = torch.randint(at, E, (T, 1), dtype=torch.int32, generator=g, device="cuda")
        gate = torch.rand((T, 1), generator=g, device="cuda")
        y = L.maskmoe_experts_forward_mx4(x, idx, gate, packed, act=act)
        assert y.float().abs().max() > 0 and y.isfinite().all()
        assert torch.equal(y, L.maskmoe_experts_forward_mx4(x, idx - at, gate, packed, act=act))


def test_python_refusals():
    x = torch.zeros((4, 64), device="cuda")
    for bad in (x[:, :48], x.half(), x.cpu(), x.t()):
        with pytest.raises((ValueError, TypeError)):
            L.maskmoe_mx4_quantize(bad)
    codes, scales = L.maskmoe_mx4_quantize(x)
    with pytest.raises(ValueError):
        L.maskmoe_mx4_dequantize(codes, scales[:, :1].contiguous(), torch.float32)
    xq, wq, dev, idx, gate = make(4, 64, 64, 2, 1, 0, 0)
    with pytest.raises(ValueError):
        L.maskmoe_mx4_pack_experts(dev[0], dev[1], dev[2][:1].contiguous(), dev[3])
    packed = L.maskmoe_mx4_pack_experts(*dev)
    it, gt = torch.from_numpy(idx).cuda(), torch.from_numpy(gate).cuda()
    with pytest.raises(ValueError):
        L.maskmoe_experts_forward_mx4(xq.cuda().float(), it, gt, packed)
    with pytest.raises(ValueError):
        L.maskmoe_experts_forward_mx4(xq.cuda(), it.long(), gt, packed)
    with pytest.raises(L.MaskMoEError):
        L.maskmoe_experts_forward_mx4(xq.cuda(), it, gt, packed, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(L.MaskMoEError):
        L.maskmoe_experts_forward_mx4(xq.cuda(), it, gt, packed, act=3)


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T", [4, 40, 1300])
def test_expert_outputs_stay_fp32(T, act):
    """Two experts whose outputs 257 v and -256 v leave v: exact in fp32, 0 where they were rounded to bf16 (257 lies
    between 256 and 258), for few tokens, a batch and enough rows for the wide tiles (2 T / 128 + 1 or 2 T / 256 + 1
    row tiles of 33: 700 and 363). Every step is exact: a = 128 s, SiLU(a) = a to fp32 from 128 on, b = s, so that
    h = 128 s^2 in every column, a block of equal powers of two; v = 128 s^2."""
    say(f"mx4 experts fp32 outputs T={T} act={act}")
    d, F = 128, 4160
    gu = np.zeros((2, 2 * F, d), np.int64)
    gu[:, :, 0] = 2                                            # the code of 1
    eg = np.zeros((2, 2 * F, d // 32), np.int64)
    eg[:, F:] = -7
    dn = np.zeros((2, d, F), np.int64)
    dn[0, :, 5:5 + 128 * 32:32], dn[0, :, F - 1] = 4, 2        # 128 twos and a one
    dn[1, :, 7:7 + 128 * 32:32] = 12                           # 128 times -2
    ed = np.zeros((2, d, F // 32), np.int64)
    dev = []
    for c, e in ((gu, eg), (dn, ed)):
        dev += [torch.from_numpy(M.pack_codes(c)).cuda(), torch.from_numpy((e + 127).astype(np.uint8)).cuda()]
    s = 2.0 ** (np.arange(T) % 3)
    x = np.zeros((T, d))
    x[:, 0] = 128 * s
    idx, gate = np.tile(np.array([0, 1], np.int32), (T, 1)), np.ones((T, 2), np.float32)
    y = call(bf16(x), dev, idx, gate, 0, act).double().cpu().numpy()
    assert (y == (128 * s * s)[:, None]).all()


def taken(T, d, F, E, K, ns, act):
    """The kernels that a call takes, by the rules of csrc/mx4_experts.hip: "few", "wide", or the parts that the batch
    kernels split the down projection's reduction into."""
    rows, G, mx = T * (K + ns), E + ns, act == L.ACT_MX4
    if T <= 16:
        return "few"
    tiles = (rows // (128 if mx else 256) + G // 2) * ((2 * F + 255) // 256)
    if rows >= (22 if mx else 280) * G and tiles >= 256:
        return "wide"
    splits, steps = 1, (F + 127) // 128
    while splits < 8 and min(rows, G) * ((d + 255) // 256) * splits < 512 and steps >= 16 * splits and 2 * splits * rows <= 8192:
        splits *= 2
    return splits


# T, d, F, E, K, shared, empty slots, parts: reductions of 16, 17, 33 and 65 steps, of which the parts start at any step
# and the last one may hold 64 columns
SPLIT = [(17, 64, 2048, 2, 1, 0, 0, 2), (33, 192, 2112, 3, 2, 0, 4, 2), (80, 64, 2112, 2, 2, 1, 5, 2), (24, 320, 2112, 5, 2, 2, 0, 2),
         (40, 192, 4160, 3, 2, 0, 0, 4), (61, 64, 4160, 4, 1, 1, 9, 4), (18, 64, 8256, 2, 1, 0, 1, 8), (70, 128, 8256, 3, 1, 1, 6, 8),
         (80, 64, 8256, 4, 2, 0, 0, 8)]


@pytest.mark.parametrize("act", [L.ACT_BF16, L.ACT_MX4])
@pytest.mark.parametrize("T,d,F,E,K,ns,pad,parts", SPLIT)
def test_batches_with_split_reductions(T, d, F, E, K, ns, pad, parts, act):
    say(f"mx4 split T={T} d={d} F={F} E={E} K={K} shared={ns} pad={pad} parts={parts} act={act}")
    assert taken(T, d, F, E, K, ns, act) == parts
    x, wq, dev, idx, gate = make(T, d, F, E, K, ns, T + d + F, pad)
    y = check(x, wq, dev, idx, gate, ns, act)
    if pad and not ns:
        assert (y[T - pad:] == 0).all()
    x[T // 2, 3] = float("nan")                                # stays in its token
    y2 = call(x, dev, idx, gate, ns, act).cpu().double()
    rows = torch.ones(T, dtype=torch.bool)
    rows[T // 2] = False
    assert torch.equal(y2[rows], torch.from_numpy(y)[rows]) and y2[T // 2].isnan().all()


@pytest.mark.parametrize("T,d,F,E,K,ns,pad,act", [(2100, 448, 4160, 2, 1, 0, 1, L.ACT_BF16), (2300, 576, 2112, 1, 1, 1, 3, L.ACT_BF16),
                                                  (500, 448, 4160, 2, 2, 0, 1, L.ACT_MX4)])
def test_wide_tiles_past_the_matrix(T, d, F, E, K, ns, pad, act):
    """Weight tiles of 256 rows that the matrix ends in, both products."""
    say(f"mx4 wide T={T} d={d} F={F} E={E} K={K} shared={ns} pad={pad} act={act}")
    assert taken(T, d, F, E, K, ns, act) == "wide"
    x, wq, dev, idx, gate = make(T, d, F, E, K, ns, T + d + F, pad)
    y = check(x, wq, dev, idx, gate, ns, act)
    if not ns:
        assert (y[T - pad:] == 0).all()


@pytest.mark.parametrize("n,d,F", [(1, 64, 64), (3, 192, 320), (2, 640, 1088)])
def test_packed_layout(n, d, F):
    """Operand order: fragment f of 16 rows, step s of 128 columns, lane l the block of row l % 16 and columns 128 s +
    32 (l / 16); scales of four steps a dword; gate and up fragments alternate; zeros past the columns."""
    g = np.random.default_rng(n + d + F)
    dev, want = [], []
    for R, C, gate_up in ((2 * F, d, True), (d, F, False)):
        codes = g.integers(0, 256, (n, R, C // 2), dtype=np.uint8)
        scales = g.integers(0, 256, (n, R, C // 32), dtype=np.uint8)
        dev += [torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()]
        steps = (C + 127) // 128
        quads = (steps + 3) // 4
        cb = np.zeros((n, R, 4 * steps, 16), np.uint8)
        cb[:, :, : C // 32] = codes.reshape(n, R, C // 32, 16)
        sb = np.zeros((n, R, 16 * quads), np.uint8)
        sb[:, :, : C // 32] = scales
        if gate_up:   # fragments 2q of W_gate, 2q + 1 of W_up
            order = np.arange(R).reshape(2, R // 32, 16).transpose(1, 0, 2).reshape(-1)
            cb, sb = cb[:, order], sb[:, order]
        want.append(cb.reshape(n, R // 16, 16, steps, 4, 16).transpose(0, 1, 3, 4, 2, 5).reshape(-1))
        want.append(sb.reshape(n, R // 16, 16, quads, 4, 4).transpose(0, 1, 3, 5, 2, 4).reshape(-1))
    packed = L.maskmoe_mx4_pack_experts(*dev)
    for t, w in zip(packed.tensors, want):
        assert np.array_equal(t.cpu().numpy(), w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_code_and_scale(dtype):
    """All 16 codes under all 256 scales; values past the type's range are infinite."""
    byte = np.arange(256)
    codes = np.tile(np.arange(16), (256, 2))
    want = torch.from_numpy(M.values(codes, np.where(byte == 255, 128, byte - 127)[:, None])).to(dtype)
    got = L.maskmoe_mx4_dequantize(torch.from_numpy(M.pack_codes(codes)).cuda(),
                                   torch.from_numpy(byte.astype(np.uint8)[:, None]).cuda(), dtype).cpu()
    assert got[255].isnan().all() and torch.equal(got[:255], want[:255])
    assert got[253:255].isinf().any() and got[:253].isfinite().all()

"""The norm with its residual, its 8-bit output and its gradient within the bounds that the oracle derives from every
rounding on the way (oracle/norm.py), and 8-bit blocks bit for bit (oracle/mx8.py)."""

import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import mx8 as M
from oracle import norm as N
from paper_2609_34077_amd import _lib as L

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float32]


def half(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------- 8-bit blocks

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (7, 96), (33, 416), (130, 2048), (1, 4096)])
def test_quantize_and_back(rows, cols, dtype):
    say(f"mx8 {rows} x {cols} {dtype}")
    g = np.random.default_rng(rows * cols)
    v = g.standard_normal((rows, cols)) * 10.0 ** g.integers(-44, 38, (rows, cols // 32)).repeat(32, 1)
    v[0, :32] = 0
    v[-1, -32:] = (g.integers(-127, 127, 32) + 0.5) / 64   # rounding borders
    v[-1, -1] = 1.9921875
    x = torch.from_numpy(np.clip(v, -3e38, 3e38).astype(np.float32)).to(dtype)
    codes, scales = L.maskmoe_mx8_quantize(x.cuda())
    co, eo = M.quantize(x.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), eo + 127)
    assert np.array_equal(codes.cpu().numpy(), co)
    want = torch.from_numpy(M.values(co, eo))
    for dt in DTYPES:
        back = L.maskmoe_mx8_dequantize(codes, scales, dt).cpu()
        assert torch.equal(back.double(), want)


def test_every_bf16_value_in_blocks():
    """Each finite bf16 number as the largest of a block, beside parts of it."""
    bits = torch.arange(0, 0x7F80, dtype=torch.int32).to(torch.int16)
    top = bits.view(torch.bfloat16).float()
    x = (top[:, None] * torch.linspace(-1, 1, 32)).bfloat16()
    x[:, 31] = top.bfloat16()
    codes, scales = L.maskmoe_mx8_quantize(x.cuda())
    co, eo = M.quantize(x.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), eo + 127) and np.array_equal(codes.cpu().numpy(), co)


def test_every_code_under_every_scale():
    codes = torch.arange(-128, 128, dtype=torch.int16).clamp(min=-127).to(torch.int8).repeat(256, 1)
    scales = torch.arange(256, dtype=torch.int32).to(torch.uint8)[:, None].repeat(1, 8)
    want = codes.double() * torch.exp2(scales.double() - 133).repeat_interleave(32, 1)
    for dt in DTYPES:
        back = L.maskmoe_mx8_dequantize(codes.cuda(), scales.cuda(), dt).cpu().double()
        assert torch.equal(back[:255], want[:255]) and back[255].isnan().all()


def test_infinities_and_nan_stay_in_their_block():
    x = torch.ones((4, 96))
    x[0, 5], x[1, 40], x[2, 95] = float("inf"), float("nan"), float("-inf")
    for dt in DTYPES:
        codes, scales = L.maskmoe_mx8_quantize(x.to(dt).cuda())
        back = L.maskmoe_mx8_dequantize(codes, scales, torch.float32).cpu()
        bad = torch.zeros((4, 3), dtype=torch.bool)
        bad[0, 0] = bad[1, 1] = bad[2, 2] = True
        assert torch.equal(back.isnan().view(4, 3, 32).all(-1), bad) and torch.equal(back.isnan().view(4, 3, 32).any(-1), bad)
        assert torch.equal(scales.cpu() == 255, bad) and (codes.cpu().view(4, 3, 32)[bad] == 0).all()


def test_no_rows():
    codes, scales = L.maskmoe_mx8_quantize(torch.empty((0, 64), device="cuda"))
    assert codes.shape == (0, 64) and scales.shape == (0, 2)
    assert L.maskmoe_mx8_dequantize(codes, scales, torch.bfloat16).shape == (0, 64)


# ---------------------------------------------------------------- the norm

def inputs(T, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    loud = 1 + 7 * (torch.rand(d, generator=g) < 0.03)
    r = lambda s: (torch.randn((T, d), generator=g) * s).to(dtype)   # noqa: E731
    return dict(x=r(0.4 * loud), residual=r(2 * loud), weight=(1 + 0.2 * torch.randn(d, generator=g)).to(dtype),
                dy=r(0.05), d_hidden=r(0.05))


def check_forward(v, dtype, eps, residual, mx8, got):
    y, hidden, codes, scales = got
    s, b_h, want, e_y, b_y = N.forward(f64(v["x"]), f64(v["residual"]) if residual else None, f64(v["weight"]), eps,
                                       half(dtype))
    tiny = 2.0 ** -130   # below the smallest normal numbers
    if y is not None:
        assert (np.abs(f64(y) - want) <= b_y + tiny).all()
    if residual:
        assert (np.abs(f64(hidden) - s) <= b_h + tiny).all()
    else:
        assert hidden is None
    if mx8:
        worst, exps = M.off_by(want, e_y + tiny, codes.cpu().numpy().astype(np.int64), scales.cpu().numpy().astype(np.int64) - 127)
        assert worst <= 0 and exps


SHAPES = [(1, 1), (1, 4096), (2, 8), (3, 7), (5, 63), (4, 64), (9, 65), (1, 32), (7, 96), (3, 512), (6, 520), (5, 1000),
          (4, 1024), (3, 1025), (33, 2048), (3, 2056), (5, 4096), (4, 4104), (3, 8192), (2, 8193), (2, 16384), (2, 20000),
          (1, 32768), (2500, 64), (9000, 24), (2100, 544),
          # last pieces that are not whole, in every number of threads a row
          (3, 9), (2, 15), (3, 511), (3, 513), (4, 1031), (600, 2047), (3, 2049), (3, 4095), (2, 4097), (2, 8191), (2, 16383),
          (1, 16385), (1, 32767)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward(T, d, dtype):
    say(f"norm forward T={T} d={d} {dtype}")
    v = inputs(T, d, dtype, T + d)
    c = {k: t.cuda() for k, t in v.items()}
    for residual in (True, False):
        for mx8 in (False, True) if d % 32 == 0 else (False,):
            got = L.maskmoe_norm_forward(c["x"], c["weight"], residual=c["residual"] if residual else None, eps=1e-5,
                                         with_mx8=mx8)
            check_forward(v, dtype, 1e-5, residual, mx8, got)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", SHAPES)
def test_backward(T, d, dtype):
    say(f"norm backward T={T} d={d} {dtype}")
    v = inputs(T, d, dtype, T * d)
    c = {k: t.cuda() for k, t in v.items()}
    for stream in (True, False):
        dx, dw = L.maskmoe_norm_backward(c["residual"], c["weight"], c["dy"], d_hidden=c["d_hidden"] if stream else None,
                                         eps=1e-5)
        wx, bx, ww, bw = N.backward(f64(v["residual"]), f64(v["weight"]), f64(v["dy"]),
                                    f64(v["d_hidden"]) if stream else None, 1e-5, half(dtype))
        assert (np.abs(f64(dx) - wx) <= bx + 2.0 ** -130).all()
        assert (np.abs(f64(dw) - ww) <= bw + 2.0 ** -130).all()
        again = L.maskmoe_norm_backward(c["residual"], c["weight"], c["dy"], d_hidden=c["d_hidden"] if stream else None,
                                        eps=1e-5)
        assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
        only = L.maskmoe_norm_backward(c["residual"], c["weight"], c["dy"], d_hidden=c["d_hidden"] if stream else None,
                                       eps=1e-5, with_d_weight=False)
        assert torch.equal(only[0], dx) and only[1] is None


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", [(3, 64), (5, 4096), (2, 96)])
@pytest.mark.parametrize("off", [1, 3])
def test_tensors_that_start_anywhere(T, d, off, dtype):
    """Contiguous views at odd offsets of their storage: the same bits as aligned ones."""
    say(f"norm offsets T={T} d={d} {dtype} {off}")
    v = inputs(T, d, dtype, d)
    c = {k: t.cuda() for k, t in v.items()}

    def moved(t):
        buf = torch.empty(t.numel() + 16, dtype=t.dtype, device="cuda")
        out = buf[off:off + t.numel()].view(t.shape)
        out.copy_(t)
        return out
    a = L.maskmoe_norm_forward(c["x"], c["weight"], residual=c["residual"], with_mx8=True)
    check_forward(v, dtype, 1e-5, True, True, a)
    b = L.maskmoe_norm_forward(moved(c["x"]), moved(c["weight"]), residual=moved(c["residual"]), with_mx8=True)
    check_forward(v, dtype, 1e-5, True, True, b)
    assert torch.equal(a[1], b[1])
    w = N.backward(f64(v["residual"]), f64(v["weight"]), f64(v["dy"]), f64(v["d_hidden"]), 1e-5, half(dtype))
    for m in (lambda t: t, moved):
        dx, dw = L.maskmoe_norm_backward(m(c["residual"]), m(c["weight"]), m(c["dy"]), d_hidden=m(c["d_hidden"]),
                                         d_x=m(c["x"]))
        assert (np.abs(f64(dx) - w[0]) <= w[1]).all() and (np.abs(f64(dw) - w[2]) <= w[3]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d", [(1, 4096), (70, 96), (3, 33), (2100, 512)])
def test_in_place(T, d, dtype):
    v = {k: t.cuda() for k, t in inputs(T, d, dtype, 5).items()}
    y, h, _, _ = L.maskmoe_norm_forward(v["x"], v["weight"], residual=v["residual"])
    for name, other in (("residual", "x"), ("x", "residual")):
        w = {k: t.clone() for k, t in v.items()}
        y2, h2, _, _ = L.maskmoe_norm_forward(w["x"], w["weight"], residual=w["residual"], hidden=w[name], y=w[other])
        assert h2 is w[name] and torch.equal(h2, h) and y2 is w[other] and torch.equal(y2, y)
    w = v["x"].clone()
    assert torch.equal(L.maskmoe_norm_forward(w, v["weight"], y=w)[0], L.maskmoe_norm_forward(v["x"], v["weight"])[0])
    dx, dw = L.maskmoe_norm_backward(h, v["weight"], v["dy"], d_hidden=v["d_hidden"])
    for name in ("h", "dy", "d_hidden"):
        w = dict(v, h=h)
        w = {k: t.clone() for k, t in w.items()}
        dx2, dw2 = L.maskmoe_norm_backward(w["h"], w["weight"], w["dy"], d_hidden=w["d_hidden"], d_x=w[name])
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw)


def test_rows_of_zeros_infinities_and_nan():
    for dtype in DTYPES:
        x = torch.randn((6, 256), generator=torch.Generator().manual_seed(1)).to(dtype)
        x[0] = 0
        x[1, 3], x[2, 200] = float("inf"), float("nan")
        x[3] = 0
        x[3, 0] = 3e38          # its square passes fp32's range
        w = torch.ones(256, dtype=dtype)
        y, _, c, s = (t.cpu() if t is not None else None for t in L.maskmoe_norm_forward(x.cuda(), w.cuda(), with_mx8=True))
        assert (y[0] == 0).all() and (s[0] == 0).all() and (c[0] == 0).all()
        assert y[1, 3].isnan() and (y[1, :3] == 0).all() and y[2].isnan().all() and (s[2] == 255).all()
        assert s[1, 0] == 255 and (s[1, 1:] == 0).all()
        assert (y[3] == 0).all() and y[4:].isfinite().all()
        y0 = L.maskmoe_norm_forward(x.cuda(), w.cuda(), eps=0.0)[0].cpu()
        assert y0[0].isnan().all() and y0[4:].isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nan_near_the_end_of_odd_rows(dtype):
    """The last eight columns of a row are in two pieces: each counts once."""
    x = torch.randn((5, 251), generator=torch.Generator().manual_seed(2)).to(dtype)
    x[1, 245], x[2, 246], x[3, 250] = float("inf"), float("nan"), float("-inf")
    w = torch.ones(251, dtype=dtype)
    y = L.maskmoe_norm_forward(x.cuda(), w.cuda())[0].cpu()
    assert y[2].isnan().all() and y[[0, 4]].isfinite().all()
    for r, c in ((1, 245), (3, 250)):
        rest = torch.arange(251) != c
        assert y[r, c].isnan() and (y[r, rest] == 0).all()
    dy = torch.randn((5, 251), generator=torch.Generator().manual_seed(3)).to(dtype)
    dy[0, 244] = float("nan")
    x[1:4] = 1
    d_x, d_w = (t.cpu() for t in L.maskmoe_norm_backward(x.cuda(), w.cuda(), dy.cuda()))
    assert d_x[0].isnan().all() and d_x[1:].isfinite().all()
    assert d_w[244].isnan() and d_w[torch.arange(251) != 244].isfinite().all()


def test_nothing_and_no_tokens():
    x, w = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda")
    y, h, c, s = L.maskmoe_norm_forward(x, w, residual=x, with_mx8=True)
    assert y.shape == h.shape == c.shape == (0, 64) and s.shape == (0, 2)
    dx, dw = L.maskmoe_norm_backward(x, w, x)
    assert dx.shape == (0, 64) and (dw == 0).all()
    with pytest.raises(L.MaskMoEError):
        L.maskmoe_norm_forward(torch.ones((2, 64), device="cuda"), w, with_y=False)


def test_binding_refuses():
    x, w = torch.ones((4, 64), device="cuda"), torch.ones(64, device="cuda")
    for f in (lambda: L.maskmoe_norm_forward(x.t(), w), lambda: L.maskmoe_norm_forward(x, w.bfloat16()),
              lambda: L.maskmoe_norm_forward(x, w[:32]), lambda: L.maskmoe_norm_forward(x, w, residual=x[:3]),
              lambda: L.maskmoe_norm_forward(x.cpu(), w), lambda: L.maskmoe_norm_forward(x, w.cpu()),
              lambda: L.maskmoe_norm_backward(x, w, x[:, ::2]), lambda: L.maskmoe_norm_backward(x, w, x.double()),
              lambda: L.maskmoe_mx8_dequantize(x, x, torch.float32)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: L.maskmoe_norm_forward(x.half(), w.half()), lambda: L.maskmoe_mx8_quantize(x.half())):
        with pytest.raises(TypeError):
            f()


def test_streams_and_graphs():
    v = {k: t.cuda() for k, t in inputs(777, 1024, torch.bfloat16, 9).items()}
    ref = L.maskmoe_norm_forward(v["x"], v["weight"], residual=v["residual"], with_mx8=True)
    gref = L.maskmoe_norm_backward(v["residual"], v["weight"], v["dy"], d_hidden=v["d_hidden"])
    torch.cuda.synchronize()
    outs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        with torch.cuda.stream(s):
            for _ in range(4):
                outs.append((L.maskmoe_norm_forward(v["x"], v["weight"], residual=v["residual"], with_mx8=True),
                             L.maskmoe_norm_backward(v["residual"], v["weight"], v["dy"], d_hidden=v["d_hidden"])))
    torch.cuda.synchronize()
    for o, g in outs:
        assert all(torch.equal(a, b) for a, b in zip(o + g, ref + gref))
    buf = {k: t.clone() for k, t in v.items()}
    ws = torch.empty(L.maskmoe_norm_backward_workspace_bytes(777, 1024), dtype=torch.uint8, device="cuda")
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        y, h, c, sc = L.maskmoe_norm_forward(buf["x"], buf["weight"], residual=buf["residual"], with_mx8=True)
        back = L.maskmoe_mx8_dequantize(c, sc, torch.bfloat16)
        dx, dw = L.maskmoe_norm_backward(h, buf["weight"], buf["dy"], d_hidden=back, workspace=ws)
    for i in range(4):
        for k in ("x", "dy"):
            buf[k].copy_(v[k].roll(i, 0))
        graph.replay()
        torch.cuda.synchronize()
        e = L.maskmoe_norm_forward(buf["x"], buf["weight"], residual=buf["residual"], with_mx8=True)
        e_back = L.maskmoe_mx8_dequantize(e[2], e[3], torch.bfloat16)
        g = L.maskmoe_norm_backward(e[1], buf["weight"], buf["dy"], d_hidden=e_back)
        assert all(torch.equal(a, b) for a, b in zip((y, h, c, sc, back, dx, dw), e + (e_back,) + g))


def test_past_32_bit_offsets():
    """More than 2^32 elements: the last rows are those of a call on them alone."""
    T, d = (1 << 20) + 3, 4096
    say(f"norm {T} x {d}")
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).fill_(0x3F80)
    g = torch.Generator(device="cuda").manual_seed(3)
    x[-5:] = torch.randn((5, d), generator=g, device="cuda").bfloat16()
    w = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16()
    y, h, c, s = L.maskmoe_norm_forward(x, w, residual=x, with_mx8=True)
    e = L.maskmoe_norm_forward(x[-5:].clone(), w, residual=x[-5:].clone(), with_mx8=True)
    assert all(torch.equal(a[-5:], b) for a, b in zip((y, h, c, s), e))
    back = L.maskmoe_mx8_dequantize(c, s, torch.bfloat16)
    assert torch.equal(back[-5:], L.maskmoe_mx8_dequantize(e[2], e[3], torch.bfloat16))
    c2, s2 = L.maskmoe_mx8_quantize(back)
    assert torch.equal(c2[-5:], c[-5:]) and torch.equal(s2[-5:], s[-5:])
    dx, _ = L.maskmoe_norm_backward(x, w, y)
    assert torch.equal(dx[-5:], L.maskmoe_norm_backward(x[-5:].clone(), w, y[-5:].clone())[0])


def test_most_rows():
    """2^31 - 1 rows: the walk over the rows ends, and the last ones are those of a call on them alone."""
    T, last = 2 ** 31 - 1, 9000
    say(f"norm {T} x 1")
    x = torch.empty((T, 1), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).fill_(0x3F80)
    g = torch.Generator(device="cuda").manual_seed(5)
    x[-last:] = torch.randn((last, 1), generator=g, device="cuda").bfloat16()
    w = torch.full((1,), 2.0, device="cuda").bfloat16()
    y, _, _, _ = L.maskmoe_norm_forward(x, w, eps=0.5)
    e, _, _, _ = L.maskmoe_norm_forward(x[-last:].clone(), w, eps=0.5)
    assert torch.equal(y[-last:], e)
    assert (y[:10].float() - 2 / 1.5 ** 0.5).abs().max() <= 2.0 ** -8 and torch.equal(y[:-last:4097], y[:1].expand(len(y[:-last:4097]), 1))
    back = L.maskmoe_norm_backward(x, w, y, eps=0.5, with_d_weight=False)[0]
    assert torch.equal(back[-last:], L.maskmoe_norm_backward(x[-last:].clone(), w, e, eps=0.5, with_d_weight=False)[0])
    assert torch.equal(back[:-last:4097], back[:1].expand(len(back[:-last:4097]), 1))

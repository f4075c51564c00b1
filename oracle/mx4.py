"""MX4 blocks (32 E2M1 elements under one E8M0 scale) and expert FFNs on such weights, in float64."""

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])   # magnitudes in code order
BLOCK = 32


def exponent(amax):
    """Scale exponent of a block: floor(log2(amax)) - 2, at least -127; -127 for zeros."""
    _, e = np.frexp(amax)   # amax = m 2^e, m in [0.5, 1)
    return np.where(amax > 0, np.maximum(e - 1 - 2, -127), -127)


def nearest_codes(u):
    """Codes (sign in bit 3) of the elements nearest to u, ties to the even code, saturating."""
    a = np.abs(u)[..., None]
    d = np.abs(a - GRID)
    low = d.min(-1, keepdims=True)
    tied = d == low
    even = tied & (np.arange(8) % 2 == 0)
    c = np.where(even.any(-1), even.argmax(-1), tied.argmax(-1))
    return c | (np.signbit(u).astype(np.int64) << 3)


def quantize(v):
    """(codes [..., n], exponents [..., n / 32]) of v [..., n]; exponent 128 marks a block with an infinity or NaN."""
    b = np.asarray(v, np.float64).reshape(v.shape[:-1] + (-1, BLOCK))
    amax = np.abs(b).max(-1)
    bad = ~np.isfinite(amax)
    e = np.where(bad, 128, exponent(np.where(bad, 1.0, amax)))
    u = np.where(bad[..., None], 0.0, b) / np.exp2(np.where(bad, 0, e).astype(np.float64))[..., None]
    return nearest_codes(u).reshape(v.shape), e


def values(codes, e):
    """The numbers that codes and exponents stand for."""
    mag = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(e == 128, np.nan, np.exp2(np.where(e == 128, 0, e).astype(np.float64)))
    return (mag.reshape(codes.shape[:-1] + (-1, BLOCK)) * s[..., None]).reshape(codes.shape)


def rounded(v):
    return values(*quantize(v))


def pack_codes(codes):
    """Two codes a byte, the even element in the low half."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def silu(a):
    with np.errstate(over="ignore"):
        return a / (1 + np.exp(-a))


def experts(x, idx, gate, w_gate_up, w_down, n_shared, mx_act, u32=2.0 ** -24, half=2.0 ** -8):
    """y [T,d] of experts with weights w_gate_up [n,2F,d], w_down [n,d,F] (values; the last n_shared are shared)
    and a bound on |y' - y| for a computation with fp32 sums (u32: relative error of an addition), h rounded
    to bf16 (half: half a bf16 step) or to MX4 blocks, and y rounded to bf16.

    The bound follows each rounding through the sums with absolute values: a sum of n products is off by at
    most n u32 times the sum of their magnitudes; SiLU has slope at most 1.1; MX4 elements of h that come within
    the error of a rounding border, or whose block comes within it of another scale, may take either value.
    """
    T, d = x.shape
    n, F2, _ = w_gate_up.shape
    F, E = F2 // 2, n - n_shared
    xq = rounded(x) if mx_act else np.asarray(x, np.float64)
    y = np.zeros((T, d))
    bound = np.zeros((T, d))
    for e in range(n):
        if e < E:
            t, k = np.nonzero(idx == e)
            g = np.asarray(gate, np.float64)[t, k]
        else:
            t, g = np.arange(T), np.ones(T)
        if not t.size:
            continue
        wg, wu, wd = w_gate_up[e, :F], w_gate_up[e, F:], w_down[e]
        v = xq[t]
        a, b = v @ wg.T, v @ wu.T
        ea, eb = (d + 8) * u32 * (np.abs(v) @ np.abs(wg).T), (d + 8) * u32 * (np.abs(v) @ np.abs(wu).T)
        h = silu(a) * b
        eh = 1.1 * ea * (np.abs(b) + eb) + np.abs(silu(a)) * eb + 8 * u32 * np.abs(h)
        if mx_act:
            hq = rounded(h)
            dev = np.zeros_like(h)
            lo, hi = h - eh, h + eh
            amax = np.abs(h).reshape(len(t), -1, BLOCK).max(-1)
            slack = eh.reshape(len(t), -1, BLOCK).max(-1)
            for am in (np.maximum(amax - slack, 0), amax, amax + slack):
                s = np.exp2(exponent(am).astype(np.float64))[..., None]
                for u in (lo, h, hi):
                    c = nearest_codes(u.reshape(s.shape[:2] + (BLOCK,)) / s)
                    q = (GRID[c & 7] * np.where(c & 8, -1.0, 1.0) * s).reshape(h.shape)
                    dev = np.maximum(dev, np.abs(q - hq))
            h, eh = hq, dev
        else:
            eh = eh + half * (np.abs(h) + eh)
        o = h @ wd.T
        eo = eh @ np.abs(wd).T + (F + 8) * u32 * ((np.abs(h) + eh) @ np.abs(wd).T)
        np.add.at(y, t, g[:, None] * o)
        np.add.at(bound, t, np.abs(g)[:, None] * (eo + 32 * u32 * np.abs(o)))
    return y, bound + half * (np.abs(y) + bound)

"""8-bit blocks (32 int8 codes under one E8M0 scale) and the experts' training pass that keeps its gate / up
pre-activations in them, in float64."""

import numpy as np

BLOCK = 32
U32, HALF = 2.0 ** -24, 2.0 ** -8   # relative errors of an fp32 operation and of a rounding to bf16
FN = 2.0 ** -19                     # of a sigmoid from the hardware's exponential and reciprocal, with what follows it


def _blocks(a):
    return a.reshape(a.shape[:-1] + (a.shape[-1] // BLOCK, BLOCK))


def quantize(v):
    """(codes [..., n] int, exponents [..., n / 32]); values are codes * 2^(exponent - 6); exponent 128 marks a block
    with an infinity or NaN."""
    v = np.asarray(v, np.float64)
    b = _blocks(v)
    amax = np.abs(b).max(-1)
    bad = ~np.isfinite(amax)
    _, e = np.frexp(np.where(bad, 1.0, amax))
    e = np.where(amax > 0, np.maximum(e - 1, -127), -127)
    u = np.where(bad[..., None], 0.0, b) * np.exp2(6.0 - e)[..., None]
    codes = np.clip(np.rint(u), -127, 127).astype(np.int64)
    return codes.reshape(v.shape), np.where(bad, 128, e)


def values(codes, e):
    c = _blocks(np.asarray(codes, np.float64))
    s = np.where(e == 128, np.nan, np.exp2(np.where(e == 128, 0, e) - 6.0))
    return (c * s[..., None]).reshape(codes.shape)


def rounded(v):
    return values(*quantize(v))


def off_by(v, err, codes, e):
    """How far codes and exponents are from blocks of numbers within err of v: the largest excess of a value over half a
    step (a whole one where the code is +-127) plus err, and whether every exponent is that of a magnitude in range."""
    step = np.exp2(e - 6.0).repeat(BLOCK, -1)
    room = np.where(np.abs(codes) == 127, 1.0, 0.5) * step + err
    lo = np.maximum(_blocks(np.abs(v) - err), 0).max(-1)
    hi = _blocks(np.abs(v) + err).max(-1)
    exp = lambda a: np.where(a > 0, np.maximum(np.frexp(a)[1] - 1, -127), -127)   # noqa: E731
    return (np.abs(values(codes, e) - v) - room).max(initial=-1.0), bool(((exp(lo) <= e) & (e <= exp(hi))).all())


def rows(idx, E, n_shared):
    """Entries (t, k, expert) of the live rows: by expert, shared ones (k >= K) last, then by token and slot."""
    T, K = idx.shape
    out = []
    for e in range(E + n_shared):
        for t in range(T):
            for k in range(K) if e < E else (K + e - E,):
                if e >= E or idx[t, k] == e:
                    out.append((t, k, e))
    return out


def _sig(a):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-a))


def forward(x, idx, gate, w_gate_up, w_down, n_shared):
    """y [T, d], a bound on it, the rows' [a b] [rows, 2F] in fp64 and a bound on their fp32 sums. Weights of E + n_shared
    experts, the shared ones last."""
    n, F2, d = w_gate_up.shape
    F = F2 // 2
    y, b_y, ab, b_ab = np.zeros_like(x), np.zeros_like(x), [], []
    for t, k, e in rows(idx, n - n_shared, n_shared):
        z = w_gate_up[e] @ x[t]
        e_z = d * U32 * (np.abs(w_gate_up[e]) @ np.abs(x[t]))
        a, b, e_a, e_b = z[:F], z[F:], e_z[:F], e_z[F:]
        silu = a * _sig(a)
        h = silu * b
        # |SiLU'| <= 1.1; then h's rounding to bf16
        e_h = 1.1 * e_a * (np.abs(b) + e_b) + np.abs(silu) * e_b + FN * np.abs(h)
        e_h = e_h + HALF * (np.abs(h) + e_h)
        o = w_down[e] @ h
        e_o = np.abs(w_down[e]) @ e_h + F * U32 * (np.abs(w_down[e]) @ (np.abs(h) + e_h))
        g = gate[t, k] if k < idx.shape[1] else 1.0
        y[t] += g * o
        b_y[t] += np.abs(g) * (e_o + 32 * U32 * np.abs(o))
        ab.append(z)
        b_ab.append(e_z)
    empty = np.zeros((0, F2))
    return y, b_y + HALF * (np.abs(y) + b_y), np.array(ab) if ab else empty, np.array(b_ab) if ab else empty


def backward(x, idx, gate, w_gate_up, w_down, n_shared, ab, dy):
    """Gradients of <dy, y> from pre-activations ab [rows, 2F] taken as they are: {name: (value, bound)} with d_x, d_gate,
    d_w_gate_up, d_w_down (the shared experts' behind the routed ones)."""
    n, F2, d = w_gate_up.shape
    F, T, K = F2 // 2, *idx.shape
    z = lambda *s: (np.zeros(s), np.zeros(s))   # noqa: E731
    dx, dg, dgu, ddn = z(T, d), z(T, K), z(n, F2, d), z(n, d, F)
    count = np.zeros(n)
    for r, (t, k, e) in enumerate(rows(idx, n - n_shared, n_shared)):
        count[e] += 1
        g = gate[t, k] if k < K else 1.0
        a, b = ab[r, :F], ab[r, F:]
        s = _sig(a)
        u = w_down[e].T @ dy[t]
        e_u = d * U32 * (np.abs(w_down[e]).T @ np.abs(dy[t]))
        h, slope = a * s * b, s * (1 + a * (1 - s))
        if k < K:
            dg[0][t, k] = u @ h
            dg[1][t, k] = e_u @ np.abs(h) + (FN + (F + 8) * U32) * ((np.abs(u) + e_u) @ np.abs(h))
        dab = np.concatenate([g * u * b * slope, g * u * a * s])
        # the slope's two terms may cancel: its error goes by their sizes
        size = np.concatenate([np.abs(b) * s * (1 + 2 * np.abs(a)), np.abs(a) * s])
        uu, ee = np.concatenate([np.abs(u), np.abs(u)]), np.concatenate([e_u, e_u])
        e_ab = np.abs(g) * (np.abs(np.concatenate([b * slope, a * s])) * ee + FN * size * (uu + ee))
        e_ab = e_ab + HALF * (np.abs(dab) + e_ab)
        gh = g * h
        e_gh = (HALF + FN) * np.abs(gh)
        W, x_t, dy_t = np.abs(w_gate_up[e]), np.abs(x[t]), np.abs(dy[t])
        dx[0][t] += dab @ w_gate_up[e]
        dx[1][t] += e_ab @ W + (F2 + 32) * U32 * ((np.abs(dab) + e_ab) @ W)
        dgu[0][e] += np.outer(dab, x[t])
        dgu[1][e] += np.outer(e_ab, x_t) + T * K * U32 * np.outer(np.abs(dab) + e_ab, x_t)
        ddn[0][e] += np.outer(dy[t], gh)
        ddn[1][e] += np.outer(dy_t, e_gh) + T * K * U32 * np.outer(dy_t, np.abs(gh) + e_gh)
    once = lambda p: (p[0], p[1] + HALF * (np.abs(p[0]) + p[1]))   # noqa: E731
    return dict(d_x=once(dx), d_gate=dg, d_w_gate_up=once(dgu), d_w_down=once(ddn))

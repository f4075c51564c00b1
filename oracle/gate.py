"""Selection by scores, balance bias and expert groups, token by token in float64.

``key_e = s_e * prior_e + bias_e`` with s the softmax (over every expert whose logit is neither NaN nor
-inf) or sigmoid of the router logits; the best groups by their largest key or the sum of their two largest;
Top-K of the keys in them, ties to the lower index; gates from the scores.
"""

import math

import numpy as np

SOFTMAX, SIGMOID = 0, 1
GROUP_MAX, GROUP_SUM2 = 0, 1
FMAX = float(np.finfo(np.float32).max)


def scores(z, score):
    """Scores of one row of logits; 0 where the logit is NaN or -inf."""
    z = np.minimum(np.asarray(z, np.float64), FMAX)
    live = z > -np.inf
    s = np.zeros(z.shape)
    if not live.any():
        return s, live
    if score == SIGMOID:
        v = z[live]
        s[live] = np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))
    else:
        e = np.exp(z[live] - z[live].max())
        s[live] = e / e.sum()
    return s, live


def log_scores(z, score):
    """log of the score up to a constant of the row, which ratios of scores need where scores underflow."""
    z = np.minimum(np.asarray(z, np.float64), FMAX)
    with np.errstate(invalid="ignore"):
        return z if score == SOFTMAX else -np.logaddexp(0.0, -z)


def forward(logits, K, score, n_group=1, topk_group=1, group_rule=GROUP_MAX, renorm=True, scale=1.0, bias=None,
            mask=None, prior=None):
    """(idx [T,K], gate [T,K], load [E]) of logits [T,E]."""
    T, E = logits.shape
    n = E // n_group
    idx = np.full((T, K), -1, np.int64)
    gate = np.zeros((T, K))
    for t in range(T):
        s, live = scores(logits[t], score)
        key = s.copy()
        if prior is not None:
            key = key * np.asarray(prior, np.float64)
        if bias is not None:
            key = key + np.asarray(bias, np.float64)
        ok = live if mask is None else live & (np.asarray(mask) != 0)
        plain = bias is None and prior is None and (n_group == 1 or group_rule == GROUP_MAX)
        if plain:   # the scores' own order, which float64 scores lose where they saturate
            key = np.minimum(np.asarray(logits[t], np.float64), FMAX)
        cand = [e for e in range(E) if ok[e]]
        if n_group > 1:
            lead = []
            for g in range(n_group):
                ks = sorted((key[e] for e in cand if e // n == g), reverse=True)
                lead.append(-math.inf if not ks else ks[0] if group_rule == GROUP_MAX else sum(ks[:2]))
            kept = sorted(range(n_group), key=lambda g: (-lead[g], g))[:topk_group]
            cand = [e for e in cand if e // n in kept]
        best = sorted(cand, key=lambda e: (-key[e], e))[:K]
        idx[t, :len(best)] = best
        if best:
            if renorm:
                ls = log_scores(logits[t], score)[best]
                w = np.exp(ls - ls.max())
                gate[t, :len(best)] = scale * w / w.sum()
            else:
                gate[t, :len(best)] = scale * s[best]
    load = np.array([(idx == e).sum() for e in range(E)])
    return idx, gate, load


def backward(logits, idx, d_gate, score, renorm=True, scale=1.0):
    """dL/dlogits [T,E] for a cotangent d_gate of the gates, idx held fixed."""
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        s, live = scores(logits[t], score)
        ent = [(int(e), float(g)) for e, g in zip(idx[t], d_gate[t]) if 0 <= e < E and live[int(e)]]
        if not ent:
            continue
        ids = [e for e, _ in ent]
        dg = np.array([g for _, g in ent])
        if renorm:
            ls = log_scores(logits[t], score)[ids]
            w = np.exp(ls - ls.max())
            w = w / w.sum()
            d = scale * w * (dg - (w * dg).sum())
            if score == SIGMOID:
                z = np.minimum(np.asarray(logits[t], np.float64), FMAX)[ids]
                d = d * np.exp(-np.logaddexp(0.0, z))
            for e, v in zip(ids, d):
                out[t, e] += v
        elif score == SIGMOID:
            for e, g in ent:
                out[t, e] += scale * g * s[e] * (1 - s[e])
        else:
            for e, g in ent:
                out[t, e] += scale * g
            out[t] = s * (out[t] - (s[ids] * scale * dg).sum())
    return out

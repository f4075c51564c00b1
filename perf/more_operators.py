"""Performance cases of the norm before an MoE layer (residual addition, root-mean-square norm, outputs in bf16 / fp32
and in 8-bit blocks, its gradient), of 8-bit blocks, and of the experts' training pass at a given routing with its
activations kept in 8-bit blocks, through the public entry points, with the operators' plain forms and their values
in 64 bits.

Model shapes as this repository's configurations, tests and benchmark use them: Mixtral-shaped (d 4096, F 14336,
8 experts, top-2), DeepSeek-shaped (d 2048, F 1408, 64 routed + 2 shared experts, top-6), a tiny one (d 256, F 512),
and one whose sizes fill no tile.

Kinds of case
  norm       s = x + residual, its stored form, s / rms(s) * weight in the input's type and / or in 8-bit blocks
  norm_bwd   gradients of the norm and of the residual stream that it reads
  mx8        a matrix to 8-bit blocks (32 int8 elements to a power of two) and back to the values they stand for
  train_fwd  routed and shared experts of one layer for a given routing; gate / up projections kept in 8-bit blocks
  train_bwd  gradients of tokens, gates and weights from those blocks
"""

import math

import torch

own = False

MODELS = {
    "mixtral": dict(d=4096, F=14336, E=8, K=2, ns=0, renorm=True),
    "deepseek": dict(d=2048, F=1408, E=64, K=6, ns=2, renorm=False),
    "tiny": dict(d=256, F=512, E=8, K=2, ns=0, renorm=True),
    "ragged": dict(d=320, F=192, E=5, K=3, ns=1, renorm=True),
}
BLOCK = 32


def _norm(T, d, **kw):
    c = dict(kind="norm", T=T, d=d, dtype="bf16", residual=True, y=True, mx8=False, eps=1e-5)
    c.update(kw)
    return c


def listed():
    return [
        # one decoded token: the latency of a norm between two layers
        dict(_norm(1, 4096), name="norm_t1_d4096"),
        # a short prompt of odd length, 8 bits beside bf16
        dict(_norm(333, 2048, mx8=True), name="norm_t333_d2048"),
        # a fine-tuning batch, 4 x 2048 tokens, whose 8-bit output is kept for the backward pass
        dict(_norm(8192, 4096, mx8=True), name="norm_t8192_d4096"),
        # a large prefill, 16 x 2048 tokens
        dict(_norm(32768, 4096), name="norm_t32768_d4096"),
        # backward pass of a short sequence
        dict(kind="norm_bwd", T=333, d=2048, dtype="bf16", stream=True, eps=1e-5, name="norm_bwd_t333_d2048"),
        # backward pass of a fine-tuning batch
        dict(kind="norm_bwd", T=8192, d=4096, dtype="bf16", stream=True, eps=1e-5, name="norm_bwd_t8192_d4096"),
        # activations of a short prompt
        dict(kind="mx8", rows=333, cols=2048, src="bf16", name="mx8_act_333"),
        # the SwiGLU activations of a fine-tuning batch: 8192 tokens x 2 experts
        dict(kind="mx8", rows=16384, cols=14336, src="bf16", name="mx8_act_16384"),
        # a short fine-tuning sequence of odd length through many small experts, some slots empty
        dict(kind="train_fwd", model="deepseek", T=333, pad=5, spread=1.3, name="train_fwd_deepseek_t333"),
        # a fine-tuning batch of large experts
        dict(kind="train_fwd", model="mixtral", T=8192, pad=0, spread=1.3, name="train_fwd_mixtral_t8192"),
        # backward pass of two sequences through many small experts, tokens kept in 8 bits too
        dict(kind="train_bwd", model="deepseek", T=4096, pad=0, spread=1.3, x8=True, name="train_bwd_deepseek_t4096"),
        # backward pass of a fine-tuning batch of large experts
        dict(kind="train_bwd", model="mixtral", T=8192, pad=0, spread=1.3, x8=False, name="train_bwd_mixtral_t8192"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm", "norm_bwd", "norm_bwd", "mx8", "train_fwd", "train_fwd", "train_bwd",
                       "train_bwd"])
    if kind in ("norm", "norm_bwd"):
        mx8 = kind == "norm" and rng.random() < 0.5
        d = BLOCK * _log_int(rng, 1, 512) if mx8 or rng.random() < 0.6 else _log_int(rng, 1, 16384)
        T = min(_log_int(rng, 1, 32768), (8192 if kind == "norm_bwd" else 16384) * 4096 // d)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        eps = rng.choice([1e-6, 1e-5])
        if kind == "norm_bwd":
            return dict(kind=kind, T=T, d=d, dtype=dtype, stream=rng.random() < 0.7, eps=eps)
        return _norm(T, d, dtype=dtype, residual=rng.random() < 0.7, y=not mx8 or rng.random() < 0.6, mx8=mx8, eps=eps)
    if kind == "mx8":
        return dict(kind="mx8", rows=_log_int(rng, 1, 16384), cols=BLOCK * _log_int(rng, 1, 448),
                    src=rng.choice(["bf16", "f32"]))
    model = rng.choice(["mixtral", "deepseek", "tiny", "ragged"])
    T = _log_int(rng, 1, 8192)
    c = dict(kind=kind, model=model, T=T, pad=rng.choice([0, 0, T // 7]), spread=round(rng.uniform(0.5, 2.5), 2))
    if kind == "train_bwd":
        c["x8"] = rng.random() < 0.5
    return c


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _p2(n):
    """2^n for integer tensors n in -126..127, exactly."""
    return ((n.to(torch.int32) + 127) << 23).view(torch.float32)


def _times_p2(v, n):
    """v * 2^n, n in -252..254: two steps, since the scale of the smallest blocks has no finite reciprocal."""
    half = torch.div(n, 2, rounding_mode="floor")
    return v * _p2(half) * _p2(n - half)


def _mx8(v):
    """Blocks of 32 along the last dimension of fp32 v: int8 codes and scale bytes."""
    v = v.unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(-1, keepdim=True)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 1, -127).clamp(-127, 127)
    codes = torch.round(_times_p2(v, 6 - e)).clamp(-127, 127)
    return codes.to(torch.int8).flatten(-2), (e + 127).to(torch.uint8).squeeze(-1)


def _mx8_values(codes, scales):
    c = codes.unflatten(-1, (-1, BLOCK)).float()
    return _times_p2(c, scales.to(torch.int32).unsqueeze(-1) - 133).flatten(-2)


def _loud(g, n):
    """A factor for each channel: a few are loud, as in the stream between layers."""
    return 1 + 7 * (torch.rand(n, generator=g, device="cuda") < 0.01)


def _norm_inputs(case, seed):
    g = _gen(seed)
    T, d = case["T"], case["d"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    loud = _loud(g, d)

    def rows(scale):
        return (torch.randn((T, d), generator=g, device="cuda") * scale).to(dt)

    s = dict(weight=(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt))
    if case["kind"] == "norm":
        s["x"] = rows(0.4 * loud)
        s["residual"] = rows(2.0 * loud) if case["residual"] else None
    else:
        s["hidden"] = rows(2.0 * loud)
        s["dy"] = rows(0.02)
        s["d_hidden"] = rows(0.02) if case["stream"] else None
    return s


def _expert_inputs(case, seed):
    """Tokens as a norm leaves them, weights N(0, 1 / fan_in), routing by the softmax of random logits (spread: their
    deviation, which decides how uneven the routing is); the last `pad` tokens are empty slots."""
    m = MODELS[case["model"]]
    d, F, E, K, ns, T = m["d"], m["F"], m["E"], m["K"], m["ns"], case["T"]
    g = _gen(seed)
    s = dict(x=(torch.randn((T, d), generator=g, device="cuda") * _loud(g, d)).bfloat16())

    def weights(n, r, c):
        return torch.randn((n, r, c), generator=g, device="cuda", dtype=torch.bfloat16).mul_(c ** -0.5)

    s["w_gate_up"], s["w_down"] = weights(E, 2 * F, d), weights(E, d, F)
    s["ws_gate_up"], s["ws_down"] = (weights(ns, 2 * F, d), weights(ns, d, F)) if ns else (None, None)
    p = torch.softmax(case["spread"] * torch.randn((T, E), generator=g, device="cuda"), -1)
    gate, idx = p.topk(K, -1)
    if m["renorm"]:
        gate = gate / gate.sum(-1, keepdim=True)
    s["idx"], s["gate"] = idx.int().contiguous(), gate.contiguous()
    if case["pad"]:
        s["idx"][T - case["pad"]:] = -1
        s["gate"][T - case["pad"]:] = 0.0
    if case["kind"] == "train_bwd":
        s["dy"] = (0.02 * torch.randn((T, d), generator=g, device="cuda")).bfloat16()
    return s


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("norm", "norm_bwd"):
        s = _norm_inputs(case, seed)
    elif kind == "mx8":
        x = torch.randn((case["rows"], case["cols"]), generator=_gen(seed), device="cuda")
        s = dict(x=x.bfloat16() if case["src"] == "bf16" else x)
    else:
        m = MODELS[case["model"]]
        s = _expert_inputs(case, seed)
        _host_view(case, s)
        R, F2 = case["T"] * (m["K"] + m["ns"]), 2 * m["F"]
        # the checkpoint's own memory; rows of empty entries, its last ones, stay as they are
        s["codes"] = torch.zeros((R, F2), dtype=torch.int8, device="cuda")
        s["scales"] = torch.zeros((R, F2 // BLOCK), dtype=torch.uint8, device="cuda")
        if kind == "train_bwd":   # what a forward pass left
            lay = _layout(case, s)
            codes, scales = _mx8(_gate_up(s, lay, s["x"].float()))
            s["codes"][:lay["n"]], s["scales"][:lay["n"]] = codes[lay["pos"]], scales[lay["pos"]]
            if case["x8"]:
                s["x_codes"], s["x_scales"] = _mx8(s["x"].float())
    s["case"] = dict(case)
    return s


# ---------------------------------------------------------------- one pass

def _norm_plain(case, s):
    v = s["x"].float()
    if s["residual"] is not None:
        v = v + s["residual"].float()
    y = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + case["eps"]) * s["weight"].float()
    out = dict(y=y.to(s["x"].dtype)) if case["y"] else {}
    if s["residual"] is not None:
        out["hidden"] = v.to(s["x"].dtype)
    if case["mx8"]:
        out["values"] = _mx8_values(*_mx8(y)).bfloat16()
    return out


def _norm_bwd_plain(case, s):
    h, w, dy = s["hidden"].float(), s["weight"].float(), s["dy"].float()
    rstd = torch.rsqrt((h * h).mean(-1, keepdim=True) + case["eps"])
    n = h * rstd
    dn = dy * w
    dx = rstd * (dn - n * (dn * n).mean(-1, keepdim=True))
    if s["d_hidden"] is not None:
        dx = dx + s["d_hidden"].float()
    return dict(d_x=dx.to(s["hidden"].dtype), d_weight=(dy * n).sum(0))


def _host_view(case, s):
    """The host's view of the routing, which the plain form lays its rows out by: the experts with rows (routed ones,
    then shared ones), and the most rows that one has."""
    m = MODELS[case["model"]]
    load = torch.bincount(s["idx"].reshape(-1).long() + 1, minlength=m["E"] + 1)[1:].cpu()
    s["active"] = load.nonzero().flatten().tolist() + list(range(m["E"], m["E"] + m["ns"]))
    s["cap"] = max([int(load.max())] + [case["T"]] * (m["ns"] > 0) + [1])


def _layout(case, s):
    """Entries (token, slot), the shared experts' behind the routed ones, in order of experts and then of entries: the
    row order of a checkpoint. Row r of it is row pos[r] of a padded [active, cap] layout."""
    m = MODELS[case["model"]]
    T, E, KS = case["T"], m["E"], m["K"] + m["ns"]
    dev = s["x"].device
    shared = torch.arange(E, E + m["ns"], device=dev).expand(T, -1)
    flat = torch.cat((torch.where(s["idx"] < 0, 1 << 20, s["idx"].long()), shared), 1).reshape(-1)
    e, order = torch.sort(flat, stable=True)
    n = T * KS - case["pad"] * m["K"]
    e, order = e[:n], order[:n]
    act = torch.tensor(s["active"], device=dev, dtype=torch.long)
    slot = torch.searchsorted(act, e)
    pos = slot * s["cap"] + torch.arange(n, device=dev) - torch.searchsorted(e, act)[slot]
    gate = torch.cat((s["gate"], torch.ones((T, m["ns"]), device=dev)), 1).reshape(-1)
    return dict(n=n, order=order, token=order // KS, pos=pos, gate=gate[order], rows=len(s["active"]) * s["cap"])


def _matrices(s, name):
    """fp32 matrices of the experts with rows."""
    w = s["w" + name] if s["ws" + name] is None else torch.cat((s["w" + name], s["ws" + name]))
    return w[s["active"]].float()


def _spread_rows(lay, v):
    out = torch.zeros((lay["rows"],) + v.shape[1:], device=v.device)
    out[lay["pos"]] = v
    return out


def _gate_up(s, lay, x):
    """W_gate x and W_up x of every row, fp32 [active * cap, 2F]."""
    rows = _spread_rows(lay, x[lay["token"]])
    return torch.bmm(rows.view(len(s["active"]), s["cap"], -1), _matrices(s, "_gate_up").transpose(1, 2)).flatten(0, 1)


def _token_sum(case, s, lay, v):
    """Sum over a token's entries of rows v [n, c]: entries one after the other."""
    m = MODELS[case["model"]]
    T, KS = case["T"], m["K"] + m["ns"]
    out = torch.zeros((T * KS, v.shape[-1]), device=v.device)
    out[lay["order"]] = v
    return out.view(T, KS, -1).sum(1)


def _train_fwd_plain(case, s):
    lay = _layout(case, s)
    ab = _gate_up(s, lay, s["x"].float())
    a, b = ab.chunk(2, -1)
    h = a / (1 + torch.exp(-a)) * b
    o = torch.bmm(h.view(len(s["active"]), s["cap"], -1), _matrices(s, "_down").transpose(1, 2)).flatten(0, 1)
    y = _token_sum(case, s, lay, o[lay["pos"]] * lay["gate"][:, None])
    s["codes"][:lay["n"]], s["scales"][:lay["n"]] = _mx8(ab[lay["pos"]])
    return dict(y=y.bfloat16(), kept=_mx8_values(s["codes"], s["scales"]).bfloat16())


def _train_bwd_plain(case, s):
    m = MODELS[case["model"]]
    T, d, F, E, K, ns = case["T"], m["d"], m["F"], m["E"], m["K"], m["ns"]
    lay, A, cap = _layout(case, s), len(s["active"]), s["cap"]
    n = lay["n"]
    x = _mx8_values(s["x_codes"], s["x_scales"]) if case["x8"] else s["x"].float()
    a, b = _mx8_values(s["codes"][:n], s["scales"][:n]).chunk(2, -1)
    dy = _spread_rows(lay, s["dy"].float()[lay["token"]]).view(A, cap, d)
    u = torch.bmm(dy, _matrices(s, "_down")).flatten(0, 1)[lay["pos"]]
    sg = 1 / (1 + torch.exp(-a))
    h = a * sg * b
    d_entry = torch.zeros(T * (K + ns), device=a.device)
    d_entry[lay["order"]] = (u * h).sum(-1)
    g = lay["gate"][:, None]
    dab = _spread_rows(lay, torch.cat((g * u * b * sg * (1 + a * (1 - sg)), g * u * a * sg), -1)).view(A, cap, 2 * F)
    dx = torch.bmm(dab, _matrices(s, "_gate_up")).flatten(0, 1)[lay["pos"]]
    rows = _spread_rows(lay, x[lay["token"]]).view(A, cap, d)
    out = dict(d_x=_token_sum(case, s, lay, dx).bfloat16(), d_gate=d_entry.view(T, K + ns)[:, :K].contiguous())
    routed = A - ns
    for name, grad in (("_gate_up", torch.bmm(dab.transpose(1, 2), rows)),
                       ("_down", torch.bmm(dy.transpose(1, 2), _spread_rows(lay, g * h).view(A, cap, F)))):
        dw = torch.zeros_like(s["w" + name])
        dw[s["active"][:routed]] = grad[:routed].bfloat16()
        out["d_w" + name] = dw
        if ns:
            out["d_ws" + name] = grad[routed:].bfloat16()
    return out


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind == "norm":
            return _norm_plain(case, s)
        if kind == "norm_bwd":
            return _norm_bwd_plain(case, s)
        if kind == "mx8":
            return dict(values=_mx8_values(*_mx8(s["x"].float())).bfloat16())
        return _train_fwd_plain(case, s) if kind == "train_fwd" else _train_bwd_plain(case, s)
    from paper_2609_34077_amd import _lib as L
    if kind == "norm":
        y, hidden, codes, scales = L.maskmoe_norm_forward(s["x"], s["weight"], residual=s["residual"], eps=case["eps"],
                                                          with_y=case["y"], with_mx8=case["mx8"])
        out = dict(y=y) if case["y"] else {}
        if s["residual"] is not None:
            out["hidden"] = hidden
        if case["mx8"]:
            out["values"] = L.maskmoe_mx8_dequantize(codes, scales, torch.bfloat16)
        return out
    if kind == "norm_bwd":
        d_x, d_weight = L.maskmoe_norm_backward(s["hidden"], s["weight"], s["dy"], d_hidden=s["d_hidden"],
                                                eps=case["eps"])
        return dict(d_x=d_x, d_weight=d_weight)
    if kind == "mx8":
        codes, scales = L.maskmoe_mx8_quantize(s["x"])
        return dict(values=L.maskmoe_mx8_dequantize(codes, scales, torch.bfloat16))
    if kind == "train_fwd":
        y, codes, scales = L.maskmoe_experts_forward_train(
            s["x"], s["idx"], s["gate"], s["w_gate_up"], s["w_down"], ws_gate_up=s["ws_gate_up"],
            ws_down=s["ws_down"], codes=s["codes"], scales=s["scales"])
        return dict(y=y, kept=L.maskmoe_mx8_dequantize(codes, scales, torch.bfloat16))
    x, x_scales = (s["x_codes"], s["x_scales"]) if case["x8"] else (s["x"], None)
    grads = L.maskmoe_experts_backward(x, s["idx"], s["gate"], s["w_gate_up"], s["w_down"], s["codes"], s["scales"],
                                       s["dy"], ws_gate_up=s["ws_gate_up"], ws_down=s["ws_down"], x_scales=x_scales)
    return {k: v for k, v in grads.items() if v is not None}


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_bwd"):
        n, el = case["T"] * case["d"], 2 if case["dtype"] == "bf16" else 4
        if kind == "norm":
            each = el * (1 + 2 * case["residual"] + case["y"]) + case["mx8"] * (1 + 1 / BLOCK)
            return dict(bytes=int(n * each) + el * case["d"], flops=6 * n)
        return dict(bytes=n * el * (3 + case["stream"]) + (4 + el) * case["d"], flops=12 * n)
    if kind == "mx8":
        n = case["rows"] * case["cols"]
        return dict(bytes=int(n * ((2 if case["src"] == "bf16" else 4) + 2 * (1 + 1 / BLOCK) + 2)), flops=4 * n)
    m = MODELS[case["model"]]
    d, F, E, K, ns = m["d"], m["F"], m["E"], m["K"], m["ns"]
    T, live = case["T"], case["T"] - case["pad"]
    rows = live * K + T * ns
    active = E * (1 - (1 - K / E) ** live) + ns   # experts read, uniform routing
    expert = 3 * d * F
    kept = rows * 2 * F * (1 + 1 / BLOCK)
    if kind == "train_fwd":
        return dict(bytes=int(2 * active * expert + kept + 4 * T * d + 8 * T * K), flops=2 * rows * expert)
    return dict(bytes=int(2 * active * expert + 2 * (E + ns) * expert + kept + 6 * T * d + 12 * T * K),
                flops=4 * rows * expert)


# ---------------------------------------------------------------- the same in 64 bits

def _blocks64(v):
    """The values of v's 8-bit blocks."""
    v = v.reshape(-1, BLOCK)
    amax = v.abs().max(1, keepdim=True).values
    e = torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0)))
    e = torch.where(torch.exp2(e) > amax, e - 1, torch.where(torch.exp2(e + 1) <= amax, e + 1, e))   # at a power of two
    step = torch.exp2(torch.where(amax > 0, e, -127.0).clamp(min=-127) - 6)
    return torch.clamp(torch.round(v / step), -127, 127) * step


def exact(case, seed):
    kind = case["kind"]
    if kind == "norm":
        s = _norm_inputs(case, seed)
        v = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
        y = v / torch.sqrt(v.pow(2).mean(1, keepdim=True) + case["eps"]) * s["weight"].double()
        out = dict(y=y) if case["y"] else {}
        if s["residual"] is not None:
            out["hidden"] = v
        if case["mx8"]:
            out["values"] = _blocks64(y).view(y.shape)
        return out
    if kind == "norm_bwd":
        s = _norm_inputs(case, seed)
        h = s["hidden"].double().requires_grad_(True)
        w = s["weight"].double().requires_grad_(True)
        y = h / torch.sqrt(h.pow(2).mean(1, keepdim=True) + case["eps"]) * w
        y.backward(s["dy"].double())
        d_x = h.grad if s["d_hidden"] is None else h.grad + s["d_hidden"].double()
        return dict(d_x=d_x, d_weight=w.grad)
    if kind == "mx8":
        x = prepare(case, seed)["x"].double()
        return dict(values=_blocks64(x).view(x.shape))
    m = MODELS[case["model"]]
    T, d, F, E, K, ns = case["T"], m["d"], m["F"], m["E"], m["K"], m["ns"]
    s = prepare(case, seed)
    entries = torch.cat((s["idx"].long(), torch.arange(E, E + ns, device="cuda").expand(T, -1)), 1)
    gates = torch.cat((s["gate"].double(), torch.ones((T, ns), dtype=torch.float64, device="cuda")), 1)
    x = s["x"].double()
    if kind == "train_bwd" and case["x8"]:
        x = _blocks64(x).view(x.shape)
    y, kept, row = torch.zeros_like(x), torch.zeros((T * (K + ns), 2 * F), dtype=torch.float64, device="cuda"), 0
    dy = s["dy"].double() if kind == "train_bwd" else None
    d_x, d_gate = torch.zeros_like(x), torch.zeros_like(gates)
    grads = {k: torch.zeros_like(s[k], dtype=torch.float64) for k in ("w_gate_up", "w_down", "ws_gate_up", "ws_down")
             if s[k] is not None} if kind == "train_bwd" else {}
    for e in range(E + ns):
        t, k = (entries == e).nonzero(as_tuple=True)   # by token, then slot
        if not t.numel():
            continue
        pre, at = ("ws", e - E) if e >= E else ("w", e)
        gu, dn = s[pre + "_gate_up"][at].double(), s[pre + "_down"][at].double()
        g = gates[t, k][:, None]
        if kind == "train_fwd":
            ab = x[t] @ gu.t()
            h = ab[:, :F] * torch.sigmoid(ab[:, :F]) * ab[:, F:]
            y.index_add_(0, t, g * (h @ dn.t()))
            kept[row:row + len(t)] = _blocks64(ab).view(ab.shape)
        else:
            step = torch.exp2(s["scales"][row:row + len(t)].double() - 133).repeat_interleave(BLOCK, 1)
            ab = s["codes"][row:row + len(t)].double() * step
            a, b = ab[:, :F].clone().requires_grad_(True), ab[:, F:].clone().requires_grad_(True)
            h = torch.nn.functional.silu(a) * b
            u = dy[t] @ dn
            d_gate[t, k] = (u * h.detach()).sum(1)
            h.backward(g * u)
            dab = torch.cat((a.grad, b.grad), 1)
            d_x.index_add_(0, t, dab @ gu)
            grads[pre + "_gate_up"][at] = dab.t() @ x[t]
            grads[pre + "_down"][at] = dy[t].t() @ (g * h.detach())
        row += len(t)
    if kind == "train_fwd":
        return dict(y=y, kept=kept)
    return dict(d_x=d_x, d_gate=d_gate[:, :K], **{"d_" + k: v for k, v in grads.items()})

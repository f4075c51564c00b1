"""Performance cases of the expert-routing rule with scores, bias and groups and of the microscaled (MX)
expert layers, through the public entry points, with the operators' plain forms and their values in 64 bits.

Two model shapes stand behind the expert cases, the ones this repository's configurations, tests and
benchmark use: Mixtral-shaped (d 4096, F 14336, 8 experts, top-2) and DeepSeek-shaped (d 2048, F 1408, 64
routed + 2 shared experts, top-6). The routing cases also take 256 experts in 8 groups, the largest
number of experts that the library routes over.

Kinds of case
  gate      scores, balance bias, groups, top-K and gates from router logits (fp32 [T, E])
  gate_bwd  the gradient of those gates with respect to the logits
  mx        quantisation of a matrix to MX blocks of 4-bit elements (E2M1, 32 to a scale) and back to the
            values they stand for
  experts   the routed and shared experts of one layer on MX weights, given the routing; the activations in
            bf16, or in MX blocks too
"""

import math

import numpy as np
import torch

own = False

MODELS = {
    "mixtral": dict(d=4096, F=14336, E=8, K=2, ns=0, renorm=True),
    "deepseek": dict(d=2048, F=1408, E=64, K=6, ns=2, renorm=False),
    "tiny": dict(d=256, F=512, E=8, K=2, ns=0, renorm=True),
}
BLOCK = 32


def _gate(T, E, K, score, **kw):
    c = dict(kind="gate", T=T, E=E, K=K, score=score, groups=1, topk_group=1, rule="max", renorm=True, scale=1.0,
             bias=False, mask=False, prior=False, spread=1.3)
    c.update(kw)
    return c


def listed():
    return [
        # one decoded token of the DeepSeek-shaped layer: the latency of a routing decision
        dict(_gate(1, 64, 6, "softmax", renorm=False), name="gate_t1_e64"),
        # a short prompt of odd length, sigmoid scores with a balance bias and groups
        dict(_gate(333, 256, 8, "sigmoid", groups=8, topk_group=4, rule="sum2", bias=True, scale=2.5),
             name="gate_t333_e256"),
        # routing of a whole batch of sequences (256 x 512 tokens) at the largest expert count
        dict(_gate(131072, 256, 8, "sigmoid", groups=8, topk_group=4, rule="sum2", bias=True, scale=2.5),
             name="gate_t131072_e256"),
        # fine-tuning step, gates p of the full softmax: a dense gradient row per token
        dict(_gate(8192, 64, 6, "softmax", renorm=False), kind="gate_bwd", name="gate_bwd_t8192_e64"),
        # pre-training batch, sigmoid scores renormalised: only the selected experts get a gradient
        dict(_gate(65536, 256, 8, "sigmoid", groups=8, topk_group=4, rule="sum2", bias=True, scale=2.5),
             kind="gate_bwd", name="gate_bwd_t65536_e256"),
        # activations of a short prompt
        dict(kind="mx", rows=333, cols=2048, src="bf16", name="mx4_act_333"),
        # one Mixtral-shaped expert's gate / up matrix to 4 bits: the conversion of a checkpoint
        dict(kind="mx", rows=28672, cols=4096, src="bf16", name="mx4_weight_mixtral"),
        # interactive decode, one token
        dict(kind="experts", model="mixtral", T=1, act="bf16", pad=0, spread=1.3, name="experts_mixtral_t1"),
        # few tokens through many small experts
        dict(kind="experts", model="deepseek", T=5, act="bf16", pad=0, spread=1.3, name="experts_deepseek_t5"),
        # a serving step with continuous batching: about a hundred sequences, some slots empty
        dict(kind="experts", model="mixtral", T=96, act="bf16", pad=5, spread=1.3, name="experts_mixtral_t96"),
        # prefill of the smaller model with 4-bit activations: the matrix units' fastest type
        dict(kind="experts", model="deepseek", T=4096, act="mx4", pad=0, spread=1.3, name="experts_deepseek_t4096"),
        # a large prefill, 4 x 2048 tokens
        dict(kind="experts", model="mixtral", T=8192, act="bf16", pad=0, spread=1.3, name="experts_mixtral_t8192"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_gate(rng):
    E, K = rng.choice([(8, 2), (16, 2), (60, 4), (64, 6), (64, 8), (160, 6), (256, 8)])
    groups = rng.choice([1, 1, 2, 4, 8]) if E % 8 == 0 else 1
    n = E // groups
    need = -(-K // n)
    return _gate(_log_int(rng, 1, 131072), E, K, rng.choice(["softmax", "sigmoid"]), groups=groups,
                 topk_group=rng.randint(need, groups), rule=rng.choice(["max", "sum2"]), renorm=rng.random() < 0.6,
                 scale=rng.choice([1.0, 1.0, 2.5, 16.0]), bias=rng.random() < 0.6, mask=rng.random() < 0.3,
                 prior=rng.random() < 0.3, spread=round(rng.uniform(0.5, 2.5), 2))


def draw(rng):
    kind = rng.choice(["gate", "gate", "gate_bwd", "mx", "experts", "experts", "experts"])
    if kind == "gate":
        return _draw_gate(rng)
    if kind == "gate_bwd":
        c = _draw_gate(rng)
        return dict(c, kind="gate_bwd", T=min(c["T"], 65536))
    if kind == "mx":
        return dict(kind="mx", rows=_log_int(rng, 1, 28000), cols=32 * _log_int(rng, 1, 128),
                    src=rng.choice(["bf16", "f32"]))
    model = rng.choice(["mixtral", "deepseek", "tiny"])
    T = _log_int(rng, 1, 8192)
    return dict(kind="experts", model=model, T=T, act=rng.choice(["bf16", "mx4"]),
                pad=rng.choice([0, 0, T // 7]), spread=round(rng.uniform(0.5, 2.5), 2))


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _pow2(byte):
    """2^(byte - 127) of E8M0 bytes, exactly (byte 0 stands for 2^-127)."""
    b = byte.to(torch.int32)
    return torch.where(b == 0, 1 << 22, b << 23).view(torch.float32)


def _mx(x):
    """Blocks of 32 along the last dimension: (element values before scaling, E8M0 bytes), fp32 and uint8."""
    v = x.float().unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(-1, keepdim=True)
    e = torch.frexp(amax).exponent - 1 - 2
    byte = torch.where(amax > 0, e + 127, 0).clamp(0, 254).to(torch.uint8)
    # two exact steps: the reciprocal of the smallest scales is no finite number
    half = byte.int() // 2
    q = v * _pow2(254 - 127 + 64 - half) * _pow2(127 + 63 - (byte.int() - half))
    mag = q.abs()
    step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    mag = (torch.round(mag / step) * step).clamp(max=6.0)
    return torch.copysign(mag, q).flatten(-2), byte.squeeze(-1)


def _mx_values(x):
    q, byte = _mx(x)
    return (q.unflatten(-1, (-1, BLOCK)) * _pow2(byte).unsqueeze(-1)).flatten(-2)


def _to_codes(q):
    """E2M1 element values to two codes a byte, the even element in the low half."""
    m = (2 * q.abs()).to(torch.uint8)   # 0 1 2 3 4 6 8 12
    c = torch.where(m < 5, m, torch.where(m < 8, 5, torch.where(m < 12, 6, 7)).to(torch.uint8))
    c = c | (torch.signbit(q).to(torch.uint8) << 3)
    return (c[..., 0::2] | (c[..., 1::2] << 4)).contiguous()


def _from_codes(codes, byte):
    """fp32 values of E2M1 codes [..., n / 2] with scales [..., n / 32]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    k = c & 7
    mag = torch.where(k < 2, k, (2 + (k & 1)) << ((k >> 1).clamp(min=1) - 1))   # in halves
    v = mag.float().mul_(0.5).mul_(1.0 - 2.0 * (c >> 3).float())
    return (v.unflatten(-1, (-1, BLOCK)) * _pow2(byte).unsqueeze(-1)).flatten(-2)


def _gate_inputs(case, seed):
    """Router logits (spread: their deviation, which decides how uneven the routing is), the balance bias of a
    router in training, a learned mask or prior."""
    g = _gen(seed)
    T, E, K = case["T"], case["E"], case["K"]
    s = dict(logits=torch.randn((T, E), generator=g, device="cuda").mul_(case["spread"]))
    s["bias"] = torch.randn(E, generator=g, device="cuda").mul_(0.05 if case["score"] == "sigmoid" else 0.2 / E) \
        if case["bias"] else None
    rs = np.random.RandomState(seed % (1 << 31))
    s["mask"] = s["prior"] = None
    if case["mask"]:   # about three quarters of the experts, at least K of them
        m = np.zeros(E, np.uint8)
        m[rs.permutation(E)[:max(K, (3 * E) // 4)]] = 1
        s["mask"] = m
    if case["prior"]:
        w = np.exp(rs.rand(E) < 0.5)
        s["prior"] = (w / w.sum()).astype(np.float32)
    if case["kind"] == "gate_bwd":
        s["d_gate"] = torch.randn((T, K), generator=g, device="cuda")
        s["idx"] = _gate_plain(case, s)[0]
    return s


def _weights(g, n, rows, cols):
    codes = torch.empty((n, rows, cols // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n, rows, cols // BLOCK), dtype=torch.uint8, device="cuda")
    for i in range(n):
        w = torch.randn((rows, cols), generator=g, device="cuda", dtype=torch.bfloat16).mul_(cols ** -0.5)
        q, scales[i] = _mx(w)
        codes[i] = _to_codes(q)
    return codes, scales


def _expert_inputs(case, seed):
    """Tokens with a few loud channels, as activations have; MX weights from N(0, 1 / fan_in); routing by the
    softmax of random logits; the last `pad` tokens are empty slots that no expert sees."""
    m = MODELS[case["model"]]
    d, F, E, K, ns, T = m["d"], m["F"], m["E"], m["K"], m["ns"], case["T"]
    g = _gen(seed)
    loud = 1 + 7 * (torch.rand(d, generator=g, device="cuda") < 0.01)
    s = dict(x=(torch.randn((T, d), generator=g, device="cuda") * loud).bfloat16())
    s["gu_codes"], s["gu_scales"] = _weights(g, E + ns, 2 * F, d)
    s["dn_codes"], s["dn_scales"] = _weights(g, E + ns, d, F)
    p = torch.softmax(case["spread"] * torch.randn((T, E), generator=g, device="cuda"), -1)
    gate, idx = p.topk(K, -1)
    if m["renorm"]:
        gate = gate / gate.sum(-1, keepdim=True)
    idx, gate = idx.int().contiguous(), gate.contiguous()
    if case["pad"]:
        idx[T - case["pad"]:] = -1
        gate[T - case["pad"]:] = 0.0
    s["idx"], s["gate"] = idx, gate
    return s


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("gate", "gate_bwd"):
        s = _gate_inputs(case, seed)
    elif kind == "mx":
        x = torch.randn((case["rows"], case["cols"]), generator=_gen(seed), device="cuda")
        s = dict(x=x.bfloat16() if case["src"] == "bf16" else x)
    else:
        s = _expert_inputs(case, seed)
        # the host's view of the routing, which the plain form lays its rows out by
        flat = s["idx"].cpu().numpy().reshape(-1)
        s["active"], counts = np.unique(flat[flat >= 0], return_counts=True)
        s["cap"] = int(counts.max(initial=1))
        if own:   # the handle that a serving program keeps: packed weights, workspace
            from paper_2609_34077_amd import _lib as L
            m = MODELS[case["model"]]
            s["packed"] = L.maskmoe_mx4_pack_experts(s["gu_codes"], s["gu_scales"], s["dn_codes"], s["dn_scales"])
            s["workspace"] = torch.empty(
                L.maskmoe_experts_mx4_workspace_bytes(case["T"], m["d"], m["E"], m["K"], m["F"], m["ns"]),
                dtype=torch.uint8, device="cuda")
    s["case"] = dict(case)
    return s


# ---------------------------------------------------------------- one pass

def _scores(case, z):
    if case["score"] == "sigmoid":
        return torch.sigmoid(z)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _gate_plain(case, s):
    """Keys in 64 bits: a selection goes by differences of nearly equal keys."""
    z = s["logits"].double()
    T, E = z.shape
    G, n, K = case["groups"], E // case["groups"], case["K"]
    sc = _scores(case, z)
    key = sc
    if s["prior"] is not None:
        key = key * torch.from_numpy(s["prior"]).to(z.device).double()
    if s["bias"] is not None:
        key = key + s["bias"].double()
    if s["mask"] is not None:
        key = key.masked_fill(torch.from_numpy(s["mask"]).to(z.device) == 0, -math.inf)
    if G > 1:
        kg = key.view(T, G, n)
        top = kg.topk(min(2, n) if case["rule"] == "sum2" else 1, -1).values
        lead = top[..., 0] + torch.where(top[..., 1] == -math.inf, 0.0, top[..., 1]) if top.shape[-1] == 2 \
            else top[..., 0]
        order = torch.sort(lead, dim=-1, descending=True, stable=True).indices[:, :case["topk_group"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=z.device).scatter_(1, order, True)
        key = kg.masked_fill(~keep[..., None], -math.inf).view(T, E)
    best, idx = torch.sort(key, dim=-1, descending=True, stable=True)
    best, idx = best[:, :K], idx[:, :K]
    gate = sc.gather(1, idx)
    live = best > -math.inf
    gate = torch.where(live, gate, 0.0)
    if case["renorm"]:
        gate = gate / gate.sum(-1, keepdim=True)
    idx = torch.where(live, idx, -1)
    load = torch.bincount(idx.reshape(-1) + 1, minlength=E + 1)[1:]
    return idx.int().contiguous(), (case["scale"] * gate).float(), load.int()


def _gate_bwd_plain(case, s):
    z = s["logits"]
    idx = s["idx"].long()
    live = idx >= 0
    at = idx.clamp(min=0)
    p = _scores(case, z)
    w = torch.where(live, p.gather(1, at), 0.0)
    dg = torch.where(live, s["d_gate"], 0.0) * case["scale"]
    if case["renorm"]:
        total = w.sum(-1, keepdim=True)
        ds = (dg - (dg * w / total).sum(-1, keepdim=True)) / total
    else:
        ds = dg
    ds = torch.zeros_like(z).scatter_add_(1, at, torch.where(live, ds, 0.0))
    if case["score"] == "sigmoid":
        return ds * p * (1 - p)
    return p * (ds - (p * ds).sum(-1, keepdim=True))


def _ffn(x, wg, ws, dg, dsc, act):
    """SwiGLU experts on rows x [n, rows, d], weights of n experts."""
    ab = torch.bmm(x, _from_codes(wg, ws).transpose(1, 2))
    a, b = ab.chunk(2, -1)
    h = a / (1 + torch.exp(-a)) * b
    if act == "mx4":
        h = _mx_values(h)
    return torch.bmm(h, _from_codes(dg, dsc).transpose(1, 2))


def _experts_plain(case, s):
    m = MODELS[case["model"]]
    E, K, T, cap = m["E"], m["K"], case["T"], s["cap"]
    x = _mx_values(s["x"]) if case["act"] == "mx4" else s["x"].float()
    y = torch.zeros_like(x)
    if len(s["active"]):
        act = torch.from_numpy(s["active"]).to(x.device).long()
        flat = s["idx"].reshape(-1).long()
        order = torch.sort(flat, stable=True).indices          # entries by expert, empty ones first
        e = flat[order]
        first = torch.searchsorted(e, act)
        slot = torch.searchsorted(act, e.clamp(min=0)).clamp(max=len(act) - 1)
        pos = slot * cap + torch.arange(T * K, device=x.device) - first[slot]   # row in [active, cap]
        live = e >= 0
        rows = torch.zeros((len(act) * cap,) + x.shape[1:], device=x.device)
        rows[pos[live]] = x[(order // K)[live]]
        o = _ffn(rows.view(len(act), cap, -1), s["gu_codes"][act], s["gu_scales"][act], s["dn_codes"][act],
                 s["dn_scales"][act], case["act"]).view(len(act) * cap, -1)
        where = torch.empty_like(pos)
        where[order] = torch.where(live, pos, 0)
        y = (o[where].view(T, K, -1) * torch.where(s["idx"] >= 0, s["gate"], 0.0)[..., None]).sum(1)
    if m["ns"]:
        y = y + _ffn(x.expand(m["ns"], -1, -1), s["gu_codes"][E:], s["gu_scales"][E:], s["dn_codes"][E:],
                     s["dn_scales"][E:], case["act"]).sum(0)
    return y.bfloat16()


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        if kind == "gate":
            idx, gate, load = _gate_plain(case, s)
            return dict(idx=idx, gate=gate, load=load)
        if kind == "gate_bwd":
            return dict(d_logits=_gate_bwd_plain(case, s))
        if kind == "mx":
            return dict(values=_mx_values(s["x"]).bfloat16())
        return dict(y=_experts_plain(case, s))
    from paper_2609_34077_amd import _lib as L
    if kind in ("gate", "gate_bwd"):
        score = L.SCORE_SIGMOID if case["score"] == "sigmoid" else L.SCORE_SOFTMAX
        if kind == "gate_bwd":
            return dict(d_logits=L.maskmoe_gate_backward(s["logits"], s["idx"], s["d_gate"], score,
                                                         renorm=case["renorm"], scale=case["scale"]))
        idx, gate, load = L.maskmoe_gate_forward(
            s["logits"], case["K"], score, n_group=case["groups"], topk_group=case["topk_group"],
            group_rule=L.GROUP_SUM2 if case["rule"] == "sum2" else L.GROUP_MAX, renorm=case["renorm"],
            scale=case["scale"], bias=s["bias"], mask=s["mask"], prior=s["prior"], with_load=True)
        return dict(idx=idx, gate=gate, load=load)
    if kind == "mx":
        codes, scales = L.maskmoe_mx4_quantize(s["x"])
        return dict(values=L.maskmoe_mx4_dequantize(codes, scales, torch.bfloat16))
    return dict(y=L.maskmoe_experts_forward_mx4(
        s["x"], s["idx"], s["gate"], s["packed"], n_shared=MODELS[case["model"]]["ns"],
        act=L.ACT_MX4 if case["act"] == "mx4" else L.ACT_BF16, workspace=s["workspace"]))


def work(case):
    kind = case["kind"]
    if kind in ("gate", "gate_bwd"):
        T, E, K = case["T"], case["E"], case["K"]
        if kind == "gate":
            return dict(bytes=4 * T * E + 8 * T * K + 4 * E, flops=10 * T * E)
        dense = case["score"] == "softmax" and not case["renorm"]
        return dict(bytes=4 * T * E + 4 * T * (E if dense else K) + 8 * T * K, flops=(10 if dense else 1) * T * E)
    if kind == "mx":
        n = case["rows"] * case["cols"]
        return dict(bytes=int(n * ((2 if case["src"] == "bf16" else 4) + 2 * (0.5 + 1 / BLOCK) + 2)), flops=4 * n)
    m = MODELS[case["model"]]
    d, F, E, K, ns = m["d"], m["F"], m["E"], m["K"], m["ns"]
    T, live = case["T"], case["T"] - case["pad"]
    active = E * (1 - (1 - K / E) ** live) + ns   # experts read, uniform routing
    expert = 3 * d * F
    return dict(bytes=int(active * expert * (0.5 + 1 / BLOCK) + 4 * T * d + 8 * T * K),
                flops=2 * (live * K + T * ns) * expert)


# ---------------------------------------------------------------- the same in 64 bits

GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)   # E2M1 magnitudes in code order


def _mx64(x):
    """The values of x's MX blocks: nearest on the scaled grid, ties to the even code."""
    grid = GRID.to(x.device)
    mids = (grid[1:] + grid[:-1]) / 2
    v = x.double().reshape(-1, BLOCK)
    amax = v.abs().max(1, keepdim=True).values
    e = torch.where(amax > 0, torch.floor(torch.log2(amax)), -200.0)
    e = torch.where(amax < torch.exp2(e), e - 1, torch.where(amax >= torch.exp2(e + 1), e + 1, e))  # log2 at a border
    scale = torch.exp2((e - 2).clamp(min=-127))
    u = (v / scale).abs()
    i = torch.bucketize(u, mids)
    i = i + ((u == mids[i.clamp(max=mids.numel() - 1)]) & (i % 2 == 1) & (i < mids.numel())).long()
    return (torch.sign(v) * grid[i] * scale).view(x.shape)


def _weight64(codes, byte):
    grid = GRID.to(codes.device)
    lut = torch.cat((grid, -grid))
    c = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.long, device=codes.device)
    c[..., 0::2], c[..., 1::2] = codes % 16, codes // 16
    return lut[c] * torch.exp2(byte.double() - 127).repeat_interleave(BLOCK, -1)


def exact(case, seed):
    kind = case["kind"]
    if kind == "mx":
        s = prepare(case, seed)
        return dict(values=_mx64(s["x"]))
    if kind == "experts":
        s = _expert_inputs(case, seed)
        m = MODELS[case["model"]]
        E, F, ns = m["E"], m["F"], m["ns"]
        x = _mx64(s["x"]) if case["act"] == "mx4" else s["x"].double()
        y = torch.zeros_like(x)
        for e in range(E + ns):
            if e < E:
                t, k = (s["idx"] == e).nonzero(as_tuple=True)
                g = s["gate"][t, k].double()
            else:
                t = torch.arange(case["T"], device=x.device)
                g = torch.ones(case["T"], dtype=torch.float64, device=x.device)
            if not t.numel():
                continue
            ab = x[t] @ _weight64(s["gu_codes"][e], s["gu_scales"][e]).t()
            h = ab[:, :F] * torch.sigmoid(ab[:, :F]) * ab[:, F:]
            if case["act"] == "mx4":
                h = _mx64(h)
            y.index_add_(0, t, g[:, None] * (h @ _weight64(s["dn_codes"][e], s["dn_scales"][e]).t()))
        return dict(y=y)
    s = _gate_inputs(case, seed)
    z = s["logits"].double()
    T, E = z.shape
    sc = torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, -1)
    if kind == "gate_bwd":
        sel = s["idx"].long()
        hot = torch.zeros_like(z).scatter_add_(1, sel.clamp(min=0), (sel >= 0).double())
        zz = z.clone().requires_grad_(True)
        p = torch.sigmoid(zz) if case["score"] == "sigmoid" else torch.softmax(zz, -1)
        gate = p.gather(1, sel.clamp(min=0)) * (sel >= 0)
        if case["renorm"]:
            gate = gate / (p * hot).sum(-1, keepdim=True)
        (case["scale"] * gate * s["d_gate"].double()).sum().backward()
        return dict(d_logits=zz.grad)
    key = sc.clone()
    if s["prior"] is not None:
        key *= torch.tensor(s["prior"], dtype=torch.float64, device=z.device)
    if s["bias"] is not None:
        key += s["bias"].double()
    dead = torch.zeros((T, E), dtype=torch.bool, device=z.device)
    if s["mask"] is not None:
        dead |= torch.tensor(s["mask"] == 0, device=z.device)
    G, n = case["groups"], E // case["groups"]
    if G > 1:
        k3 = key.masked_fill(dead, -math.inf).view(T, G, n)
        lead = k3.max(-1).values
        if case["rule"] == "sum2" and n > 1:
            second = k3.scatter(2, k3.argmax(-1, keepdim=True), -math.inf).max(-1).values
            lead = lead + torch.where(torch.isinf(second), 0.0, second)
        out = torch.ones((T, G), dtype=torch.bool, device=z.device)
        for _ in range(case["topk_group"]):   # the best group left, the lowest of equal ones
            best = lead.masked_fill(~out, -math.inf).argmax(-1, keepdim=True)
            out.scatter_(1, best, False)
        dead |= out.repeat_interleave(n, -1)
    left = key.masked_fill(dead, -math.inf)
    idx, gate = [], []
    for _ in range(case["K"]):
        best = left.argmax(-1, keepdim=True)
        live = left.gather(1, best) > -math.inf
        idx.append(torch.where(live, best, -1))
        gate.append(torch.where(live, sc.gather(1, best), 0.0))
        left = left.scatter(1, best, -math.inf)
    idx, gate = torch.cat(idx, 1), torch.cat(gate, 1)
    if case["renorm"]:
        gate = gate / gate.sum(-1, keepdim=True)
    load = torch.stack([(idx == e).sum() for e in range(E)])
    return dict(idx=idx.int(), gate=case["scale"] * gate, load=load.int())

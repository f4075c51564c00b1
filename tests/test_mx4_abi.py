"""Refusals of the gate and MX4 entry points, without a GPU: every invalid argument is told before
anything is enqueued."""

import ctypes
import os

import numpy as np
import pytest
import torch

from paper_2609_34077_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libmaskmoe.so not built")

FAKE = 0x10000   # aligned, never read: only used where validation must fail


def gate_desc(**kw):
    d = dict(T=4, E=64, K=6, score=L.SCORE_SIGMOID, n_group=1, topk_group=1, group_rule=L.GROUP_MAX, renorm=1, scale=1.0)
    d.update(kw)
    return L.GateDesc(*[d[n] for n, _ in L.GateDesc._fields_])


def fwd(desc, logits=FAKE, mask=None, prior=None, bias=None, idx=FAKE, gate=FAKE, load=None):
    return L.load().maskmoe_gate_forward(ctypes.byref(desc), logits, mask, prior, bias, idx, gate, load, None)


def bwd(desc, logits=FAKE, idx=FAKE, dg=FAKE, out=FAKE):
    return L.load().maskmoe_gate_backward(ctypes.byref(desc), logits, idx, dg, out, None)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(E=0), dict(E=257), dict(K=0), dict(K=65), dict(K=17), dict(score=2),
                                dict(score=-1), dict(renorm=2), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_gate_rejects_descs(kw):
    assert fwd(gate_desc(**kw)) == L.E_INVAL and bwd(gate_desc(**kw)) == L.E_INVAL


@pytest.mark.parametrize("kw", [dict(n_group=0), dict(n_group=7), dict(n_group=128), dict(n_group=8, topk_group=0),
                                dict(n_group=8, topk_group=9), dict(n_group=16, topk_group=1), dict(group_rule=2)])
def test_gate_rejects_groups(kw):
    assert fwd(gate_desc(**kw)) == L.E_INVAL


def test_gate_rejects_pointers_and_priors():
    d = gate_desc()
    for kw in (dict(logits=None), dict(idx=None), dict(gate=None), dict(logits=FAKE + 2), dict(bias=FAKE + 1),
               dict(idx=FAKE + 1), dict(gate=FAKE + 3), dict(load=FAKE + 2)):
        assert fwd(d, **kw) == L.E_INVAL, kw
    for kw in (dict(logits=None), dict(idx=None), dict(dg=None), dict(out=None), dict(out=FAKE + 2)):
        assert bwd(d, **kw) == L.E_INVAL, kw
    for v in (0.0, -1.0, np.inf, np.nan):
        p = np.full(64, 0.5, np.float32)
        p[63] = v
        assert fwd(d, prior=p.ctypes.data_as(ctypes.c_void_p)) == L.E_INVAL
    lib = L.load()
    assert lib.maskmoe_gate_forward(None, FAKE, None, None, None, FAKE, FAKE, None, None) == L.E_INVAL
    assert lib.maskmoe_gate_backward(None, FAKE, FAKE, FAKE, FAKE, None) == L.E_INVAL
    assert bwd(gate_desc(T=0), logits=None, idx=None, dg=None, out=None) == L.OK
    assert fwd(gate_desc(T=0), logits=None, idx=None, gate=None) == L.OK


def test_gate_rejects_more_tokens_than_it_counts_and_gradients_in_place():
    d = gate_desc(T=(1 << 30) + 1, E=1, K=1)
    assert fwd(d) == L.E_UNSUPPORTED and bwd(d, out=FAKE + 64) == L.E_UNSUPPORTED
    assert bwd(gate_desc(), logits=FAKE, out=FAKE) == L.E_INVAL


@pytest.mark.parametrize("v", [2.0 ** -101, 2.0 ** 101])
def test_gate_rejects_priors_that_leave_the_range_of_keys(v):
    p = np.ones(64, np.float32)
    p[5] = v
    assert fwd(gate_desc(), prior=p.ctypes.data_as(ctypes.c_void_p)) == L.E_INVAL


def test_experts_mx4_rejects_launches_above_the_limit():
    for T, want in ((16, L.E_UNSUPPORTED), (17, L.E_WORKSPACE)):
        d = L.make_desc(T=T, d=64, E=256, K=16, F=1 << 21, n_shared=0)
        assert experts(d, ws=None) == want


@pytest.mark.parametrize("fn", ["maskmoe_mx4_quantize", "maskmoe_mx4_dequantize"])
def test_mx4_conversion_rejects(fn):
    f = getattr(L.load(), fn)
    assert f(-1, 32, L.BF16, FAKE, FAKE, FAKE, None) == L.E_INVAL
    assert f(1, 0, L.BF16, FAKE, FAKE, FAKE, None) == L.E_INVAL
    assert f(1, 32, 2, FAKE, FAKE, FAKE, None) == L.E_INVAL
    assert f(1, 48, L.F32, FAKE, FAKE, FAKE, None) == L.E_UNSUPPORTED
    assert f(1 << 40, 32, L.F32, FAKE, FAKE, FAKE, None) == L.E_UNSUPPORTED
    for i in range(3):
        a = [FAKE] * 3
        a[i] = None
        assert f(1, 32, L.BF16, *a, None) == L.E_INVAL
    vec, codes = (0, 1) if fn == "maskmoe_mx4_quantize" else (2, 0)
    for i in (vec, codes):
        a = [FAKE] * 3
        a[i] = FAKE + 8
        assert f(1, 32, L.BF16, *a, None) == L.E_INVAL
    assert f(0, 32, L.BF16, None, None, None, None) == L.OK


def test_mx4_packed_bytes_and_pack():
    lib = L.load()
    b = (ctypes.c_size_t * 4)()
    d = L.make_desc(0, 192, 1, 1, 320)
    assert lib.maskmoe_mx4_packed_bytes(ctypes.byref(d), 3, b) == L.OK
    # 640 rows of two 128-column steps (1.5 used), 192 rows of three; scales of up to four steps per dword
    assert list(b) == [3 * 40 * 2 * 1024, 3 * 40 * 256, 3 * 12 * 3 * 1024, 3 * 12 * 256]
    for kw in (dict(d=96), dict(F=80), dict(d=1 << 16, F=1 << 15)):
        bad = L.make_desc(0, **{**dict(d=192, E=1, K=1, F=320), **kw})
        assert lib.maskmoe_mx4_packed_bytes(ctypes.byref(bad), 1, b) == L.E_UNSUPPORTED, kw
    assert lib.maskmoe_mx4_packed_bytes(ctypes.byref(d), -1, b) == L.E_INVAL
    assert lib.maskmoe_mx4_packed_bytes(None, 1, b) == L.E_INVAL
    assert lib.maskmoe_mx4_packed_bytes(ctypes.byref(d), 1, None) == L.E_INVAL
    src, dst = L.Mx4Experts(*[FAKE + 4096 * i for i in range(4)]), L.Mx4Experts(*[FAKE + 4096 * (i + 8) for i in range(4)])

    def pack(s, p, n=1):
        return lib.maskmoe_mx4_pack_experts(ctypes.byref(d), n, s and ctypes.byref(s), p and ctypes.byref(p), None)
    assert pack(None, dst) == L.E_INVAL and pack(src, None) == L.E_INVAL and pack(src, src) == L.E_INVAL
    for f, _ in L.Mx4Experts._fields_:
        bad = L.Mx4Experts(*[getattr(dst, n) for n, _ in L.Mx4Experts._fields_])
        setattr(bad, f, getattr(dst, f) + 8)
        assert pack(src, bad) == L.E_INVAL, f
        setattr(bad, f, None)
        assert pack(src, bad) == L.E_INVAL and pack(bad, dst) == L.E_INVAL, f
    assert pack(None, None, n=0) == L.OK


def experts(desc, act=0, x=FAKE, idx=FAKE, gate=FAKE, w=None, y=FAKE + 65536, ws=FAKE, ws_bytes=1 << 40):
    w = L.Mx4Experts(FAKE, FAKE, FAKE, FAKE) if w is None else w
    return L.load().maskmoe_experts_forward_mx4(ctypes.byref(desc), act, x, idx, gate, ctypes.byref(w), y, ws, ws_bytes, None)


def test_experts_mx4_rejects():
    ok = dict(T=4, d=64, E=8, K=2, F=64, n_shared=1)
    lib = L.load()
    for kw in (dict(T=-1), dict(E=0), dict(E=257), dict(K=0), dict(K=9), dict(n_shared=9), dict(n_shared=-1), dict(d=0),
               dict(F=0), dict(dtype=5)):
        d = L.make_desc(**{**ok, **kw})
        assert experts(d) == L.E_INVAL, kw
        assert lib.maskmoe_experts_mx4_workspace_bytes(ctypes.byref(d)) == 0
    for kw in (dict(d=96), dict(F=96), dict(dtype=L.F32), dict(T=1 << 25, d=4096), dict(d=1 << 16, F=1 << 15),
               dict(T=1 << 20, F=1024)):
        assert experts(L.make_desc(**{**ok, **kw})) == L.E_UNSUPPORTED, kw
    d = L.make_desc(**ok)
    for kw in (dict(act=2), dict(x=None), dict(x=FAKE + 8), dict(idx=None), dict(idx=FAKE + 2), dict(gate=None), dict(y=None),
               dict(y=FAKE), dict(y=FAKE + 8), dict(w=L.Mx4Experts(FAKE, FAKE, None, FAKE)),
               dict(w=L.Mx4Experts(FAKE, FAKE + 4, FAKE, FAKE))):
        assert experts(d, **kw) == L.E_INVAL, kw
    need = lib.maskmoe_experts_mx4_workspace_bytes(ctypes.byref(d))
    for kw in (dict(ws=None), dict(ws=FAKE + 128), dict(ws_bytes=need - 1)):
        assert experts(d, **kw) == L.E_WORKSPACE, kw
    assert experts(L.make_desc(**{**ok, "T": 0}), x=None, y=None, idx=None, gate=None, ws=None) == L.OK


def test_experts_mx4_workspace_is_monotone_in_tokens():
    f = lambda T: L.maskmoe_experts_mx4_workspace_bytes(T, 192, 64, 6, 320, 2)
    sizes = [f(T) for T in (0, 1, 16, 17, 100, 1000, 5000)]
    assert sizes == sorted(sizes)


def test_sizes_that_int32_does_not_hold():
    """ctypes would pass their low 32 bits: a batch of 2^32 + 5 rows as one of 5, whose other results nothing writes."""
    meta = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="meta")
    i32, u8 = torch.int32, torch.uint8
    few = meta(4, 64)
    calls = [lambda: L.maskmoe_gate_forward(meta(2 ** 32 + 5, 1), 1, L.SCORE_SOFTMAX),
             lambda: L.maskmoe_gate_forward(few, 2 ** 32 + 2, L.SCORE_SOFTMAX),
             lambda: L.maskmoe_gate_forward(few, 2, L.SCORE_SOFTMAX, n_group=2 ** 32 + 8, topk_group=2),
             lambda: L.maskmoe_gate_backward(meta(2 ** 32 + 5, 1), meta(2 ** 32 + 5, 1, dtype=i32), meta(2 ** 32 + 5, 1), 0),
             lambda: L.maskmoe_gate_backward(meta(1, 8), meta(1, 2 ** 32 + 2, dtype=i32), meta(1, 2 ** 32 + 2), 0),
             lambda: L.maskmoe_mx4_quantize(meta(2 ** 32 + 32)),
             lambda: L.maskmoe_mx4_dequantize(meta(2 ** 31 + 16, dtype=u8), meta(2 ** 27 + 1, dtype=u8), torch.bfloat16)]
    packed = L.PackedMx4Experts(4, 64, 64, [torch.empty(1, dtype=u8)] * 4)
    calls.append(lambda: L.maskmoe_experts_forward_mx4(meta(4, 64), meta(4, 2, dtype=i32), meta(4, 2), packed, n_shared=2 ** 32))
    for f in calls:
        with pytest.raises(ValueError, match="below 2"):
            f()

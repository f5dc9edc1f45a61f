"""Host-side checks of include/rope.h, include/norm.h, include/xattn.h and the norm of include/w8a8.h (no GPU needed): the
library exports what the headers declare, and every refusal comes before any launch."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2512_16093_amd import binding as sla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(0x1000)      # non-NULL, 16-byte aligned, never dereferenced: a refusal comes first
ODD = ctypes.c_void_p(0x1008)
WS = ctypes.c_void_p(0x10000)
BIG = 1 << 44


def _declared(header, prefix):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    return set(re.findall(r"\b(%s_[a-z0-9_]+)\s*\(" % prefix, text))


@pytest.mark.parametrize("prefix,names", [("rope", sla.ROPE_EXPORTS), ("norm", sla.NORM_EXPORTS), ("xattn", sla.XATTN_EXPORTS)])
def test_library_exports_every_declared_symbol(prefix, names):
    assert _declared(prefix + ".h", prefix) == set(names)
    for n in names:
        assert hasattr(sla.lib(), n), n


def test_status_of_a_scalar_out_of_range():
    assert "range" in sla.sla_status_string(sla.ERR_VALUE) and sla.sla_status_string(sla.ERR_VALUE) != "unknown status"


def test_plans():
    p = sla.rope_make_plan((22, 21, 21), (10000.0, 10000.0, 500.0), "halves")
    assert list(p.axis) == [0] * 22 + [1] * 21 + [2] * 21 and p.pairing == 1
    for j, (base, i, n) in enumerate([(10000.0, i, 22) for i in range(22)] + [(10000.0, i, 21) for i in range(21)] +
                                     [(500.0, i, 21) for i in range(21)]):
        assert abs(p.turns[j] * 2.0 ** -64 * 6.283185307179586 - base ** (-i / n)) < 1e-15
    # at the farthest position the angle is off by less than 2^-28 turns, whatever the base
    turn = 2 * np.longdouble("3.14159265358979323846264338327950288")
    for pairs in ((64, 0, 0), (1, 62, 1), (10, 20, 34)):
        for base in (1.0, 1.0000001, 1.5, 500.0, 1e12):
            p, j = sla.rope_make_plan(pairs, base), 0
            for n in pairs:
                for i in range(n):
                    want = np.longdouble(base) ** (-np.longdouble(i) / n) / turn
                    assert abs(float(np.longdouble(p.turns[j]) / np.longdouble(2) ** 64 - want)) * 2 ** 31 < 2 ** -28, (pairs, base, i)
                    j += 1
    L = sla.lib()
    out = sla.RopePlan()

    def make(pairs=(22, 21, 21), theta=(1e4, 1e4, 1e4), pairing=0):
        return L.rope_make_plan((ctypes.c_int32 * 3)(*pairs), (ctypes.c_double * 3)(*theta), pairing, ctypes.byref(out))
    assert make() == sla.SLA_OK and make(pairs=(0, 0, 64)) == sla.SLA_OK
    assert make(pairs=(22, 21, 20)) == sla.ERR_SHAPE and make(pairs=(-1, 44, 21)) == sla.ERR_SHAPE
    assert make(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 66)) == sla.ERR_SHAPE
    for bad in (0.5, 0.0, -1.0, 1e13, float("nan"), float("inf")):
        assert make(theta=(1e4, bad, 1e4)) == sla.ERR_VALUE
    assert make(pairing=2) == sla.ERR_UNSUPPORTED
    assert L.rope_make_plan(None, (ctypes.c_double * 3)(1, 1, 1), 0, ctypes.byref(out)) == sla.ERR_NULL
    for bad in (dict(pairs=(64,)), dict(theta=(1.0, 2.0)), dict(pairing="both")):
        with pytest.raises(ValueError):
            sla.rope_make_plan(**bad)


def _st(*s):
    return ctypes.byref(sla.Strides(*s))


def test_rope_argument_errors():
    L, plan = sla.lib(), sla.rope_make_plan()

    def fwd(q=FAKE, k=FAKE, qo=FAKE, ko=FAKE, qs=None, kos=None, pos=FAKE, pb=0, qw=FAKE, norm=2, eps=1e-6, B=1, H=4, Hk=4, N=10,
            d=128, plan=plan):
        return L.rope_qk_fwd(q, k, qo, ko, qs, None, None, kos, pos, pb, qw, FAKE, norm, eps, B, H, Hk, N, d,
                             None if plan is None else ctypes.byref(plan), None)

    for kw in (dict(q=None), dict(qo=None), dict(ko=None), dict(k=None), dict(pos=None), dict(plan=None)):
        assert fwd(**kw) == sla.ERR_NULL, kw
    for kw in (dict(B=0), dict(N=0), dict(H=0), dict(H=65), dict(Hk=0), dict(Hk=65), dict(d=64), dict(N=1 << 24), dict(B=1 << 12, N=1 << 12)):
        assert fwd(**kw) == sla.ERR_SHAPE, kw
    for kw in (dict(norm=3), dict(norm=-1), dict(plan=sla.RopePlan())):
        assert fwd(**kw) == sla.ERR_UNSUPPORTED, kw
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-60, 1e300):
        assert fwd(eps=eps) == sla.ERR_VALUE
    for kw in (dict(q=ODD), dict(ko=ODD), dict(qw=ODD), dict(pb=29), dict(pb=-30), dict(pos=ctypes.c_void_p(0x1002)),
               dict(qs=_st(0, 128, 100)), dict(kos=_st(5120, 132, 512)), dict(qs=_st(-8, 128, 512))):
        assert fwd(**kw) == sla.ERR_LAYOUT, kw

    need = sla.rope_bwd_workspace_bytes(1, 4, 2, 10, 128, "token")
    assert need == 3 * 4 * 128 * 4 + 3 * 2 * 128 * 4          # ten tokens: three workgroups of four teams
    assert sla.rope_bwd_workspace_bytes(1, 4, 2, 10, 64, "token") == 0 and sla.rope_bwd_workspace_bytes(1, 65, 2, 10, 128, "head") == 0

    def bwd(dqo=FAKE, dko=FAKE, q=FAKE, k=FAKE, dq=FAKE, dk=FAKE, dqw=FAKE, dkw=FAKE, s=None, norm=2, eps=1e-6, Hk=2, ws=WS, wsb=BIG):
        return L.rope_qk_bwd(dqo, dko, q, k, dq, dk, dqw, dkw, s, FAKE, 0, None, None, norm, eps, 1, 4, Hk, 10, 128,
                             ctypes.byref(plan), ws, wsb, None)

    for kw in (dict(dqo=None), dict(dq=None), dict(dk=None), dict(dko=None), dict(q=None), dict(k=None), dict(dko=None, dk=None)):
        assert bwd(**kw) == sla.ERR_NULL, kw
    assert bwd(norm=0) == sla.ERR_UNSUPPORTED and bwd(norm=7, dqw=None, dkw=None) == sla.ERR_UNSUPPORTED
    assert bwd(Hk=0) == sla.ERR_SHAPE and bwd(eps=0.0) == sla.ERR_VALUE
    assert bwd(ws=None) == sla.ERR_WORKSPACE and bwd(wsb=need - 1) == sla.ERR_WORKSPACE
    assert bwd(ws=ctypes.c_void_p(0x10010)) == sla.ERR_WORKSPACE
    bad = sla.RopeBwdStrides(None, None, None, ctypes.pointer(sla.Strides(0, 0, 64)), None, None)
    assert bwd(s=ctypes.byref(bad)) == sla.ERR_LAYOUT and bwd(dqw=ctypes.c_void_p(0x1002)) == sla.ERR_LAYOUT


def test_norm_argument_errors():
    L = sla.lib()

    def fwd(x=FAKE, res=FAKE, w=FAKE, h=FAKE, y=FAKE, M=3, K=64, eps=1e-6):
        return L.norm_rms_fwd(x, res, w, h, y, M, K, eps, None)

    for kw in (dict(x=None), dict(y=None), dict(h=None), dict(res=None)):
        assert fwd(**kw) == sla.ERR_NULL, kw
    shapes = (dict(M=0), dict(M=(1 << 22) + 1), dict(K=0), dict(K=4), dict(K=100), dict(K=16392))
    for kw in shapes:
        assert fwd(**kw) == sla.ERR_SHAPE, kw
    assert fwd(eps=0.0) == sla.ERR_VALUE and fwd(eps=float("nan")) == sla.ERR_VALUE
    for kw in (dict(x=ODD), dict(res=ODD), dict(w=ODD), dict(h=ODD), dict(y=ODD)):
        assert fwd(**kw) == sla.ERR_LAYOUT, kw
    need = sla.norm_bwd_workspace_bytes(9, 64)
    assert need == 3 * 64 * 4 and sla.norm_bwd_workspace_bytes(9, 60) == 0

    def bwd(dy=FAKE, dh=FAKE, h=FAKE, w=FAKE, dx=FAKE, dw=FAKE, M=9, K=64, eps=1e-6, ws=WS, wsb=BIG):
        return L.norm_rms_bwd(dy, dh, h, w, dx, dw, M, K, eps, ws, wsb, None)

    for kw in (dict(dy=None), dict(h=None), dict(dx=None)):
        assert bwd(**kw) == sla.ERR_NULL, kw
    for kw in shapes:
        assert bwd(**kw) == sla.ERR_SHAPE, kw
    assert bwd(eps=-1.0) == sla.ERR_VALUE and bwd(ws=None) == sla.ERR_WORKSPACE and bwd(wsb=need - 1) == sla.ERR_WORKSPACE
    for kw in (dict(dy=ODD), dict(dh=ODD), dict(h=ODD), dict(w=ODD), dict(dx=ODD), dict(dw=ctypes.c_void_p(0x1001))):
        assert bwd(**kw) == sla.ERR_LAYOUT, kw


def test_norm_linear_argument_errors():
    L = sla.lib()
    need = sla.w8a8_norm_workspace_bytes(300, 384)
    assert need == sla.w8a8_workspace_bytes(300, 384) + (300 * 4 + 255) // 256 * 256
    for bad in ((0, 128), (5, 100), (5, 16384 + 128), ((1 << 22) + 1, 128)):
        assert sla.w8a8_norm_workspace_bytes(*bad) == 0

    def quant(x=FAKE, res=FAKE, w=FAKE, h=FAKE, M=300, K=384, eps=1e-6, ws=WS, wsb=BIG):
        return L.w8a8_norm_quantize_act(x, res, w, h, M, K, eps, ws, wsb, None)

    def linear(wq=WS, bias=None, y=FAKE, N=256, **kw):
        a = dict(dict(x=FAKE, res=FAKE, w=FAKE, h=FAKE, M=300, K=384, eps=1e-6, ws=WS, wsb=BIG), **kw)
        return L.w8a8_norm_linear_fwd(a["x"], a["res"], a["w"], a["h"], wq, bias, y, a["M"], N, a["K"], a["eps"], a["ws"], a["wsb"], None)

    for call in (quant, linear):
        for kw in (dict(x=None), dict(res=None), dict(h=None)):
            assert call(**kw) == sla.ERR_NULL, kw
        for kw in (dict(M=0), dict(K=130), dict(K=16512)):
            assert call(**kw) == sla.ERR_SHAPE, kw
        assert call(eps=0.0) == sla.ERR_VALUE
        assert call(ws=None) == sla.ERR_WORKSPACE and call(wsb=need - 1) == sla.ERR_WORKSPACE
        for kw in (dict(x=ODD), dict(res=ODD), dict(w=ODD), dict(h=ODD)):
            assert call(**kw) == sla.ERR_LAYOUT, kw
    assert linear(wq=None) == sla.ERR_NULL and linear(y=None) == sla.ERR_NULL and linear(N=100) == sla.ERR_SHAPE
    assert linear(wq=ctypes.c_void_p(0x10010)) == sla.ERR_WORKSPACE
    assert linear(y=ODD) == sla.ERR_LAYOUT and linear(bias=ctypes.c_void_p(0x1004)) == sla.ERR_LAYOUT


def test_xattn_argument_errors():
    L = sla.lib()
    need, need_b = sla.xattn_workspace_bytes(1, 40, 10, 1, 8192, 128), sla.xattn_bwd_workspace_bytes(1, 40, 10, 1, 8192, 128)
    assert need > 2 * 40 * 128 * 4 and need_b > 2 * 40 * 128 * 4                     # few queries: pieces of the walk over the keys
    assert sla.xattn_workspace_bytes(1, 40, 40, 75600, 512, 128) == 256
    shapes = (dict(B=0), dict(H=0), dict(Hkv=0), dict(Nq=0), dict(Nk=0), dict(d=64), dict(H=40, Hkv=12), dict(B=65536, H=1, Hkv=1),
              dict(H=64, Hkv=64, Nq=1 << 24), dict(H=64, Hkv=64, Nk=1 << 24))
    strides = (sla.Strides(0, 0, 64), sla.Strides(0, 132, 256), sla.Strides(-8, 128, 256))

    def fwd(q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=None, qs=None, vs=None, lens=None, B=1, H=40, Hkv=10, Nq=1, Nk=8192, d=128, scale=0.0,
            ws=WS, wsb=BIG):
        return L.xattn_fwd(q, k, v, out, lse, qs, None, vs, None, lens, B, H, Hkv, Nq, Nk, d, scale, ws, wsb, None)

    def bwd(s=None, lens=None, B=1, H=40, Hkv=10, Nq=1, Nk=8192, d=128, scale=0.0, ws=WS, wsb=BIG, **kw):
        p = [kw.get(n, FAKE) for n in ("q", "k", "v", "out", "dout", "lse", "dq", "dk", "dv")]
        return L.xattn_bwd(*p, s, lens, B, H, Hkv, Nq, Nk, d, scale, ws, wsb, None)

    for n in ("q", "k", "v", "out"):
        assert fwd(**{n: None}) == sla.ERR_NULL and fwd(**{n: ODD}) == sla.ERR_LAYOUT, n
    for n in ("q", "k", "v", "out", "dout", "lse", "dq", "dk", "dv"):
        assert bwd(**{n: None}) == sla.ERR_NULL, n
        assert bwd(**{n: ODD if n != "lse" else ctypes.c_void_p(0x1002)}) == sla.ERR_LAYOUT, n
    for call, bytes_ in ((fwd, need), (bwd, need_b)):
        for kw in shapes:
            assert call(**kw) == sla.ERR_SHAPE, kw
        for bad in (-0.1, float("nan"), float("inf"), 1e-40):
            assert call(scale=bad) == sla.ERR_VALUE
        assert call(ws=None) == sla.ERR_WORKSPACE and call(wsb=bytes_ - 1) == sla.ERR_WORKSPACE
        assert call(ws=ctypes.c_void_p(0x10010)) == sla.ERR_WORKSPACE
        assert call(lens=ctypes.c_void_p(0x1002)) == sla.ERR_LAYOUT
    for bad in strides:
        assert fwd(qs=ctypes.byref(bad)) == sla.ERR_LAYOUT and fwd(vs=ctypes.byref(bad)) == sla.ERR_LAYOUT
        for i in range(8):
            each = [None] * 8
            each[i] = ctypes.pointer(bad)
            assert bwd(s=ctypes.byref(sla.XattnBwdStrides(*each))) == sla.ERR_LAYOUT
    for kw in shapes:
        a = dict(dict(B=1, H=40, Hkv=10, Nq=1, Nk=8192, d=128), **kw)
        assert sla.xattn_workspace_bytes(**a) == 0 and sla.xattn_bwd_workspace_bytes(**a) == 0


def test_binding_refuses_wrong_tensors():
    x = torch.zeros((1, 2, 64, 128), dtype=torch.bfloat16)      # CPU tensors
    m = torch.zeros((4, 128), dtype=torch.bfloat16)
    pos, plan = torch.zeros((64, 3), dtype=torch.int32), sla.rope_make_plan()
    for call in (lambda: sla.rope_qk_fwd(x, x, pos, plan), lambda: sla.rope_qk_bwd(x, x, pos, plan),
                 lambda: sla.rope_qk_fwd(x, x, pos, plan, norm="row"), lambda: sla.norm_rms_fwd(m, None),
                 lambda: sla.norm_rms_bwd(m, m, None), lambda: sla.w8a8_norm_quantize_act(m, None),
                 lambda: sla.w8a8_norm_linear_fwd(m, None, m, 128), lambda: sla.xattn_fwd(x, x, x), lambda: sla.xattn_fwd(x, x, x, scale=-1.0),
                 lambda: sla.xattn_bwd(x, x, x, x, x, torch.zeros(128))):
        with pytest.raises(ValueError):
            call()

"""Host-side checks of the layer norm of include/norm.h and of include/mxfp4.h (no GPU needed): the library exports what the
headers declare, and every refusal comes before any launch."""
import ctypes
import os
import re

import pytest
import torch

from paper_2512_16093_amd import binding as sla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(0x1000)      # non-NULL, 16-byte aligned, never dereferenced: a refusal comes first
ODD = ctypes.c_void_p(0x1008)
WS = ctypes.c_void_p(0x10000)
BIG = 1 << 44


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mxfp4.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(mxfp4_[a-z0-9_]+)\s*\(", text)) == set(sla.MXFP4_EXPORTS)
    for n in sla.MXFP4_EXPORTS:
        assert hasattr(sla.lib(), n), n


def _mod(gate=None, scale=0x1000, shift=0x1000, strides=(64, 64, 64), rows=3):
    return ctypes.byref(sla.NormModulation(gate, scale, shift, *strides, rows))


SHAPES = (dict(M=0), dict(M=(1 << 22) + 1), dict(K=0), dict(K=4), dict(K=100), dict(K=16392))
EPS = (0.0, -1.0, float("nan"), float("inf"), 1e-60, 1e300)


def _layer_refusals(call):
    """What every forward form of the layer norm refuses; call(x, res, w, b, mod, h, M, K, eps)."""
    assert call(x=None) == call(h=None) == call(res=None) == sla.ERR_NULL
    assert call(res=None, h=None, mod=_mod(gate=0x1000)) == sla.ERR_NULL
    for kw in SHAPES + (dict(mod=_mod(rows=0)), dict(mod=_mod(rows=-1))):
        assert call(**kw) == sla.ERR_SHAPE, kw
    for eps in EPS:
        assert call(eps=eps) == sla.ERR_VALUE
    for kw in (dict(x=ODD), dict(res=ODD), dict(w=ODD), dict(b=ODD), dict(h=ODD), dict(mod=_mod(gate=0x1008)), dict(mod=_mod(scale=0x1004)),
               dict(mod=_mod(shift=0x1008)), dict(mod=_mod(strides=(64, 66, 64))), dict(mod=_mod(strides=(64, 64, -64))),
               dict(mod=_mod(gate=0x1000, strides=(2, 64, 64)))):
        assert call(**kw) == sla.ERR_LAYOUT, kw


def test_layer_norm_argument_errors():
    L = sla.lib()

    def fwd(x=FAKE, res=FAKE, w=FAKE, b=FAKE, mod=None, h=FAKE, y=FAKE, M=3, K=64, eps=1e-6):
        return L.norm_layer_fwd(x, res, w, b, mod, h, y, M, K, eps, None)
    _layer_refusals(fwd)
    assert fwd(y=None) == sla.ERR_NULL and fwd(y=ODD) == sla.ERR_LAYOUT

    need = sla.norm_layer_bwd_workspace_bytes(30, 64, 10)
    assert need > 0 and need % 256 == 0
    for bad in ((0, 64, 1), (3, 60, 1), (3, 64, 0), (3, 16392, 3)):
        assert sla.norm_layer_bwd_workspace_bytes(*bad) == 0, bad

    def bwd(dy=FAKE, dh=FAKE, h=FAKE, res=FAKE, w=FAKE, b=FAKE, mod=None, dx=FAKE, dres=None, grads=(0x1000, 0x1000, None, None, None),
            M=30, K=64, eps=1e-6, ws=WS, wsb=BIG):
        g = None if grads is None else ctypes.byref(sla.NormLayerGrads(*grads))
        return L.norm_layer_bwd(dy, dh, h, res, w, b, mod, dx, dres, g, M, K, eps, ws, wsb, None)
    gated = _mod(gate=0x1000, rows=10)
    for kw in (dict(dy=None), dict(h=None), dict(dx=None), dict(dres=FAKE), dict(dres=FAKE, mod=_mod()), dict(grads=(None, None, 0x1000, None, None)),
               dict(grads=(None, None, 0x1000, None, None), mod=gated, res=None)):
        assert bwd(**kw) == sla.ERR_NULL, kw
    for kw in SHAPES + (dict(mod=_mod(rows=0)),):
        assert bwd(**kw) == sla.ERR_SHAPE, kw
    for eps in EPS:
        assert bwd(eps=eps) == sla.ERR_VALUE
    for kw in (dict(ws=None), dict(ws=ctypes.c_void_p(0x10010)), dict(mod=gated, wsb=need - 1)):
        assert bwd(**kw) == sla.ERR_WORKSPACE, kw
    for kw in (dict(dy=ODD), dict(dh=ODD), dict(h=ODD), dict(res=ODD), dict(w=ODD), dict(b=ODD), dict(dx=ODD), dict(dres=ODD, mod=gated),
               dict(grads=(0x1004, None, None, None, None)), dict(grads=(None, None, None, 0x1008, None)), dict(mod=_mod(scale=0x1004)),
               dict(mod=_mod(gate=0x1000, strides=(6, 64, 64)))):
        assert bwd(**kw) == sla.ERR_LAYOUT, kw
    assert bwd(grads=None, ws=None, wsb=0, dy=ODD) == sla.ERR_LAYOUT          # (no vector's gradient: no workspace asked for)


def test_object_sizes():
    behind = 256 * 64                                   # (what a tile of the product may read behind the last row)
    assert sla.mxfp4_bytes(1, 8) == 32 * 128 + 256 + behind == sla.mxfp4_bytes(32, 256)
    assert sla.mxfp4_bytes(33, 264) == 64 * 2 * 128 + 64 * 2 * 8 + behind
    assert sla.mxfp4_bytes(1 << 22, 65536) == (1 << 22) * 256 * 136 + behind
    for bad in ((0, 64), (-1, 64), ((1 << 22) + 1, 64), (1, 0), (1, 4), (1, 36), (1, 65544)):
        assert sla.mxfp4_bytes(*bad) == 0, bad


def test_mxfp4_argument_errors():
    L = sla.lib()
    need = sla.mxfp4_bytes(3, 64)
    calls = {
        "quantize": lambda x=FAKE, q=WS, qb=BIG, R=3, K=64: L.mxfp4_quantize(x, R, K, q, qb, None),
        "dequantize": lambda x=FAKE, q=WS, qb=BIG, R=3, K=64: L.mxfp4_dequantize(q, qb, R, K, x, None),
        "pack": lambda x=FAKE, q=WS, qb=BIG, R=3, K=64: L.mxfp4_pack(x, x, R, K, q, qb, None),
        "unpack": lambda x=FAKE, q=WS, qb=BIG, R=3, K=64: L.mxfp4_unpack(q, qb, R, K, x, x, None),
    }
    for name, f in calls.items():
        assert f(q=None) == sla.ERR_NULL, name
        if name != "unpack":
            assert f(x=None) == sla.ERR_NULL, name
        for kw in (dict(R=0), dict(R=(1 << 22) + 1), dict(K=0), dict(K=12), dict(K=65544)):
            assert f(**kw) == sla.ERR_SHAPE, (name, kw)
        for kw in (dict(q=ctypes.c_void_p(0x10080)), dict(qb=need - 1)):
            assert f(**kw) == sla.ERR_WORKSPACE, (name, kw)
        if name.endswith("quantize"):
            assert f(x=ODD) == sla.ERR_LAYOUT, name
    assert L.mxfp4_pack(FAKE, None, 3, 64, WS, BIG, None) == sla.ERR_NULL

    def gemm(xq=WS, xb=BIG, wq=WS, wb=BIG, bias=FAKE, y=FAKE, M=3, N=8, K=64):
        return L.mxfp4_gemm_fwd(xq, xb, wq, wb, bias, y, M, N, K, None)

    def linear(x=FAKE, wq=WS, wb=BIG, bias=FAKE, y=FAKE, M=3, N=8, K=64, ws=WS, wsb=BIG):
        return L.mxfp4_linear_fwd(x, wq, wb, bias, y, M, N, K, ws, wsb, None)

    def norm_linear(x=FAKE, res=FAKE, w=FAKE, b=FAKE, mod=None, h=FAKE, wq=WS, wb=BIG, bias=FAKE, y=FAKE, M=3, N=8, K=64, eps=1e-6, ws=WS,
                    wsb=BIG):
        return L.mxfp4_norm_linear_fwd(x, res, w, b, mod, h, wq, wb, bias, y, M, N, K, eps, ws, wsb, None)

    def norm_quantize(x=FAKE, res=FAKE, w=FAKE, b=FAKE, mod=None, h=FAKE, q=WS, qb=BIG, M=3, K=64, eps=1e-6):
        return L.mxfp4_norm_quantize(x, res, w, b, mod, h, q, qb, M, K, eps, None)
    _layer_refusals(norm_linear)
    _layer_refusals(norm_quantize)
    assert norm_quantize(q=None) == sla.ERR_NULL
    assert norm_quantize(qb=need - 1) == norm_quantize(q=ctypes.c_void_p(0x10010)) == sla.ERR_WORKSPACE
    for f in (gemm, linear, norm_linear):
        assert f(wq=None) == f(y=None) == sla.ERR_NULL
        for kw in (dict(M=0), dict(M=(1 << 22) + 1), dict(N=0), dict(N=4), dict(N=65544), dict(K=60)):
            assert f(**kw) == sla.ERR_SHAPE, kw
        for kw in (dict(wq=ctypes.c_void_p(0x10010)), dict(wb=sla.mxfp4_bytes(8, 64) - 1)):
            assert f(**kw) == sla.ERR_WORKSPACE, kw
        for kw in (dict(bias=ODD), dict(y=ODD)):
            assert f(**kw) == sla.ERR_LAYOUT, kw
    assert gemm(xq=None) == linear(x=None) == sla.ERR_NULL
    assert gemm(xb=need - 1) == gemm(xq=ctypes.c_void_p(0x10010)) == sla.ERR_WORKSPACE
    for f in (linear, norm_linear):
        for kw in (dict(ws=None), dict(ws=ctypes.c_void_p(0x10010)), dict(wsb=need - 1)):
            assert f(**kw) == sla.ERR_WORKSPACE, kw
    assert linear(x=ODD) == sla.ERR_LAYOUT


def test_binding_refuses_tensors_that_are_not_what_it_says():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)          # (on the CPU: refused, whatever else is right)
    q = torch.zeros(sla.mxfp4_bytes(4, 64), dtype=torch.uint8)
    for f in (lambda: sla.norm_layer_fwd(x), lambda: sla.norm_layer_bwd(x, x), lambda: sla.mxfp4_quantize(x),
              lambda: sla.mxfp4_dequantize(q, 4, 64), lambda: sla.mxfp4_unpack(q, 4, 64), lambda: sla.mxfp4_linear_fwd(x, q, 4),
              lambda: sla.mxfp4_gemm_fwd(q, q, 4, 4, 64), lambda: sla.mxfp4_norm_linear_fwd(x, q, 8), lambda: sla.mxfp4_norm_quantize(x),
              lambda: sla.mxfp4_pack(q.view(-1, 32), q.view(-1, 32))):
        with pytest.raises(ValueError):
            f()

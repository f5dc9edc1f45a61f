"""Rotary positions, root-mean-square norm and the norm in front of a W8A8 layer on the GPU, against the float64 oracle.

Tolerances.  A result in bf16 is off by at most half a step, 2^-8 of its size.  In fp32 before that: the mean of squares is
a tree of at most 2^-20 of its size (chains of up to 32 terms per thread, then pairs), the reciprocal root, the factors and the
sine or cosine add a few 2^-23 each: together below 2^-19 of the terms that are added up, which the oracle gives as `scale`
where they can cancel.  Sums over tokens (a weight's gradient): at most 2^-15 of the sum of the terms' sizes for the lengths here
(a chain of a team's tokens, at most a few dozen here, then two short trees)."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2512_16093_amd import binding as sla

pytestmark = pytest.mark.gpu

HALF, F32, SUMS = 2.0 ** -8, 2.0 ** -19, 2.0 ** -15
PAIRS, THETA = (22, 21, 21), (10000.0,) * 3


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(r, shape, amp=1.0):
    return torch.from_numpy((amp * r.standard_normal(shape)).astype(np.float32)).bfloat16()


def _near(got, want, scale, what):
    bad = np.abs(_np(got) - want) > HALF * np.abs(want) + F32 * scale + 1e-37
    assert not bad.any(), "%s: %d of %d off, worst %.3e" % (what, bad.sum(), bad.size, np.abs(_np(got) - want).max())


def _layouts(x, kind):
    """x [B, H, N, d] on the GPU in one of the memory orders the library takes, and whatever lies around it."""
    B, H, N, d = x.shape
    if kind == "contiguous":
        return x.cuda(), None
    if kind == "token":
        return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3), None
    around = torch.full((B, N, 3, H, d), 7.0, dtype=torch.bfloat16, device="cuda")      # one of three in a packed projection
    around[:, :, 1] = x.permute(0, 2, 1, 3).cuda()
    return around[:, :, 1].permute(0, 2, 1, 3), around


ROPE = [  # B, H, Hk, N, norm, pairing, memory order, positions per sample
    (1, 1, 1, 1, "none", "interleaved", "contiguous", False),
    (2, 3, 3, 5, "none", "halves", "token", True),
    (1, 12, 12, 257, "token", "interleaved", "packed", False),
    (2, 4, 4, 33, "head", "halves", "packed", True),
    (1, 16, 2, 67, "token", "halves", "token", False),
    (1, 5, 17, 19, "head", "interleaved", "token", False),
    (1, 17, 5, 31, "token", "interleaved", "contiguous", False),
    (1, 32, 32, 9, "token", "interleaved", "packed", False),
    (3, 40, 40, 11, "token", "interleaved", "packed", True),
    (1, 40, 8, 13, "head", "halves", "contiguous", False),
    (1, 64, 64, 6, "token", "halves", "token", False),
    (1, 49, 1, 7, "none", "interleaved", "token", False),
    (1, 8, 8, 4100, "head", "interleaved", "token", False),      # more tokens than the backward pass has teams
    (1, 20, 20, 1100, "token", "interleaved", "token", False),
]


def _rope_case(B, H, Hk, N, norm, pairing, order, per_sample):
    r = np.random.default_rng([B, H, Hk, N])
    pos = r.integers(-(1 << 31), 1 << 31, (B if per_sample else 1, N, 3))
    pos[:, ::2] = r.integers(0, 90, pos[:, ::2].shape)
    x = [_bf16(r, (B, h, N, 128), 1.7) for h in (H, Hk)]
    width = lambda h: 128 if norm == "head" else h * 128
    w = [None if norm == "none" else (1 + 0.2 * _bf16(r, width(h))).bfloat16() for h in (H, Hk)]
    ang = np.broadcast_to(bo.angles(pos, PAIRS, THETA), (B, N, 64))
    p = torch.from_numpy(pos.astype(np.int32)).cuda()
    return r, x, w, ang, (p if per_sample else p[0].contiguous()), sla.rope_make_plan(PAIRS, THETA[0], pairing)


@pytest.mark.parametrize("B,H,Hk,N,norm,pairing,order,per_sample", ROPE)
def test_rope_forward(B, H, Hk, N, norm, pairing, order, per_sample):
    r, x, w, ang, pos, plan = _rope_case(B, H, Hk, N, norm, pairing, order, per_sample)
    g = [_layouts(t, order) for t in x]
    outs = [_layouts(torch.zeros(t.shape, dtype=torch.bfloat16), order) for t in x]
    wg = [None if t is None else t.cuda() for t in w]
    got = sla.rope_qk_fwd(g[0][0], g[1][0], pos, plan, wg[0], wg[1], norm, 1e-6, outs[0][0], outs[1][0])
    torch.cuda.synchronize()
    for i, name in enumerate("qk"):
        w64 = None if w[i] is None else _np(w[i])
        want = bo.rope_fwd(_np(x[i]), ang, pairing, w64, norm)
        size = np.abs(bo.rope_fwd(_np(x[i]), ang * 0, pairing, w64, norm))      # the numbers that are turned
        lo, hi = bo.pair_channels(pairing)
        scale = np.empty_like(size)
        scale[..., lo] = scale[..., hi] = size[..., lo] + size[..., hi]
        _near(got[i], want, scale, name)
        if i == 0:
            near_q = lambda y, what, want=want, scale=scale: _near(y, want, scale, what)
        assert torch.equal(g[i][0].cpu(), x[i])                                 # inputs as they were
        if outs[i][1] is not None:
            assert (outs[i][1][:, :, 0] == 7).all() and (outs[i][1][:, :, 2] == 7).all()
    alone = sla.rope_qk_fwd(g[0][0], None, pos, plan, wg[0], None, norm)        # q alone, into a tensor of the binding's own
    assert alone[1] is None
    near_q(alone[0], "q alone")


@pytest.mark.parametrize("B,H,Hk,N,norm,pairing,order,per_sample", ROPE)
def test_rope_backward(B, H, Hk, N, norm, pairing, order, per_sample):
    r, x, w, ang, pos, plan = _rope_case(B, H, Hk, N, norm, pairing, order, per_sample)
    dy = [_bf16(r, t.shape, 0.01) for t in x]
    g, dg = [_layouts(t, order)[0] for t in x], [_layouts(t, order)[0] for t in dy]
    outs = [_layouts(torch.zeros(t.shape, dtype=torch.bfloat16), order) for t in x]
    wg = [None if t is None else t.cuda() for t in w]
    call = lambda **kw: sla.rope_qk_bwd(dg[0], dg[1], pos, plan, g[0], g[1], wg[0], wg[1], norm, 1e-6, **kw)
    got = call(dq=outs[0][0], dk=outs[1][0])
    again = call()
    torch.cuda.synchronize()
    for i, name in enumerate(("dq", "dk")):
        dx, dw, scale = bo.rope_bwd(_np(dy[i]), _np(x[i]), ang, pairing, None if w[i] is None else _np(w[i]), norm)
        _near(got[i], dx, scale, name)
        assert torch.equal(got[i].cpu(), again[i].cpu())
        if outs[i][1] is not None:
            assert (outs[i][1][:, :, 0] == 7).all() and (outs[i][1][:, :, 2] == 7).all()
        if norm == "none":
            assert got[2 + i] is None
            continue
        assert torch.equal(got[2 + i], again[2 + i])
        a64 = np.abs(_np(x[i]))
        r64 = np.broadcast_to(1 / np.sqrt((a64 ** 2).mean((3,) if norm == "head" else (1, 3), keepdims=True) + 1e-6), a64.shape)
        lo, hi = bo.pair_channels(pairing)
        size = np.empty_like(a64)
        size[..., lo] = size[..., hi] = np.abs(_np(dy[i]))[..., lo] + np.abs(_np(dy[i]))[..., hi]
        terms = (size * a64 * r64).sum((0, 1, 2) if norm == "head" else (0, 2)).reshape(-1)
        err = np.abs(_np(got[2 + i]) - dw)
        assert (err <= SUMS * terms).all(), (name, float((err / terms).max()))
    if norm != "none":
        assert call(want_dw=False)[2:] == (None, None)


def test_rope_without_a_weight_and_with_axes_left_out():
    r = np.random.default_rng(5)
    x, pos = _bf16(r, (1, 6, 21, 128)), r.integers(0, 1000, (1, 21, 3))
    for pairs, theta in (((64, 0, 0), (10000.0, 1.0, 1.0)), ((0, 10, 54), (1.0, 100.0, 1e12))):
        plan = sla.rope_make_plan(pairs, theta)
        ang = bo.angles(pos, pairs, theta)
        p = torch.from_numpy(pos.astype(np.int32)).cuda()
        got = sla.rope_qk_fwd(x.cuda(), None, p, plan, norm="token", eps=1e-3)[0]
        want = bo.rope_fwd(_np(x), ang, "interleaved", None, "token", 1e-3)
        _near(got, want, 2 * np.abs(want).max(), "unit weights")
        dy = _bf16(r, x.shape)
        dx, _, scale = bo.rope_bwd(_np(dy), _np(x), ang, "interleaved", None, "token", 1e-3)
        _near(sla.rope_qk_bwd(dy.cuda(), None, p, plan, q=x.cuda(), norm="token", eps=1e-3)[0], dx, scale, "gradient")


NORM = [(1, 8), (1, 128), (3, 520), (129, 1536), (5, 1000), (70, 2048), (33, 2056), (257, 5120), (19, 6144 - 8), (6, 8192), (11, 8200),
        (4, 13824), (3, 16384), (5000, 64), (1300, 4104)]


@pytest.mark.parametrize("M,K", NORM)
@pytest.mark.parametrize("with_res", [False, True])
def test_norm_forward_and_backward(M, K, with_res):
    r = np.random.default_rng([M, K])
    x, res, dy, dh = (_bf16(r, (M, K), a) for a in (3.0, 0.5, 0.01, 0.01))
    x[0] = 0                                       # a token of zeros: 1 / sqrt(eps) times nothing
    if with_res:
        res[0] = 0
    w = (1 + 0.2 * _bf16(r, K)).bfloat16() if K != 1000 else None
    wg, w64 = (None, None) if w is None else (w.cuda(), _np(w))
    y, h = sla.norm_rms_fwd(x.cuda(), wg, res.cuda() if with_res else None)
    want_h = (x.float() + res.float()).bfloat16() if with_res else x
    assert torch.equal(h.cpu(), want_h)
    want = bo.norm_fwd(_np(want_h), w64, 1e-6)
    _near(y, want, np.abs(want), "y")
    got = sla.norm_rms_bwd(dy.cuda(), h, wg, dh.cuda() if with_res else None)
    again = sla.norm_rms_bwd(dy.cuda(), h, wg, dh.cuda() if with_res else None)
    dx, dw, scale = bo.norm_bwd(_np(dy), _np(want_h), w64, _np(dh) if with_res else None, 1e-6)
    _near(got[0], dx, scale, "dx")
    h64 = np.abs(_np(want_h))
    terms = (np.abs(_np(dy)) * h64 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-6)).sum(0)
    assert (np.abs(_np(got[1]) - dw) <= SUMS * terms + 1e-37).all()
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    assert sla.norm_rms_bwd(dy.cuda(), h, wg, want_dw=False)[1] is None


def _codes(ws, M, K):
    codes, scales = sla.w8a8_debug_unpack(ws, False, M, K)
    return _np(codes), _np(scales)


@pytest.mark.parametrize("M,K", [(1, 128), (1, 5120), (7, 384), (127, 1536), (128, 256), (129, 640), (257, 5120), (300, 13824), (1025, 2048),
                                 (64, 16384)])
@pytest.mark.parametrize("with_res", [False, True])
def test_norm_quantised_for_a_linear_layer(M, K, with_res):
    r = np.random.default_rng([M, K, 1])
    x, res = _bf16(r, (M, K), 3.0), _bf16(r, (M, K), 0.5)
    x[:, :: 37] *= 20
    if M > 128:
        x[0:128, 0:128] = 0                        # a block of zeros: scale 1, codes 0
        res[0:128, 0:128] = 0
    w = (1 + 0.2 * _bf16(r, K)).bfloat16()
    ws, h = sla.w8a8_norm_quantize_act(x.cuda(), w.cuda(), res.cuda() if with_res else None)
    want_h = (x.float() + res.float()).bfloat16() if with_res else x
    assert torch.equal(h.cpu(), want_h)
    n = bo.norm_fwd(_np(want_h), _np(w), 1e-6)
    codes, scales = _codes(ws, M, K)
    rows = -(-M // 128)
    blocks = np.zeros((rows * 128, K))
    blocks[:M] = n
    amax = np.abs(blocks.reshape(rows, 128, K // 128, 128)).max((1, 3))
    want_scales = np.where(amax > 0, amax / 127, 1.0)
    assert (np.abs(scales - want_scales) <= F32 * want_scales).all()
    # a code is the nearest integer to n over the scale: off by half a step, and what fp32 adds at 127 steps
    steps = n / np.repeat(np.repeat(want_scales, 128, 0), 128, 1)[:M]
    assert (np.abs(codes - steps) <= 0.5 + 127 * 2 * F32).all()
    assert np.abs(codes).max() == 127


@pytest.mark.parametrize("M", [2, 5, 200])
def test_norm_quantised_without_a_weight(M):
    x = _bf16(np.random.default_rng(M), (M, 640), 2.0).cuda()
    ones = torch.ones(640, dtype=torch.bfloat16, device="cuda")
    a, b = (_codes(sla.w8a8_norm_quantize_act(x, w)[0], M, 640) for w in (None, ones))
    assert all((u == v).all() for u, v in zip(a, b))


@pytest.mark.parametrize("M,N,K", [(1, 256, 512), (130, 384, 1536), (1500, 1536, 640)])
def test_norm_linear(M, N, K):
    r = np.random.default_rng([M, N, K])
    x, res, wt = _bf16(r, (M, K), 2.0).cuda(), _bf16(r, (M, K), 0.5).cuda(), _bf16(r, (N, K), K ** -0.5).cuda()
    w, bias = (1 + 0.2 * _bf16(r, K)).bfloat16().cuda(), _bf16(r, N, 0.1).cuda()
    wq = sla.w8a8_quantize_weight(wt)
    y, h = sla.w8a8_norm_linear_fwd(x, w, wq, N, res=res, bias=bias)
    ws, h2 = sla.w8a8_norm_quantize_act(x, w, res=res)
    assert torch.equal(y, sla.w8a8_gemm_fwd(ws, wq, M, N, K, bias=bias)) and torch.equal(h, h2)
    # against the product in 64 bits of the codes' values: the accumulation's bound (two steps a block of 128 features of the
    # largest block, include/w8a8.h) and the rounding of the result
    codes, scales = _codes(ws, M, K)
    wc, wsc = [_np(t) for t in sla.w8a8_debug_unpack(wq, True, N, K)]
    step = np.repeat(np.repeat(scales, 128, 0), 128, 1)[:M]
    want = (codes * step) @ (wc * np.repeat(np.repeat(wsc, 128, 0), 128, 1)).T + _np(bias)
    slack = 2 * (K // 128) * scales.max() * wsc.max()
    assert (np.abs(_np(y) - want) <= HALF * np.abs(want) + slack).all()


def test_another_stream_and_a_captured_graph():
    """The calls on a side stream, and recorded into a graph that is replayed on fresh inputs with eager work between."""
    r = np.random.default_rng(9)
    H, N, K = 12, 130, 1536
    plan = sla.rope_make_plan()
    pos = torch.from_numpy(r.integers(0, 50, (N, 3)).astype(np.int32)).cuda()
    x, res, dy = (_bf16(r, (N, K)).cuda() for _ in range(3))
    w = _bf16(r, K).cuda()
    wq = sla.w8a8_quantize_weight(_bf16(r, (256, K), 0.03).cuda())

    def calls():
        y, h = sla.w8a8_norm_linear_fwd(x, w, wq, 256, res=res)
        heads = lambda t: t.view(1, N, H, 128).permute(0, 2, 1, 3)
        q, k = sla.rope_qk_fwd(heads(x), heads(h), pos, plan, w, w, "token")
        back = sla.rope_qk_bwd(q, k, pos, plan, heads(x), heads(h), w, w, "token")
        return [y, h, q, k, *back, *sla.norm_rms_fwd(x, w, res), *sla.norm_rms_bwd(dy, x, w, dh=res)]

    eager = [t.clone() for t in calls()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for seed in range(3):
        r = np.random.default_rng([10, seed])
        for t in (x, res, dy):
            t.copy_(_bf16(r, (N, K)))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(replayed, calls())), seed

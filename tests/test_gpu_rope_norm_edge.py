"""Rotary positions and root-mean-square norm at the ends of what their headers allow, on the GPU against the float64 oracle.
Tolerances as in test_gpu_rope_norm.py: half a step of bf16, and 2^-19 of the terms for what comes before in fp32."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2512_16093_amd import binding as sla

pytestmark = pytest.mark.gpu

HALF, F32, SUMS = 2.0 ** -8, 2.0 ** -19, 2.0 ** -15


def _np(t):
    return t.detach().double().cpu().numpy()


def _bf16(r, shape, amp=1.0):
    return torch.from_numpy((amp * r.standard_normal(shape)).astype(np.float32)).bfloat16()


def _near(got, want, scale, what):
    bad = ~(np.abs(_np(got) - want) <= HALF * np.abs(want) + F32 * scale)
    assert not bad.any(), "%s: %d of %d off" % (what, bad.sum(), bad.size)


TINY_EPS = 1.2e-38       # nearly the smallest that is taken


@pytest.mark.parametrize("M,K", [(5, 128), (9, 1536), (3, 5120)])
def test_gradient_of_the_norm_of_tiny_rows(M, K):
    """Rows of 2e-18 with next to no eps: r is 5e17, r^3 beyond fp32, the gradient (5e21) is not."""
    r = np.random.default_rng([M, K, 2])
    x = _bf16(r, (M, K), 2e-18)
    dy = (1e4 * x.float().sign() + 1e3 * _bf16(r, (M, K)).float()).bfloat16()      # (along x: the mean of x w dy is as large as it can be)
    w = (1 + 0.2 * _bf16(r, K)).bfloat16()
    dx, dw, scale = bo.norm_bwd(_np(dy), _np(x), _np(w), None, TINY_EPS)
    got = sla.norm_rms_bwd(dy.cuda(), x.cuda(), w.cuda(), eps=TINY_EPS)
    _near(got[0], dx, scale, "dx")
    x64 = np.abs(_np(x))
    terms = (np.abs(_np(dy)) * x64 / np.sqrt((x64 ** 2).mean(1, keepdims=True) + TINY_EPS)).sum(0)
    assert (np.abs(_np(got[1]) - dw) <= SUMS * terms).all()


@pytest.mark.parametrize("H,norm,pairing", [(3, "head", "interleaved"), (12, "token", "halves"), (20, "token", "interleaved"), (20, "head", "halves")])
def test_gradient_of_the_rotation_of_tiny_heads(H, norm, pairing):
    r = np.random.default_rng([H, 3])
    x = _bf16(r, (1, H, 7, 128), 2e-18)
    pos = np.zeros((1, 7, 3), dtype=np.int64)
    pos[:, 3:] = r.integers(0, 90, (1, 4, 3))
    ang = bo.angles(pos, (22, 21, 21), (10000.0,) * 3)
    dy = torch.from_numpy(bo.rotate(1e4 * np.sign(_np(x)), ang[:, None], pairing)).bfloat16()
    w = (1 + 0.2 * _bf16(r, 128 if norm == "head" else H * 128)).bfloat16()
    dx, _, scale = bo.rope_bwd(_np(dy), _np(x), ang, pairing, _np(w), norm, TINY_EPS)
    p = torch.from_numpy(pos[0].astype(np.int32)).cuda()
    plan = sla.rope_make_plan((22, 21, 21), 10000.0, pairing)
    got = sla.rope_qk_bwd(dy.cuda(), None, p, plan, q=x.cuda(), q_weight=w.cuda(), norm=norm, eps=TINY_EPS)
    _near(got[0], dx, scale, "dx")
    assert torch.isfinite(got[2]).all()


def _large(r, shape):
    """Values up to 1e17, half of them of that size: what the headers promise of every width."""
    x = 1e17 * r.choice((-1.0, 1.0), shape) * np.where(r.random(shape) < 0.5, 1.0, r.random(shape))
    return torch.from_numpy((x * (1 - 2.0 ** -7)).astype(np.float32)).bfloat16()


@pytest.mark.parametrize("M,K", [(3, 1024), (5, 5120), (2, 16384)])
@pytest.mark.parametrize("with_res", [False, True])
def test_norm_of_the_largest_values(M, K, with_res):
    r = np.random.default_rng([M, K, 4])
    x, w, dy = _large(r, (M, K)), (1 + 0.2 * _bf16(r, K)).bfloat16(), _bf16(r, (M, K))
    res = (x.float() * -0.25).bfloat16() if with_res else None
    h = x if res is None else (x.float() + res.float()).bfloat16()
    rg = None if res is None else res.cuda()
    n = bo.norm_fwd(_np(h), _np(w), 1e-6)
    y, got_h = sla.norm_rms_fwd(x.cuda(), w.cuda(), rg)
    assert torch.equal(got_h.cpu(), h)
    _near(y, n, np.abs(n), "y")
    dx, _, scale = bo.norm_bwd(_np(dy), _np(h), _np(w), None, 1e-6)
    _near(sla.norm_rms_bwd(dy.cuda(), h.cuda(), w.cuda())[0], dx, scale, "dx")
    ws, _ = sla.w8a8_norm_quantize_act(x.cuda(), w.cuda(), rg)
    codes, scales = (_np(t) for t in sla.w8a8_debug_unpack(ws, False, M, K))
    want = np.abs(n.reshape(M, K // 128, 128)).max((0, 2)) / 127
    assert (np.abs(scales[0] - want) <= F32 * want).all()
    assert (np.abs(codes - n / np.repeat(want, 128)) <= 0.5 + 127 * 2 * F32).all()


@pytest.mark.parametrize("H,norm", [(3, "head"), (12, "token"), (64, "token"), (64, "head")])
def test_rotation_of_the_largest_values(H, norm):
    r = np.random.default_rng([H, 5])
    x, w, dy = _large(r, (1, H, 5, 128)), (1 + 0.2 * _bf16(r, 128 if norm == "head" else H * 128)).bfloat16(), _bf16(r, (1, H, 5, 128))
    pos = r.integers(0, 90, (1, 5, 3))
    ang, p, plan = bo.angles(pos, (22, 21, 21), (10000.0,) * 3), torch.from_numpy(pos[0].astype(np.int32)).cuda(), sla.rope_make_plan()
    want = bo.rope_fwd(_np(x), ang, "interleaved", _np(w), norm)
    size = np.abs(bo.rope_fwd(_np(x), ang * 0, "interleaved", _np(w), norm))
    y = sla.rope_qk_fwd(x.cuda(), None, p, plan, w.cuda(), norm=norm)[0]
    _near(y, want, np.repeat(size[..., 0::2] + size[..., 1::2], 2, -1), "y")
    dx, _, scale = bo.rope_bwd(_np(dy), _np(x), ang, "interleaved", _np(w), norm)
    got = sla.rope_qk_bwd(dy.cuda(), None, p, plan, q=x.cuda(), q_weight=w.cuda(), norm=norm)
    _near(got[0], dx, scale, "dx")


@pytest.mark.parametrize("M,K", [(2, 384), (3, 1536), (4, 128), (4, 5120), (4, 8192), (5, 8192), (5, 384), (1, 13824), (4, 16384)])
@pytest.mark.parametrize("with_res", [False, True])
def test_few_rows_quantised_for_a_linear_layer(M, K, with_res):
    """Either side of the rule for few rows; every row has an amplitude of its own, so that another row's factor would show.  A code
    is off by half a step and what fp32 adds at 127 steps."""
    r = np.random.default_rng([M, K, 6])
    amp = np.array([3.0, 0.01, 200.0, 0.5, 17.0])[:M, None]
    x, res = (torch.from_numpy((a * amp * r.standard_normal((M, K))).astype(np.float32)).bfloat16() for a in (1.0, 0.3))
    w = (1 + 0.2 * _bf16(r, K)).bfloat16()
    h = (x.float() + res.float()).bfloat16() if with_res else x
    into = torch.full((M, K), float("nan"), dtype=torch.bfloat16, device="cuda") if with_res else None
    ws, got_h = sla.w8a8_norm_quantize_act(x.cuda(), w.cuda(), res.cuda() if with_res else None, h=into)
    assert torch.equal(got_h.cpu(), h)
    n = bo.norm_fwd(_np(h), _np(w), 1e-6)
    codes, scales = (_np(t) for t in sla.w8a8_debug_unpack(ws, False, M, K))
    want = np.abs(n.reshape(M, K // 128, 128)).max((0, 2)) / 127
    assert (np.abs(scales[0] - want) <= F32 * want).all()
    assert (np.abs(codes - n / np.repeat(want, 128)) <= 0.5 + 127 * 2 * F32).all()
    # and through the layer: the product of these codes
    wq = sla.w8a8_quantize_weight(_bf16(r, (256, K), K ** -0.5).cuda())
    y, _ = sla.w8a8_norm_linear_fwd(x.cuda(), w.cuda(), wq, 256, res=res.cuda() if with_res else None)
    assert torch.equal(y, sla.w8a8_gemm_fwd(ws, wq, M, 256, K))


@pytest.mark.parametrize("M", [1, 3, 4, 5])
def test_one_row_and_few_of_the_norm(M):
    """Single tokens at a model's widths, forward and backward."""
    for K in (1536, 5120, 8960):
        r = np.random.default_rng([M, K, 7])
        x, res, dy, dh = (_bf16(r, (M, K), a) for a in (3.0, 0.5, 0.01, 0.01))
        w = (1 + 0.2 * _bf16(r, K)).bfloat16()
        y, h = sla.norm_rms_fwd(x.cuda(), w.cuda(), res.cuda())
        assert torch.equal(h.cpu(), (x.float() + res.float()).bfloat16())
        want = bo.norm_fwd(_np(h), _np(w), 1e-6)
        _near(y, want, np.abs(want), "y")
        got = sla.norm_rms_bwd(dy.cuda(), h, w.cuda(), dh.cuda())
        dx, dw, scale = bo.norm_bwd(_np(dy), _np(h), _np(w), _np(dh), 1e-6)
        _near(got[0], dx, scale, "dx")
        h64 = np.abs(_np(h))
        terms = (np.abs(_np(dy)) * h64 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-6)).sum(0)
        assert (np.abs(_np(got[1]) - dw) <= SUMS * terms).all()

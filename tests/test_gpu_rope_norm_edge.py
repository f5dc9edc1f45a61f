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

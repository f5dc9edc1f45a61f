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

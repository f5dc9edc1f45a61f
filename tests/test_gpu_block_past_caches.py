"""Norm and rotation of tensors that do not fit the memory-side cache (256 MiB together): kernels of their own, which load and
store past the caches.  Every width of a team is compared with the same rows taken in parts small enough for the other kernels, bit for
bit, and sampled rows with float64; and a memory of more than 4 GB whose last keys decide."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2512_16093_amd import binding as sla

pytestmark = pytest.mark.gpu
U, F32, SUMS = 2.0 ** -8, 2.0 ** -19, 2.0 ** -15       # (test_gpu_rope_norm.py)
CACHE = 256 << 20
PARTS = 8


def _np(t):
    return t.detach().double().cpu().numpy()


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _normal(shape, seed, amp=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").mul_(amp).bfloat16()


@pytest.mark.parametrize("H", [4, 8, 12, 16, 32, 40, 64])          # one for each width of a token's team
@pytest.mark.parametrize("norm", ["none", "head", "token"])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_rotation_past_the_caches(H, norm, pairing):
    N = CACHE // (2 * 2 * 2 * H * 128) // 64 * 64 + 67             # q and k, in and out: just beyond; a rest in the last workgroup
    q, k = (_normal((1, N, H, 128), s, 1.7).permute(0, 2, 1, 3) for s in (1, 2))
    n = torch.arange(N, device="cuda")
    pos = torch.stack((n // 3600, n // 80 % 45, n % 80), 1).int().contiguous()
    w = [None if norm == "none" else (1 + 0.2 * _normal((128 if norm == "head" else H * 128,), s)).bfloat16() for s in (3, 4)]
    plan = sla.rope_make_plan(pairing=pairing)
    y = sla.rope_qk_fwd(q, k, pos, plan, w[0], w[1], norm)
    back = sla.rope_qk_bwd(y[0], y[1], pos, plan, q, k, w[0], w[1], norm)      # (of its own output: sums of one sign for the weights)
    dw = [0, 0]
    for part in torch.arange(N, device="cuda").chunk(PARTS):
        s = slice(int(part[0]), int(part[-1]) + 1)
        a = [t[:, :, s] for t in (q, k)]
        p = pos[s].contiguous()
        small = sla.rope_qk_fwd(a[0], a[1], p, plan, w[0], w[1], norm)
        grads = sla.rope_qk_bwd(small[0], small[1], p, plan, a[0], a[1], w[0], w[1], norm)
        for i in range(2):
            assert torch.equal(small[i], y[i][:, :, s]) and torch.equal(grads[i], back[i][:, :, s])
            if norm != "none":
                dw[i] = dw[i] + grads[2 + i].double()
    some = torch.tensor([0, 5, N // 2, N - 1], device="cuda")
    ang = bo.angles(pos[some].cpu().numpy()[None], (22, 21, 21), (10000.0,) * 3)
    lo, hi = bo.pair_channels(pairing)
    for i, src in enumerate((q, k)):
        x64, y64, w64 = _np(src[:, :, some]), _np(y[i][:, :, some]), None if w[i] is None else _np(w[i])
        want = bo.rope_fwd(x64, ang, pairing, w64, norm)
        size = np.abs(bo.rope_fwd(x64, ang * 0, pairing, w64, norm))
        scale = np.empty_like(size)
        scale[..., lo] = scale[..., hi] = size[..., lo] + size[..., hi]
        assert (np.abs(y64 - want) <= U * np.abs(want) + F32 * scale).all()
        dx, _, scale = bo.rope_bwd(y64, x64, ang, pairing, w64, norm)
        assert (np.abs(_np(back[i][:, :, some]) - dx) <= U * np.abs(dx) + F32 * scale).all()
        if norm != "none":
            assert ((back[2 + i].double() - dw[i]).abs() <= 2 * SUMS * dw[i].abs()).all()


@pytest.mark.parametrize("K", [512, 1024, 1536, 2048, 4096, 5120, 6144, 8192, 13824])     # one for each width of a row's team
@pytest.mark.parametrize("with_res", [False, True])
def test_norm_past_the_caches(K, with_res):
    M = CACHE // (2 * 2 * K) // 1024 * 1024 + 1024 + 61
    x, dy = _normal((M, K), 1, 2.0), _normal((M, K), 2)
    res = _normal((M, K), 3, 0.5) if with_res else None
    w = (1 + 0.2 * _normal((K,), 4)).bfloat16()
    cut = lambda t, s: None if t is None else t[s]
    y, h = sla.norm_rms_fwd(x, w, res)
    dx, dw = sla.norm_rms_bwd(y, h, w, res)
    total = 0
    for m0 in range(0, M, 1024 * (M // 1024 // PARTS + 1)):
        s = slice(m0, min(M, m0 + 1024 * (M // 1024 // PARTS + 1)))
        small = sla.norm_rms_fwd(x[s], w, cut(res, s))
        grads = sla.norm_rms_bwd(y[s], h[s], w, cut(res, s))
        assert torch.equal(small[0], y[s]) and torch.equal(small[1], h[s]) and torch.equal(grads[0], dx[s])
        total = total + grads[1].double()
    assert ((dw.double() - total).abs() <= 2 * SUMS * total.abs()).all()
    some = torch.tensor([0, 3, M // 2, M - 1], device="cuda")
    want = bo.norm_fwd(_np(h[some]), _np(w), 1e-6)
    assert (np.abs(_np(y[some]) - want) <= (U + F32) * np.abs(want)).all()
    want, _, scale = bo.norm_bwd(_np(y[some]), _np(h[some]), _np(w), None if res is None else _np(res[some]), 1e-6)
    assert (np.abs(_np(dx[some]) - want) <= U * np.abs(want) + F32 * scale).all()


@pytest.mark.parametrize("K", [1536, 5120])
@pytest.mark.parametrize("with_res", [False, True])
def test_norm_quantised_past_the_caches(K, with_res):
    M = CACHE // (2 * K) // 1024 * 1024 + 1024 + 61                            # (h alone is beyond)
    x, w = _normal((M, K), 1, 2.0), (1 + 0.2 * _normal((K,), 4)).bfloat16()
    res = _normal((M, K), 3, 0.5) if with_res else None
    ws, h = sla.w8a8_norm_quantize_act(x, w, res)
    codes, scales = sla.w8a8_debug_unpack(ws, False, M, K)
    step = 1024 * (M // 1024 // PARTS + 1)
    for m0 in range(0, M, step):
        s = slice(m0, min(M, m0 + step))
        ws2, h2 = sla.w8a8_norm_quantize_act(x[s], w, None if res is None else res[s])
        c2, s2 = sla.w8a8_debug_unpack(ws2, False, h2.shape[0], K)
        assert torch.equal(h2, h[s]) and torch.equal(c2, codes[s]) and torch.equal(s2, scales[m0 // 128:m0 // 128 + s2.shape[0]])


def test_the_last_keys_of_a_memory_beyond_4_gb_decide():
    """The last key that counts is along one query, the one before along another: those rows are these keys' values.  The one behind
    the last would win by far, and does not count.  Scores: 3 |q|^2 / 128^(1/2), 136, 85 at least here; the others' log-sum-exp is
    below 17 + 12 (17 million of a variance of 4), so that all of them weigh less than e^-50."""
    Nk = 17_000_000
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.empty((1, 1, Nk, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (k, v):
        for part in t.view(-1).split(1 << 27):
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    q = _normal((1, 2, 3, 128), 3, 2.0)
    k[0, 0, -2], k[0, 0, -3], k[0, 0, -1] = 3 * q[0, 0, 0], 3 * q[0, 1, 2], 100 * q[0, 0, 0]
    assert float((3 * q.double().pow(2).sum(3) * 128 ** -0.5).min()) > 85
    lens = torch.tensor([Nk - 1], dtype=torch.int32, device="cuda")
    out, lse = sla.xattn_fwd(q, k, v, k_lens=lens, want_lse=True)
    for (h, n), row in (((0, 0), -2), ((1, 2), -3)):
        assert torch.equal(out[0, h, n], v[0, 0, row])
        want = float(q[0, h, n].double() @ k[0, 0, row].double()) * 128 ** -0.5
        assert abs(float(lse[0, h, n]) - want) <= 2.0 ** -20 * (1 + want)
